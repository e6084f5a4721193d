"""How many bits the gradient of packed attention keeps where few keys, small gradients or long sequences ask for them, against the
definition in 64 bits.  h is half a step of the type relative to the value (finfo.eps / 2)."""
import numpy as np
import pytest
import torch

from paper_2409_09708_b200 import synth

TYPES = [torch.bfloat16, torch.float16]
NAMES = ["bf16", "f16"]


@pytest.fixture(scope="module")
def lib():
    from paper_2409_09708_b200 import binding
    return binding


def both_ways(lib, q, k, v, da, lengths, heads, kv_heads, causal=False, scale=None):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    plan = lib.make_packed_plan([0] + np.cumsum(lengths).tolist(), dev_status=status)
    a, lse = lib.elsa_packed_attention(q, k, v, plan, heads, kv_heads, causal=causal, scale=scale, want_lse=True, dev_status=status)
    grads = lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, kv_heads, causal=causal, scale=scale, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return a, dict(zip(("dq", "dk", "dv"), grads))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("lengths", [[64], [65], [100, 129], [300, 1, 70], [2500]], ids=lambda l: "-".join(map(str, l)))
def test_first_rows_of_causal_sequences(lib, lengths, D, dtype):
    """The first 64 rows have all their keys in the first tile of the walk, and the fewest keys: their delta carries no rounding of a.
    da is zero in the other rows, so that dk is theirs alone.  With d for what fp32 leaves (2e-5: lse of up to 24 binary orders three
    times rounded, 4e-6, two scores of up to 6 summed in another order, 2e-6, and the approximate exponential, 3e-7, on a p that all
    of them scale) and t = 2^-24 for a ds of fp16 below its normal range
      E_ds = (h + d) |ds| + d p (sum |da| |v| + |delta|) + t      dq: h |dq| + |scale| sum E_ds |k|      dk: h |dk| + |scale| sum E_ds |q|."""
    h, d, t = torch.finfo(dtype).eps / 2, 2e-5, 2.0 ** -24 if dtype == torch.float16 else 0.0
    heads, rows = 2, sum(lengths)
    q, k, v = synth.randn((rows, 3 * heads * D), 41, 1.0, dtype, "cuda").split(heads * D, dim=1)
    da = synth.randn((rows, heads * D), 42, 1.0, dtype, "cuda")
    starts = [0] + np.cumsum(lengths).tolist()
    for b, e in zip(starts, starts[1:]):
        da[min(b + 64, e):e] = 0
    _, got = both_ways(lib, q, k, v, da, lengths, heads, heads, causal=True)
    scale = D ** -0.5
    for b, e in zip(starts, starts[1:]):
        r = slice(b, min(b + 64, e))
        n = r.stop - b
        for i in range(heads):
            c = slice(i * D, (i + 1) * D)
            Q, K, V, G = (x[r, c].double() for x in (q, k, v, da))
            p = torch.softmax((scale * Q @ K.t()).masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -torch.inf), dim=1)
            dp = G @ V.t()
            delta = (p * dp).sum(1, keepdim=True)
            ds = p * (dp - delta)
            eds = (h + d) * ds.abs() + d * p * (G.abs() @ V.abs().t() + delta.abs()) + t * (p > 0)
            for name, ref, tol in (("dq", scale * ds @ K, scale * eds @ K.abs()), ("dk", scale * ds.t() @ Q, scale * eds.t() @ Q.abs())):
                off = (got[name][r, c].double() - ref).abs() - h * ref.abs() - tol - 1e-7
                assert (off <= 0).all(), "%s of head %d: %g above what is allowed" % (name, i, off.max())
