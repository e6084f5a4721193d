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


def exact(q, k, v, da, scale, heads=1, kv_heads=1, error=None):
    """dq, dk and dv of one sequence without a mask in 64 bits, some query rows at a time; error: what error(ds, p, sum |da| |v|) in each
    ds may make of dq and dk instead."""
    D, n = q.shape[1] // heads, q.shape[0]
    q, k, v, da = (x.double() for x in (q, k, v, da))
    dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v))
    for i in range(heads):
        j = i // (heads // kv_heads)
        ci, cj = slice(i * D, (i + 1) * D), slice(j * D, (j + 1) * D)
        for b in range(0, n, 4096):
            r = slice(b, min(b + 4096, n))
            p = torch.softmax(scale * q[r, ci] @ k[:, cj].t(), dim=1)
            dp = da[r, ci] @ v[:, cj].t()
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            K, Q = k[:, cj], q[r, ci]
            if error is not None:
                ds, K, Q = error(ds, p, da[r, ci].abs() @ v[:, cj].abs().t()), K.abs(), Q.abs()
            dq[r, ci] = scale * ds @ K
            dk[:, cj] += scale * ds.t() @ Q
            dv[:, cj] += p.t() @ da[r, ci]
    return {"dq": dq, "dk": dk, "dv": dv}


# q and k 2^-10 and the scale 2^20 of ordinary ones: the scores are the same, dq and dk stand 2^10 higher above the type's lowest values.
SMALL, SCALE = 2.0 ** -10, 2.0 ** 17


@pytest.mark.gpu
@pytest.mark.parametrize("size", [0.5, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("n", [1000, 4096, 16384])
def test_small_gradients_of_long_sequences(lib, n, D, size):
    """fp16: the relative error does not depend on the size of da or the number of keys.  Random inputs: of independent roundings of at most
    h each a Frobenius norm shows no more than h; there are the output's, ds's (or p's) and, through delta, a's with the probabilities'
    in it: 4 h, and half a step, 2^-25, for each stored value below the type's normal range."""
    h = torch.finfo(torch.float16).eps / 2
    q, k = (synth.randn((n, D), 50 + i, SMALL, torch.float16, "cuda") for i in range(2))
    v, da = synth.randn((n, D), 52, 1.0, torch.float16, "cuda"), synth.randn((n, D), 53, size, torch.float16, "cuda")
    scale = SCALE * 8.0 / D ** 0.5
    _, got = both_ways(lib, q, k, v, da, [n], 1, 1, scale=scale)
    for name, ref in exact(q, k, v, da, scale).items():
        off = float((got[name].double() - ref).norm())
        assert off <= 4 * h * float(ref.norm()) + 2.0 ** -25 * ref.numel() ** 0.5, "%s: %g of %g" % (name, off, ref.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("lengths", [[1000], [50, 3000, 1], [9000]], ids=lambda l: "-".join(map(str, l)))
def test_a_power_of_two_passes_through(lib, lengths, D):
    """fp16: the gradient is linear in da.  With da 2^-24 of whole numbers (exact: steps of the lowest values) it is 2^-24 of theirs but for
    the rounding of what is stored: half a step of the one, h times the value, and of the other, at least 2^-25.  The products da . v are
    sums in fp32 whose bits are no power of two apart where the operands are below the normal range (the matrix unit lines them up by
    their exponents, which end there): up to 2e-5 of sum |da| |v| with its delta.  Two ds that near each other may round to neighbours,
    2 h |ds| apart.  So dq and dk may differ by |scale| sum (2 h |ds| + 4e-5 p sum |da| |v|) |k|, and |q|, besides.  Values that the larger da
    takes past 65504 (less 2 %, for what is rounded on the way) are left out: infinite is right for them."""
    h, rows, heads = torch.finfo(torch.float16).eps / 2, sum(lengths), 2
    q, k = (synth.randn((rows, w * D), 60 + i, SMALL, torch.float16, "cuda") for i, w in enumerate((heads, 1)))
    v = synth.randn((rows, D), 62, 1.0, torch.float16, "cuda")
    da = synth.randn((rows, heads * D), 63, 64.0, torch.float16, "cuda").float().round().clamp(-1024, 1024)
    scale = SCALE * 8.0 / D ** 0.5
    _, large = both_ways(lib, q, k, v, da.half(), lengths, heads, 1, scale=scale)
    _, small = both_ways(lib, q, k, v, (da * 2.0 ** -24).half(), lengths, heads, 1, scale=scale)
    starts = [0] + np.cumsum(lengths).tolist()
    for b, e in zip(starts, starts[1:]):
        r = slice(b, e)
        apart = exact(q[r], k[r], v[r], da[r], scale, heads, 1, lambda ds, p, dav: 2 * h * ds.abs() + 4e-5 * p * dav)
        for name, ref in exact(q[r], k[r], v[r], da[r], scale, heads, 1).items():
            x, y = large[name][r].double(), small[name][r].double() * 2.0 ** 24
            inside = ref.abs() < 64000.0
            more = apart[name] if name != "dv" else 0.0
            assert inside.double().mean() > 0.9 and torch.isfinite(y).all()
            near = (x - y).abs() <= 2 * h * x.abs() + 0.5 + more
            assert near[inside].all(), "%s: %g" % (name, (x - y)[inside].abs().max())


@pytest.mark.gpu
@pytest.mark.parametrize("D", [32, 64, 128])
def test_probabilities_below_the_type(lib, D):
    """fp16: half the keys have probabilities of two or three of the type's lowest steps, in every row alike, so that nothing averages
    out.  dv: h |dv| + (h + 2e-4) sum p |da| for the output, p and fp32, 2^-25 of it stored."""
    h, n = torch.finfo(torch.float16).eps / 2, 4096
    q, k = torch.zeros(n, D, device="cuda"), torch.zeros(n, D, device="cuda")
    q[:, 0] = 8.0
    k[::2, 0] = -1.0
    v = synth.randn((n, D), 71, 1.0, torch.float16, "cuda")
    da = (0.5 + synth.randn((n, D), 72, 0.1, torch.float16, "cuda").float()).half()
    _, got = both_ways(lib, q.half(), k.half(), v, da, [n], 1, 1, scale=1.0)
    ref = exact(q, k, v, da, 1.0)["dv"]
    off = (got["dv"].double() - ref).abs()
    assert (off <= (2 * h + 2e-4) * ref.abs() + 2.0 ** -25).all(), "%g of %g" % (off.max(), ref.abs().max())


@pytest.mark.gpu
@pytest.mark.parametrize("D", [32, 64, 128])
def test_ds_above_the_type(lib, D):
    """fp16: ds of large da and v passes the type's highest value, dq and dk, by a small scale, do not.  Few keys: delta is exact, the
    tolerances are those of the first rows of causal sequences."""
    h, d, n, scale = torch.finfo(torch.float16).eps / 2, 2e-5, 6, 2.0 ** -12
    q, k = (synth.randn((n, D), 80 + i, 1.0, torch.float16, "cuda") for i in range(2))
    v, da = synth.randn((n, D), 82, 4096.0, torch.float16, "cuda"), synth.randn((n, D), 83, 512.0, torch.float16, "cuda")
    _, got = both_ways(lib, q, k, v, da, [n], 1, 1, scale=scale)
    Q, K, V, G = (x.double() for x in (q, k, v, da))
    p = torch.softmax(scale * Q @ K.t(), dim=1)
    dp = G @ V.t()
    delta = (p * dp).sum(1, keepdim=True)
    ds = p * (dp - delta)
    assert float(ds.abs().max()) > 65504.0
    eds = (h + d) * ds.abs() + d * p * (G.abs() @ V.abs().t() + delta.abs())
    for name, ref, tol in (("dq", scale * ds @ K, scale * eds @ K.abs()), ("dk", scale * ds.t() @ Q, scale * eds.t() @ Q.abs())):
        off = (got[name].double() - ref).abs() - h * ref.abs() - tol - 2.0 ** -25
        assert (off <= 0).all(), "%s: %g above what is allowed" % (name, off.max())


@pytest.mark.gpu
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("filler", [65504.0, float("inf"), float("nan")], ids=["highest", "inf", "nan"])
def test_a_sequence_keeps_its_own_range(lib, filler, D):
    """fp16: small gradients of a sequence have the same bits beside one of the highest values, infinities or NaN, and alone."""
    lengths, heads, kv_heads = [200, 333, 70], 4, 2
    rows, r = sum(lengths), slice(200, 533)
    q, k, v = (synth.randn((rows, w * D), 90 + w + i, 1.0, torch.float16, "cuda") for i, w in enumerate((heads, kv_heads, kv_heads)))
    da = synth.randn((rows, heads * D), 97, 1e-4, torch.float16, "cuda")
    _, alone = both_ways(lib, q[r], k[r], v[r], da[r], lengths[1:2], heads, kv_heads)
    for x in (v, da):
        x[:200] = filler
        x[533:] = filler
    _, got = both_ways(lib, q, k, v, da, lengths, heads, kv_heads)
    for name in alone:
        assert torch.isfinite(alone[name]).all() and torch.equal(alone[name], got[name][r]), name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_gradient_against_differences_along_itself(lib, D, causal, dtype):
    """Differences of f = sum of da a, a by the definition in 64 bits, which no formula of the gradient enters, along the kernel's own
    gradient g: the slope is |g|^2 where g is right.  With g off by a relative e in the Frobenius norm they are e |g|^2 apart at most;
    e is 8 h: the four roundings of the small-gradients test, twice, since of few keys they do not average out.  A gradient that is
    zero, has another sign, scale or mask fails.  The third difference leaves step^2, 1e-8, of it."""
    lengths, heads, kv_heads = [90, 41, 140], 4, 2
    h, rows, scale = torch.finfo(dtype).eps / 2, sum(lengths), D ** -0.5
    q, k, v = (synth.randn((rows, w * D), 110 + i, 1.0, dtype, "cuda") for i, w in enumerate((heads, kv_heads, kv_heads)))
    da = synth.randn((rows, heads * D), 113, 0.5, dtype, "cuda")
    _, got = both_ways(lib, q, k, v, da, lengths, heads, kv_heads, causal=causal)

    def f(q, k, v):
        total, starts = 0.0, [0] + np.cumsum(lengths).tolist()
        for b, e in zip(starts, starts[1:]):
            for i in range(heads):
                j = i // (heads // kv_heads)
                ci, cj = slice(i * D, (i + 1) * D), slice(j * D, (j + 1) * D)
                s = scale * q[b:e, ci] @ k[b:e, cj].t()
                if causal:
                    s = torch.where(torch.ones_like(s, dtype=torch.bool).tril(), s, -torch.inf)
                total += float(((torch.softmax(s, dim=1) @ v[b:e, cj]) * da[b:e, ci].double()).sum())
        return total

    for which, name in enumerate(("dq", "dk", "dv")):
        x, g = [t.double() for t in (q, k, v)], got[name].double()
        size = float(g.square().sum())
        step = 1e-4 / size ** 0.5 * x[which].numel() ** 0.5                       # 1e-4 of each value's size on average

        def at(e):
            y = list(x)
            y[which] = y[which] + e * g
            return f(*y)

        slope = (at(step) - at(-step)) / (2 * step)
        assert size > 1.0 and abs(slope - size) <= (8 * h + 1e-5) * size, "%s: slope %g, %g expected" % (name, slope, size)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [32, 64, 128])
def test_captured_with_other_gradients(lib, D):
    """fp16: a captured gradient into thirds of one tensor takes the range of the da that it finds at each replay, and leaves rows of no
    sequence alone."""
    lengths, heads, kv_heads, rows = [130, 1, 300], 4, 2, 450
    parts = [heads * D, kv_heads * D, kv_heads * D]
    q, k, v = synth.randn((rows, sum(parts)), 130, 1.0, torch.float16, "cuda").split(parts, dim=1)
    da = torch.zeros(rows, heads * D, dtype=torch.float16, device="cuda")
    plan = lib.make_packed_plan([7] + (7 + np.cumsum(lengths)).tolist(), rows)
    a, lse = lib.elsa_packed_attention(q, k, v, plan, heads, kv_heads, causal=True, want_lse=True)
    dqkv = torch.full((rows, sum(parts)), 7.0, dtype=torch.float16, device="cuda")
    dq, dk, dv = dqkv.split(parts, dim=1)
    work = torch.empty(int(lib._packed_ws(rows, heads)), dtype=torch.uint8, device="cuda")
    step = lambda: lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, kv_heads, causal=True, dq=dq, dk=dk, dv=dv, workspace=work)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for size in (1.0, 1e-5, 300.0, 0.0, 1e-3):
        da.copy_(synth.randn((rows, heads * D), 131, size, torch.float16, "cuda") if size > 0 else torch.zeros_like(da))
        dqkv[7:7 + sum(lengths)] = float("nan")
        graph.replay()
        torch.cuda.synchronize()
        got = dqkv.clone()
        assert torch.isfinite(got).all() and (got[:7] == 7.0).all() and (got[7 + sum(lengths):] == 7.0).all()
        want = lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, kv_heads, causal=True)
        for x, y in zip(got.split(parts, dim=1), want):
            assert torch.equal(x[7:7 + sum(lengths)], y[7:7 + sum(lengths)]) and (size > 0 or not y.any())
