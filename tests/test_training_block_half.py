"""Norm, masked qkv, rotary positions, packed attention, projection and residual in a row, and their gradients back to the input and
every weight, as a training step on images of different sizes makes them, against 64-bit autograd.

Fourteen tensors are rounded to the type on the way there and back (h = finfo.eps / 2 each, relative to their values), the linear
stages between them carry the errors on, the softmax and the norm damp those of common size: 14 h in the Frobenius norm."""
import math

import numpy as np
import pytest
import torch

from oracle import elsa_oracle as eo
from paper_2409_09708_b200 import synth


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("causal,kv_heads", [(False, 4), (True, 2)], ids=["full", "causal-shared"])
def test_step_and_gradients(dtype, causal, kv_heads):
    from paper_2409_09708_b200 import binding as lib
    heads, D, N, M = 4, 64, 2, 4
    dim, width = heads * D, (heads + 2 * kv_heads) * D
    lengths = [197, 50, 0, 130, 1]
    rows = sum(lengths)
    grid = [(i, j) for n in lengths for i, j in ((t // 14, t % 14) for t in range(n))]
    positions = torch.tensor(grid, dtype=torch.int32, device="cuda")
    x, r, dout = (synth.randn((rows, dim), i, 1.0, dtype, "cuda") for i in (1, 2, 3))
    gain, bias = synth.randn((dim,), 4, 0.1, dtype, "cuda") + 1.0, synth.randn((dim,), 5, 0.1, dtype, "cuda")
    W = {"qkv": synth.randn((width, dim), 6, 1.0 / math.sqrt(dim / 2), dtype, "cuda"), "proj": synth.randn((dim, dim), 7, 1.0 / math.sqrt(dim / 2), dtype, "cuda")}
    b = {"qkv": synth.randn((width,), 8, 0.1, dtype, "cuda"), "proj": synth.randn((dim,), 9, 0.1, dtype, "cuda")}
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    plan = lib.make_packed_plan([0] + np.cumsum(lengths).tolist(), rows, dev_status=status)
    turn = lib.make_rotary_plan(D, [16, 16])
    both, parts = (heads + kv_heads) * D, [heads * D, kv_heads * D, kv_heads * D]

    # there
    y, s, stats = lib.elsa_layer_norm(x, gain, bias, 1e-6, residual=r, want_stats=True)
    packed = {n: lib.elsa_nm_compress(w, N, M) for n, w in W.items()}
    qkv = lib.elsa_nm_linear(y, *packed["qkv"], b["qkv"], width, dim, N, M, dev_status=status)
    lib.elsa_rotary(qkv[:, :both], positions, turn, y=qkv[:, :both])
    q, k, v = qkv.split(parts, dim=1)
    a, lse = lib.elsa_packed_attention(q, k, v, plan, heads, kv_heads, causal=causal, want_lse=True, dev_status=status)
    o = lib.elsa_nm_linear(a, *packed["proj"], b["proj"], dim, dim, N, M, dev_status=status)
    # and back: dout arrives at out = s + o
    da, dWp, dbp = lib.elsa_nm_linear_backward(dout, a, *packed["proj"], dim, dim, N, M, dev_status=status)
    dqkv = torch.empty_like(qkv)
    dq, dk, dv = dqkv.split(parts, dim=1)
    lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, kv_heads, causal=causal, dq=dq, dk=dk, dv=dv, dev_status=status)
    lib.elsa_rotary(dqkv[:, :both], positions, turn, y=dqkv[:, :both], inverse=True)
    dy, dWq, dbq = lib.elsa_nm_linear_backward(dqkv, y, *packed["qkv"], width, dim, N, M, dev_status=status)
    dx, dgain, dbias = lib.elsa_layer_norm_backward(dy, s, gain, stats, ds=dout)
    torch.cuda.synchronize()
    assert int(status.item()) == 0

    # the same in 64 bits
    masks = {n: torch.from_numpy(eo.nm_compress(synth.bits(w), N, M)[2].astype(np.float64)).cuda().reshape(w.shape) for n, w in W.items()}
    leaf = {n: t.double().requires_grad_() for n, t in dict(x=x, gain=gain, bias=bias, Wq=W["qkv"], Wp=W["proj"], bq=b["qkv"], bp=b["proj"]).items()}
    S = leaf["x"] + r.double()
    c = S - S.mean(1, keepdim=True)
    Y = c / torch.sqrt(c.square().mean(1, keepdim=True) + 1e-6) * leaf["gain"] + leaf["bias"]
    QKV = Y @ (leaf["Wq"] * masks["qkv"]).t() + leaf["bq"]
    rate = torch.tensor([10000.0 ** (-i / 16) for i in range(16)], dtype=torch.float64, device="cuda")
    angle = torch.cat([positions[:, ax:ax + 1].double() * rate for ax in (0, 1)], dim=1)[:, None]
    h = QKV[:, :both].reshape(rows, -1, D)
    h = torch.cat([h[..., :32] * angle.cos() - h[..., 32:] * angle.sin(), h[..., 32:] * angle.cos() + h[..., :32] * angle.sin()], dim=-1)
    V = QKV[:, both:].reshape(rows, kv_heads, D)
    out, begin = [], 0
    for n in lengths:
        rr = slice(begin, begin + n)
        begin += n
        K, VV = (t.repeat_interleave(heads // kv_heads, dim=1) for t in (h[rr, heads:], V[rr]))
        sc = torch.einsum("ihd,jhd->hij", h[rr, :heads], K) / 8.0
        if causal:
            sc = sc.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -torch.inf)
        out.append(torch.einsum("hij,jhd->ihd", torch.softmax(sc, dim=-1), VV).reshape(n, dim))
    A = torch.cat(out)
    O = A @ (leaf["Wp"] * masks["proj"]).t() + leaf["bp"]
    ref = dict(zip(leaf, torch.autograd.grad(S + O, list(leaf.values()), dout.double())))
    bound = 14 * torch.finfo(dtype).eps / 2
    for name, got, want in (("a", a, A), ("o", o, O), ("x", dx, ref["x"]), ("gain", dgain, ref["gain"]), ("bias", dbias, ref["bias"]),
                            ("Wq", dWq, ref["Wq"]), ("bq", dbq, ref["bq"]), ("Wp", dWp, ref["Wp"]), ("bp", dbp, ref["bp"])):
        rel = float((got.double() - want.detach()).norm() / want.detach().norm())
        assert rel <= bound, "%s: %g, allowed %g" % (name, rel, bound)
