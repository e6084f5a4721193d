"""What the training and serving of blocks with images of many sizes asks of the library beside the pruned linears.

Three operators and their gradients, as a program that trains or serves a pruned vision transformer calls them:

  norm        LayerNorm of token rows, alone at inference; in training with the residual added ahead of it, its
              statistics kept, and its gradient with those of gain and bias
  rotary      rotary positions with one, two or three axes (row and column of a patch; frame, row and column) on the
              query and key columns of qkv, and the gradient (the inverse rotation)
  attention   softmax attention over packed sequences of different lengths (images of many sizes side by side in one
              batch, prompts of patches), with shared key heads, causal or not; alone at inference and as a training
              step with its gradients

Sizes are those of DeiT-B, Swin-B and generic wider ones.  ``own`` false: the operators written out in elementary
operations in 32 bits, sequences padded to the longest.  ``own`` true: the library's calls.  ``exact``: the definitions
in 64 bits, head by head and sequence by sequence.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # LayerNorm of one image's tokens at inference: the smallest call, where latency is what is paid for.
        {"name": "norm_one_image", "op": "norm", "train": False, "rows": 197, "dim": 768, "dtype": "f16"},
        # A training step's LayerNorm at DeiT-B's full batch, the residual added on the way.
        {"name": "norm_train_deit_b256", "op": "norm", "train": True, "rows": 50432, "dim": 768, "dtype": "bf16"},
        # A width that no model of the repository has and rows that fill nothing evenly.
        {"name": "norm_train_odd", "op": "norm", "train": True, "rows": 12345, "dim": 1384, "dtype": "f16"},
        # Queries and keys of one image, positions by patch row and column.
        {"name": "rotary_one_image", "op": "rotary", "rows": 197, "heads": 12, "kv_heads": 12, "head_dim": 64, "axes": 2,
         "far": 16, "interleaved": False, "inverse": False, "dtype": "f16"},
        # The gradient of the rotation for a full batch of images.
        {"name": "rotary_gradient_b256", "op": "rotary", "rows": 50432, "heads": 12, "kv_heads": 12, "head_dim": 64, "axes": 2,
         "far": 64, "interleaved": False, "inverse": True, "dtype": "bf16"},
        # A clip of video: frame, row and column, wide heads with shared keys, frames far into a stream.
        {"name": "rotary_video", "op": "rotary", "rows": 16384, "heads": 32, "kv_heads": 8, "head_dim": 128, "axes": 3,
         "far": 200000, "interleaved": True, "inverse": False, "dtype": "bf16"},
        # Serving one image.
        {"name": "attention_one_image", "op": "attention", "train": False, "sequences": 1, "shortest": 197, "longest": 197,
         "heads": 12, "kv_heads": 12, "head_dim": 64, "causal": False, "dtype": "f16"},
        # Evaluating images of many sizes packed into one batch.
        {"name": "attention_packed_images", "op": "attention", "train": False, "sequences": 128, "shortest": 49, "longest": 1024,
         "heads": 12, "kv_heads": 12, "head_dim": 64, "causal": False, "dtype": "bf16"},
        # One long prompt of patches, causal, four query heads to a key head.
        {"name": "attention_prompt", "op": "attention", "train": False, "sequences": 1, "shortest": 16384, "longest": 16384,
         "heads": 8, "kv_heads": 2, "head_dim": 128, "causal": True, "dtype": "bf16"},
        # A training step on a handful of small images.
        {"name": "attention_train_small", "op": "attention", "train": True, "sequences": 8, "shortest": 1, "longest": 130,
         "heads": 6, "kv_heads": 6, "head_dim": 64, "causal": False, "dtype": "f16"},
        # A training step on a packed batch of images.
        {"name": "attention_train_packed_images", "op": "attention", "train": True, "sequences": 64, "shortest": 49, "longest": 1024,
         "heads": 12, "kv_heads": 12, "head_dim": 64, "causal": False, "dtype": "bf16"},
        # A training step on one long causal sequence with shared key heads.
        {"name": "attention_train_prompt", "op": "attention", "train": True, "sequences": 1, "shortest": 8192, "longest": 8192,
         "heads": 16, "kv_heads": 4, "head_dim": 128, "causal": True, "dtype": "bf16"},
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    dtype = rng.choice(["f16", "bf16"])
    op = rng.choice(["norm", "rotary", "attention", "attention"])
    if op == "norm":
        dim = 8 * _spread(rng, 8, 512)
        return {"op": op, "train": rng.random() < 0.7, "rows": _spread(rng, 1, min(50432, 38000000 // dim)), "dim": dim, "dtype": dtype}
    if op == "rotary":
        head_dim = rng.choice([32, 64, 128])
        kv_heads = rng.choice([1, 2, 3, 4, 6, 12])
        heads = kv_heads * rng.choice([1, 1, 2, 4])
        rows = _spread(rng, 1, min(50432, 80000000 // ((heads + kv_heads) * head_dim)))
        return {"op": op, "rows": rows, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "axes": rng.choice([1, 2, 3]),
                "far": _spread(rng, 16, 1000000), "interleaved": rng.random() < 0.5, "inverse": rng.random() < 0.5, "dtype": dtype}
    head_dim = rng.choice([32, 64, 128])
    kv_heads = rng.choice([1, 2, 3, 4])
    heads = kv_heads * rng.choice([1, 2, 4])
    longest = _spread(rng, 1, 4096)
    most = max(1, min(256, 16384 // longest))
    return {"op": op, "train": rng.random() < 0.5, "sequences": _spread(rng, 1, most), "shortest": rng.randint(1, longest),
            "longest": longest, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "causal": rng.random() < 0.5, "dtype": dtype}


def _lengths(case):
    """Lengths between the shortest and the longest, both among them, the same for every seed."""
    n, low, high = case["sequences"], case["shortest"], case["longest"]
    lengths = np.random.default_rng(97).integers(low, high + 1, n)
    lengths[0] = high
    if n > 1:
        lengths[-1] = low
    return lengths.tolist()


def _sections(head_dim, axes):
    """Pairs of an axis: an even split, what is left over goes to the first axis."""
    pairs = head_dim // 2
    return [pairs // axes + (pairs % axes if i == 0 else 0) for i in range(axes)]


def prepare(case, seed):
    dtype = DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)

    state = {"case": case}
    if case["op"] == "norm":
        rows, dim = case["rows"], case["dim"]
        state["x"] = normal(rows, dim)
        state["gain"] = (1.0 + 0.1 * torch.randn(dim, generator=gen, device="cuda")).to(dtype)
        state["bias"] = normal(dim, scale=0.1)
        if case["train"]:
            state["residual"] = normal(rows, dim, scale=2.0)
            state["dy"] = normal(rows, dim, scale=0.5)
            state["ds"] = normal(rows, dim, scale=0.5)       # what arrives along the residual path
        return state
    if case["op"] == "rotary":
        rows, width = case["rows"], case["head_dim"]
        both = case["heads"] + case["kv_heads"]
        state["qkv"] = normal(rows, (both + case["kv_heads"]) * width)
        state["positions"] = torch.randint(0, case["far"], (rows, case["axes"]), generator=gen, device="cuda", dtype=torch.int32)
        state["sections"] = _sections(width, case["axes"])
        if own:
            from paper_2409_09708_b200 import binding as lib
            state["plan"] = lib.make_rotary_plan(width, state["sections"], interleaved=case["interleaved"])
        else:
            pairs = [(axis, i / n) for axis, n in enumerate(state["sections"]) for i in range(n)]
            state["axis"] = torch.tensor([a for a, _ in pairs], device="cuda")
            state["rate"] = torch.tensor([10000.0 ** -e for _, e in pairs], dtype=torch.float64, device="cuda")
        return state
    lengths = _lengths(case)
    offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    rows, width = int(offsets[-1]), case["head_dim"]
    state["qkv"] = normal(rows, (case["heads"] + 2 * case["kv_heads"]) * width)
    if case["train"]:
        state["da"] = normal(rows, case["heads"] * width, scale=0.5)
    if own:
        from paper_2409_09708_b200 import binding as lib
        state["plan"] = lib.make_packed_plan(offsets.tolist(), rows)
    else:
        place = np.arange(max(lengths))[None, :]
        inside = place < np.asarray(lengths)[:, None]
        state["inside"] = torch.from_numpy(inside).cuda()
        state["row"] = torch.from_numpy(np.where(inside, offsets[:-1, None] + place, 0)).cuda()
        state["sequence"] = torch.from_numpy(np.repeat(np.arange(len(lengths)), lengths)).cuda()
        state["place"] = torch.from_numpy(np.concatenate([np.arange(n) for n in lengths])).cuda()
    return state


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    if case["op"] == "norm":
        return _plain_norm(state, case)
    if case["op"] == "rotary":
        return _plain_rotary(state, case)
    return _plain_attention(state, case)


def _run_own(state):
    from paper_2409_09708_b200 import binding as lib
    case = state["case"]
    if case["op"] == "norm":
        if not case["train"]:
            return lib.elsa_layer_norm(state["x"], state["gain"], state["bias"], EPS)[0]
        y, s, stats = lib.elsa_layer_norm(state["x"], state["gain"], state["bias"], EPS, residual=state["residual"], want_stats=True)
        dx, dgain, dbias = lib.elsa_layer_norm_backward(state["dy"], s, state["gain"], stats, ds=state["ds"])
        return {"y": y, "s": s, "dx": dx, "dgain": dgain, "dbias": dbias}
    heads, kv_heads, width = case["heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "rotary":
        both = heads + kv_heads
        return lib.elsa_rotary(state["qkv"][:, :both * width], state["positions"], state["plan"], inverse=case["inverse"])
    q, k, v = state["qkv"].split([heads * width, kv_heads * width, kv_heads * width], dim=1)
    if not case["train"]:
        return lib.elsa_packed_attention(q, k, v, state["plan"], heads, kv_heads, causal=case["causal"])[0]
    a, lse = lib.elsa_packed_attention(q, k, v, state["plan"], heads, kv_heads, causal=case["causal"], want_lse=True)
    dq, dk, dv = lib.elsa_packed_attention_backward(state["da"], q, k, v, a, lse, state["plan"], heads, kv_heads, causal=case["causal"])
    return {"a": a, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _plain_norm(state, case):
    x, gain, bias = state["x"].float(), state["gain"].float(), state["bias"].float()
    dtype = state["x"].dtype
    if case["train"]:
        s = (x + state["residual"].float()).to(dtype)       # the stream is kept in the 16-bit type
        x = s.float()
    centred = x - x.mean(dim=1, keepdim=True)
    rstd = (centred.square().mean(dim=1, keepdim=True) + EPS).rsqrt()
    xhat = centred * rstd
    y = (xhat * gain + bias).to(dtype)
    if not case["train"]:
        return y
    dy = state["dy"].float()
    g = dy * gain
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True)) + state["ds"].float()
    return {"y": y, "s": s, "dx": dx.to(dtype), "dgain": (dy * xhat).sum(dim=0).to(dtype), "dbias": dy.sum(dim=0).to(dtype)}


def _plain_rotary(state, case):
    both, width = case["heads"] + case["kv_heads"], case["head_dim"]
    x = state["qkv"][:, :both * width].float().view(-1, both, width)
    angle = state["positions"].double()[:, state["axis"]] * state["rate"]      # far positions need the 64 bits
    if case["inverse"]:
        angle = -angle
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if case["interleaved"]:
        first, second = x[..., 0::2], x[..., 1::2]
        turned = torch.stack([first * cos - second * sin, second * cos + first * sin], dim=-1)
    else:
        first, second = x[..., :width // 2], x[..., width // 2:]
        turned = torch.cat([first * cos - second * sin, second * cos + first * sin], dim=-1)
    return turned.reshape(x.shape[0], both * width).to(state["qkv"].dtype)


def _plain_attention(state, case):
    heads, kv_heads, width = case["heads"], case["kv_heads"], case["head_dim"]
    dtype, row, inside = state["qkv"].dtype, state["row"], state["inside"]
    group, scale = heads // kv_heads, 1.0 / math.sqrt(width)

    def padded(t, n):                                        # [rows][n * width] -> [sequence][head][place][width]
        return (t.float().view(-1, n, width)[row] * inside[:, :, None, None]).transpose(1, 2)

    def packed(t, n):                                        # and back
        return t[state["sequence"], :, state["place"]].reshape(-1, n * width).to(dtype)

    q, k, v = state["qkv"].split([heads * width, kv_heads * width, kv_heads * width], dim=1)
    q = padded(q, heads).unflatten(1, (kv_heads, group))
    k, v = padded(k, kv_heads).unsqueeze(2), padded(v, kv_heads).unsqueeze(2)
    hidden = ~inside[:, None, None, None, :]
    if case["causal"]:
        places = torch.arange(inside.shape[1], device=row.device)
        hidden = hidden | (places[None, :] > places[:, None])
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).masked_fill_(hidden, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    p.div_(total)
    a = torch.matmul(p, v)
    out = packed(a.flatten(1, 2), heads)
    if not case["train"]:
        return out
    lse = (top + total.log()).flatten(1, 2).squeeze(-1)[state["sequence"], :, state["place"]].t().contiguous()
    da = padded(state["da"], heads).unflatten(1, (kv_heads, group))
    dv = torch.matmul(p.transpose(-1, -2), da).sum(dim=2)
    ds = torch.matmul(da, v.transpose(-1, -2)).sub_((da * a).sum(dim=-1, keepdim=True)).mul_(p)
    dq = torch.matmul(ds, k).mul_(scale).flatten(1, 2)
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(dim=2).mul_(scale)
    return {"a": out, "lse": lse, "dq": packed(dq, heads), "dk": packed(dk, kv_heads), "dv": packed(dv, kv_heads)}


def work(case):
    """Each input read once and each output written once; the products of the attention over the pairs that its mask leaves."""
    if case["op"] == "norm":
        values = case["rows"] * case["dim"]
        tensors = 7 if case["train"] else 2                  # x, residual, dy, ds in; y, s, dx out
        return {"bytes": 2 * tensors * values, "flops": (24 if case["train"] else 8) * values}
    both, width = case["heads"] + case["kv_heads"], case["head_dim"]
    if case["op"] == "rotary":
        return {"bytes": 4 * case["rows"] * both * width + 4 * case["rows"] * case["axes"], "flops": 3 * case["rows"] * both * width}
    lengths = np.asarray(_lengths(case), dtype=np.float64)
    rows, pairs = lengths.sum(), (lengths * (lengths + 1) / 2 if case["causal"] else lengths ** 2).sum()
    wide, narrow = case["heads"] * width, case["kv_heads"] * width
    if not case["train"]:
        return {"bytes": int(2 * rows * (2 * wide + 2 * narrow)), "flops": int(4 * pairs * wide)}
    return {"bytes": int(2 * rows * (4 * wide + 4 * narrow) + 4 * rows * case["heads"]), "flops": int(14 * pairs * wide)}


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(state, case)
    if case["op"] == "rotary":
        return _exact_rotary(state, case)
    return _exact_attention(state, case)


def _exact_norm(state, case):
    x = state["x"].double()
    if case["train"]:
        s = x + state["residual"].double()
        x = s.to(state["x"].dtype).double()                  # the norm is taken of the stream as it is kept
    x.requires_grad_(case["train"])
    gain, bias = (state[n].double().requires_grad_(case["train"]) for n in ("gain", "bias"))
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    y = (x - mean) / torch.sqrt(var + EPS) * gain + bias
    if not case["train"]:
        return y
    dx, dgain, dbias = torch.autograd.grad(y, (x, gain, bias), state["dy"].double())
    return {"y": y.detach(), "s": s, "dx": dx + state["ds"].double(), "dgain": dgain, "dbias": dbias}


def _exact_rotary(state, case):
    """Each pair of values as a complex number, turned by its position's angle."""
    both, width, sections = case["heads"] + case["kv_heads"], case["head_dim"], state["sections"]
    x = state["qkv"][:, :both * width].double().reshape(-1, both, width)
    pairs = x.reshape(-1, both, width // 2, 2) if case["interleaved"] else x.reshape(-1, both, 2, width // 2).transpose(2, 3)
    angles = []
    for axis, n in enumerate(sections):
        rate = torch.pow(10000.0, -torch.arange(n, dtype=torch.float64, device="cuda") / n)
        angles.append(state["positions"][:, axis].double()[:, None] * rate[None, :])
    angle = torch.cat(angles, dim=1)[:, None, :]
    turn = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    return (z if case["interleaved"] else z.transpose(2, 3)).reshape(-1, both * width)


def _exact_attention(state, case):
    heads, kv_heads, width = case["heads"], case["kv_heads"], case["head_dim"]
    qkv = state["qkv"].double()
    rows = qkv.shape[0]
    a = torch.zeros(rows, heads * width, dtype=torch.float64, device="cuda")
    lse = torch.zeros(heads, rows, dtype=torch.float64, device="cuda")
    grad = torch.zeros_like(qkv)
    begin = 0
    for n in _lengths(case):
        part = slice(begin, begin + n)
        begin += n
        for h in range(heads):
            at = [h, heads + h // (heads // kv_heads), heads + kv_heads + h // (heads // kv_heads)]
            q, k, v = (qkv[part, c * width:(c + 1) * width] for c in at)
            s = (q / math.sqrt(width)) @ k.t()
            if case["causal"]:
                s = torch.where(torch.ones_like(s, dtype=torch.bool).tril(), s, -torch.inf)
            lse[h, part] = torch.logsumexp(s, dim=1)
            p = torch.softmax(s, dim=1)
            a[part, h * width:(h + 1) * width] = p @ v
            if not case["train"]:
                continue
            da = state["da"][part, h * width:(h + 1) * width].double()
            dp = da @ v.t()
            ds = p * (dp - (dp * p).sum(dim=1, keepdim=True)) / math.sqrt(width)
            for c, g in zip(at, (ds @ k, ds.t() @ q, p.t() @ da)):
                grad[part, c * width:(c + 1) * width] += g
    if not case["train"]:
        return a
    dq, dk, dv = grad.split([heads * width, kv_heads * width, kv_heads * width], dim=1)
    return {"a": a, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
