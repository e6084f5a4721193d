"""Attention over packed sequences and its gradient against the definition in 64 bits.

Tolerances, with h half a step of the type relative to the value (finfo.eps / 2) and d = 2e-4 for everything in fp32 (the scores'
sums of up to 128 products, exponentials of approximate units, sums of probabilities; scores here stay below 64 in size):
  a      E_a = h |a| + (h + d) sum p |v| + t sum |v|        probabilities rounded once, t = 2^-24 for those of fp16 below its normal range
  lse    d (1 + |lse|)
  dv     h |dv| + (h + d) sum p |da| + t sum |da|
  ds     E_ds = (h + d) |ds| + p sum |da| E_a + d p (sum |da| |v| + |delta|) + t      delta comes from the rounded a; ds rounded once
  dq, dk h |.| + |scale| sum E_ds |k|  and  |scale| sum E_ds |q|
"""
import threading

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


def formula(q, k, v, lengths, heads, kv_heads, causal, scale, da=None):
    """The definitions, sequence by sequence and head by head, in 64 bits, and the errors the header allows."""
    dev, dtype = q.device, q.dtype
    h, d = torch.finfo(dtype).eps / 2, 2e-4
    t = 2.0 ** -24 if dtype == torch.float16 else 0.0
    D = q.shape[1] // heads
    rows = q.shape[0]
    q, k, v = q.double(), k.double(), v.double()
    out = {"a": torch.zeros_like(q), "lse": torch.zeros(heads, rows, dtype=torch.float64, device=dev), "dq": torch.zeros_like(q),
           "dk": torch.zeros_like(k), "dv": torch.zeros_like(v)}
    tol = {n: torch.zeros_like(x) for n, x in out.items()}
    begin = 0
    for n in lengths:
        r = slice(begin, begin + n)
        begin += n
        if n == 0:
            continue
        for i in range(heads):
            j = i // (heads // kv_heads)
            ci, cj = slice(i * D, (i + 1) * D), slice(j * D, (j + 1) * D)
            s = scale * q[r, ci] @ k[r, cj].t()
            if causal:
                s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=dev).triu(1), -torch.inf)
            lse = torch.logsumexp(s, dim=1)
            p = torch.exp(s - lse[:, None])
            a = p @ v[r, cj]
            va = v[r, cj].abs()
            ea = h * a.abs() + (h + d) * (p @ va) + t * va.sum(0)
            out["a"][r, ci], tol["a"][r, ci] = a, ea
            out["lse"][i, r], tol["lse"][i, r] = lse, d * (1 + lse.abs())
            if da is None:
                continue
            g = da[r, ci].double()
            delta = (g * a).sum(1, keepdim=True)
            dp = g @ v[r, cj].t()
            ds = p * (dp - delta)
            eds = (h + d) * ds.abs() + p * (g.abs() * ea).sum(1, keepdim=True) + d * p * (g.abs() @ va.t() + delta.abs()) + t * (p > 0)
            out["dq"][r, ci] += scale * ds @ k[r, cj]
            out["dk"][r, cj] += scale * ds.t() @ q[r, ci]
            out["dv"][r, cj] += p.t() @ g
            tol["dq"][r, ci] += abs(scale) * eds @ k[r, cj].abs()
            tol["dk"][r, cj] += abs(scale) * eds.t() @ q[r, ci].abs()
            tol["dv"][r, cj] += (h + d) * (p.t() @ g.abs()) + t * g.abs().sum(0)
    for n in ("dq", "dk", "dv"):
        tol[n] += h * out[n].abs()
    return out, tol


def near(name, got, ref, tol):
    got = got.double()
    assert torch.isfinite(got).all(), name
    over = (got - ref).abs() - tol - 1e-7
    worst = over.argmax()
    assert (over <= 0).all(), "%s: off by %g, allowed %g" % (name, (got - ref).abs().flatten()[worst], tol.flatten()[worst])


def inputs(lengths, heads, kv_heads, D, dtype, seed=5, size=1.0):
    rows = sum(lengths)
    qkv = synth.randn((rows, (heads + 2 * kv_heads) * D), seed, size, dtype, "cuda")
    da = synth.randn((rows, heads * D), seed + 1, 0.5, dtype, "cuda")
    return qkv, qkv.split([heads * D, kv_heads * D, kv_heads * D], dim=1), da


def offsets_of(lengths):
    return [0] + np.cumsum(lengths).tolist()


def check(lib, lengths, heads, kv_heads, D, causal, dtype, size=1.0, scale=None, change=None):
    qkv, (q, k, v), da = inputs(lengths, heads, kv_heads, D, dtype, size=size)
    if change is not None:
        change(q, k, v)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    plan = lib.make_packed_plan(offsets_of(lengths), dev_status=status)
    a, lse = lib.elsa_packed_attention(q, k, v, plan, heads, kv_heads, causal=causal, scale=scale, want_lse=True, dev_status=status)
    grads = lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, kv_heads, causal=causal, scale=scale, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0, "device status %#x" % int(status.item())
    ref, tol = formula(q, k, v, lengths, heads, kv_heads, causal, D ** -0.5 if scale is None else scale, da)
    for name, got in zip(("a", "lse", "dq", "dk", "dv"), (a, lse) + grads):
        near(name, got, ref[name], tol[name])


LENGTHS = [[1], [5], [16], [17], [64], [65], [127], [128], [129], [197], [256], [257], [600], [0, 5, 0], [127, 128, 129, 1], [1] * 9,
           [63, 64, 65, 0, 1, 300], [1025, 3, 130]]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("lengths", LENGTHS, ids=["-".join(map(str, l)) for l in LENGTHS])
def test_lengths(lib, lengths, D, causal, dtype):
    check(lib, lengths, 2, 2, D, causal, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("heads", [(1, 1), (5, 5), (4, 2), (6, 2), (8, 1), (12, 3)], ids=lambda h: "%d-%d" % h)
def test_shared_key_heads(lib, heads, D, causal):
    check(lib, [70, 200, 33, 300], heads[0], heads[1], D, causal, torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("D", [32, 64, 128])
def test_many_items(lib, D, dtype):
    """More tiles than SMs, long and short sequences mixed."""
    lengths = np.random.default_rng(3).integers(1, 700, 60).tolist()
    check(lib, lengths, 3, 3, D, False, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_long_sequences(lib, D, causal):
    """Of a length that has the gradient's kernels of long sequences, beside short ones that they then meet too."""
    check(lib, [4500], 2, 1, D, causal, torch.bfloat16)
    check(lib, [2600, 1, 4000], 2, 2, D, causal, torch.float16)
    check(lib, [1500, 70, 999], 2, 1, D, causal, torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_scores_that_grow_along_the_keys(lib, causal, D, dtype):
    """The running reference has to rise within a tile and from tile to tile, by single rows and by all of them."""
    def change(q, k, v):
        rows = k.shape[0]
        q[:, 0::D] = 8.0
        k[:, 0::D] = (torch.arange(rows, device="cuda") * (60.0 / rows) * D ** 0.5 / 8.0).to(k.dtype)[:, None]
        q[5::7, 0::D] = -8.0
    check(lib, [500], 2, 2, D, causal, dtype, size=0.5, change=change)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.25, 0.9])
def test_scale(lib, scale):
    check(lib, [150, 40], 2, 2, 64, True, torch.float16, size=0.8, scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("filler", [float("nan"), float("inf"), -65504.0], ids=["nan", "inf", "lowest"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_other_rows_take_no_part_and_stay(lib, causal, D, filler):
    """A sequence's results do not depend on its neighbours or on rows of no sequence, whatever these hold; rows of no sequence are
    not written.  The plan is made from offsets on the device."""
    heads, kv_heads, dtype = 4, 2, torch.float16
    lengths = [37, 200, 3, 129]
    before, behind = 11, 90
    rows = before + sum(lengths) + behind
    base, _, _ = inputs([rows], heads, kv_heads, D, dtype)
    da0 = synth.randn((rows, heads * D), 9, 0.5, dtype, "cuda")
    starts = np.cumsum([before] + lengths)
    results = []
    for fill in (False, True):
        qkv, da = base.clone(), da0.clone()
        if fill:
            for x in (qkv, da):
                x[:before] = filler
                x[starts[-1]:] = filler
                x[starts[2]:starts[3]] = filler                       # the third sequence
        q, k, v = qkv.split([heads * D, kv_heads * D, kv_heads * D], dim=1)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        plan = lib.make_packed_plan(torch.tensor(starts, dtype=torch.int32, device="cuda"), rows, dev_status=status)
        a = torch.full((rows, heads * D), 7.0, dtype=dtype, device="cuda")
        lse = torch.full((heads, rows), 7.0, device="cuda")
        dqkv = torch.full_like(qkv, 7.0)
        dq, dk, dv = dqkv.split([heads * D, kv_heads * D, kv_heads * D], dim=1)
        lib.elsa_packed_attention(q, k, v, plan, heads, kv_heads, causal=causal, a=a, lse=lse, dev_status=status)
        lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, kv_heads, causal=causal, dq=dq, dk=dk, dv=dv, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        for x in (a, dqkv, lse.t()):
            assert (x[:before] == 7.0).all() and (x[starts[-1]:] == 7.0).all()
        results.append((a, dqkv, lse.t()))
    for x, y in zip(*results):
        for i in (0, 1, 3):
            r = slice(starts[i], starts[i + 1])
            assert torch.isfinite(x[r]).all() and torch.equal(x[r], y[r])


@pytest.mark.gpu
@pytest.mark.parametrize("D", [32, 64, 128])
def test_tiles_with_idle_warps_many_times(lib, D):
    """Last tiles of which some warps have no rows, beside full ones on the same SM: the same bits in each of many runs."""
    for lengths in (np.random.default_rng(3).integers(1, 700, 60).tolist(), [3000, 2500, 130, 3100, 5000]):
        qkv, (q, k, v), da = inputs(lengths, 3, 3, D, torch.bfloat16)
        plan = lib.make_packed_plan(offsets_of(lengths))
        first = None
        for _ in range(100):
            a, lse = lib.elsa_packed_attention(q, k, v, plan, 3, want_lse=True)
            got = (a, lse) + lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, 3)
            first = first or got
            assert all(torch.equal(x, y) for x, y in zip(first, got))


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
def test_same_bits_every_time_and_in_graphs_and_streams(lib, D):
    lengths, heads, kv_heads = [300, 77, 1, 513], 4, 2
    qkv, (q, k, v), da = inputs(lengths, heads, kv_heads, D, torch.bfloat16)
    plan = lib.make_packed_plan(offsets_of(lengths))

    def step(workspace=None):
        a, lse = lib.elsa_packed_attention(q, k, v, plan, heads, kv_heads, causal=True, want_lse=True)
        return (a, lse) + lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, kv_heads, causal=True, workspace=workspace)

    first = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = step()
    for t in third:
        t.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for x, y, z in zip(first, second, third):
        assert torch.equal(x, y) and torch.equal(x, z)


@pytest.mark.gpu
def test_calls_on_several_streams_at_once(lib):
    """Narrow and wide heads, forward and gradient, side by side on the device: each result is the one of the call alone."""
    cases = [([700, 300, 64], 4, 2, 64), ([900, 5], 2, 1, 128), ([200] * 20, 3, 3, 32), ([2500], 2, 2, 64)]
    work = []
    for i, (lengths, heads, kv_heads, D) in enumerate(cases):
        qkv, (q, k, v), da = inputs(lengths, heads, kv_heads, D, torch.bfloat16, seed=30 + 2 * i)
        work.append((q, k, v, da, lib.make_packed_plan(offsets_of(lengths)), heads, kv_heads))

    def step(q, k, v, da, plan, heads, kv_heads):
        a, lse = lib.elsa_packed_attention(q, k, v, plan, heads, kv_heads, causal=True, want_lse=True)
        return (a, lse) + lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, kv_heads, causal=True)

    alone = [step(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(10):
        got = []
        for s, w in zip(streams, work):
            with torch.cuda.stream(s):
                got.append([step(*w) for _ in range(3)])
        torch.cuda.synchronize()
        for x, ys in zip(alone, got):
            for y in ys:
                assert all(torch.equal(u, w) for u, w in zip(x, y))


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
def test_given_stream_and_outputs_of_its_own(lib, D):
    """stream= without making it current: with rows of no sequence the call's own outputs hold zeros there."""
    rows, n, heads = 300, 210, 2
    qkv, (q, k, v), da = inputs([rows], heads, heads, D, torch.float16)
    side = torch.cuda.Stream()
    plan = lib.make_packed_plan([20, 20 + n], rows)
    torch.cuda.synchronize()
    a, lse = lib.elsa_packed_attention(q, k, v, plan, heads, want_lse=True, stream=side)
    grads = lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, stream=side)
    side.synchronize()
    r = slice(20, 20 + n)
    ref, tol = formula(q[r], k[r], v[r], [n], heads, heads, False, D ** -0.5, da[r])
    for name, got in zip(("a", "dq", "dk", "dv"), (a,) + grads):
        near(name, got[r], ref[name], tol[name])
        assert (got[:20] == 0).all() and (got[20 + n:] == 0).all()


@pytest.mark.gpu
def test_memory_of_a_call_belongs_to_its_stream(lib):
    """A call on a stream that is not current, while the current one has writes to freed blocks before it: what the call allocates is
    neither such a block nor goes back to that stream while the call runs."""
    lengths, heads, D = [512, 300], 4, 64
    qkv, (q, k, v), da = inputs(lengths, heads, heads, D, torch.float16)
    rows = sum(lengths)
    x = da.contiguous()
    gain = torch.ones(heads * D, dtype=torch.float16, device="cuda")
    side = torch.cuda.Stream()
    plan = lib.make_packed_plan(offsets_of(lengths))
    offsets = torch.tensor(offsets_of(lengths), dtype=torch.int32, device="cuda")

    def step(stream):
        another = lib.make_packed_plan(offsets, rows, stream=stream)
        b, _ = lib.elsa_packed_attention(q, k, v, another, heads, causal=True, stream=stream)
        a, lse = lib.elsa_packed_attention(q, k, v, plan, heads, want_lse=True, stream=stream)
        y, _, stats = lib.elsa_layer_norm(x, gain, gain, want_stats=True, stream=stream)
        return (a, b, lse, y, stats) + lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, stream=stream) + \
            lib.elsa_layer_norm_backward(x, x, gain, stats, stream=stream)

    ref = step(None)
    torch.cuda.synchronize()
    sizes = [t.numel() * t.element_size() for t in ref] + [1 << 20, 1 << 16, 1 << 12]
    freed = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
    torch.cuda._sleep(50_000_000)
    for t in freed:
        t.fill_(0x7f)
    del freed, t
    got = step(side)
    torch.cuda.synchronize()
    assert all(torch.equal(u, w) for u, w in zip(ref, got))
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    got = step(side)
    others = [torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0x7f) for n in sizes for _ in range(4)]       # on the current stream
    torch.cuda.synchronize()
    assert len(others) > 0 and all(torch.equal(u, w) for u, w in zip(ref, got))


@pytest.mark.gpu
def test_empty_sequences_alone(lib):
    """A batch whose rows all belong to no sequence: everything that a call allocates is zero."""
    qkv, (q, k, v), da = inputs([70], 2, 2, 64, torch.bfloat16)
    plan = lib.make_packed_plan([9, 9, 9], 70)
    a, lse = lib.elsa_packed_attention(q, k, v, plan, 2, want_lse=True)
    for t in (a, lse) + lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, 2):
        assert (t == 0).all()


@pytest.mark.gpu
def test_two_threads_and_the_default_stream(lib):
    """Calls from two host threads at once, and with the default stream given while another one is current."""
    work = []
    for seed, (lengths, D) in enumerate((([300, 80], 64), ([150, 260], 128))):
        qkv, (q, k, v), da = inputs(lengths, 2, 1, D, torch.float16, seed=60 + seed)
        work.append((q, k, v, da, lib.make_packed_plan(offsets_of(lengths))))

    def step(q, k, v, da, plan, stream=None):
        a, lse = lib.elsa_packed_attention(q, k, v, plan, 2, 1, want_lse=True, stream=stream)
        return (a, lse) + lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, 2, 1, stream=stream)

    alone = [step(*w) for w in work]
    torch.cuda.synchronize()
    got = [[], []]

    def many(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(50):
                got[i].append(step(*work[i]))
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=many, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    with torch.cuda.stream(torch.cuda.Stream()):
        for i in range(2):
            got[i].append(step(*work[i], stream=torch.cuda.default_stream()))
    torch.cuda.synchronize()
    for x, ys in zip(alone, got):
        assert len(ys) == 51 and all(torch.equal(u, w) for y in ys for u, w in zip(x, y))


@pytest.mark.gpu
def test_plans_that_do_not_fit(lib):
    """Offsets that are none, and a plan of another batch: nothing is written, dev_status tells."""
    heads, D, rows = 2, 64, 100
    qkv, (q, k, v), da = inputs([rows], heads, heads, D, torch.float16)
    for bad in ([0, 60, 40, 100], [-1, 50, 100], [0, 101], [5, 3]):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        plan = lib.make_packed_plan(torch.tensor(bad, dtype=torch.int32, device="cuda"), rows, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 2 | 69 << 8
        a = torch.full((rows, heads * D), 7.0, dtype=q.dtype, device="cuda")
        lib.elsa_packed_attention(q, k, v, plan, heads, a=a, dev_status=status)
        torch.cuda.synchronize()
        assert (a == 7.0).all()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    plan = lib.make_packed_plan([0, 60, 100])
    plan.sequences = 1
    a = torch.full((rows, heads * D), 7.0, dtype=q.dtype, device="cuda")
    lib.elsa_packed_attention(q, k, v, plan, heads, a=a, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 2 | 79 << 8 and (a == 7.0).all()
    plan.sequences = 2
    lib.elsa_packed_attention(q, k, v, plan, heads, a=a)
    assert not (a == 7.0).any()


@pytest.mark.gpu
def test_plan_lists_every_tile_once(lib):
    """The plan's tiles of 128 and 256 rows, read back: each tile of each sequence once, longest sequences first."""
    rng = np.random.default_rng(11)
    for lengths in ([1], [0, 0], [128], [129, 0, 128], rng.integers(0, 900, 3000).tolist(), [200000, 5, 140000, 139000, 0, 7], [1] * 5000):
        offsets = np.concatenate([[0], np.cumsum(lengths)])
        rows = max(1, int(offsets[-1]))
        plan = lib.make_packed_plan(offsets.tolist(), rows)
        words = plan.buffer.cpu().numpy().view(np.int32)
        n128, n256 = int(words[3]), int(words[4])
        assert words[1] == rows and words[2] == len(lengths)
        first = 0
        for size, n in ((128, n128), (256, n256)):
            want = sorted((int(o), int(l), t) for o, l in zip(offsets, lengths) for t in range(-(-l // size)))
            cap = min(rows, rows // size + len(lengths))
            got = words[16 + 4 * first:16 + 4 * (first + n)].reshape(n, 4)
            assert n <= cap and sorted(map(tuple, got[:, :3].tolist())) == want
            tiles = -(-got[:, 1].astype(np.int64) // 128)
            assert (np.diff(np.minimum(tiles, 1023)) <= 0).all()
            first += cap


@pytest.mark.gpu
def test_rows_past_32_bits(lib):
    """A tensor of more than 2^31 values, the sequence at its end."""
    heads, kv_heads, D, n = 2, 1, 64, 333
    pitch, rows = 12288, 180000
    big = torch.zeros((rows, pitch), dtype=torch.float16, device="cuda")
    big[rows - n:, -512:] = synth.randn((n, 512), 21, 1.0, torch.float16, "cuda")
    q, k, v, da = big[:, -512:-384], big[:, -384:-320], big[:, -320:-256], big[:, -256:-128]
    plan = lib.make_packed_plan(torch.tensor([rows - n, rows], dtype=torch.int32, device="cuda"), rows)
    a, lse = lib.elsa_packed_attention(q, k, v, plan, heads, kv_heads, causal=True, want_lse=True)
    grads = lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, kv_heads, causal=True)
    end = slice(rows - n, rows)
    ref, tol = formula(q[end], k[end], v[end], [n], heads, kv_heads, True, D ** -0.5, da[end])
    for name, got in zip(("a", "dq", "dk", "dv"), (a,) + grads):
        near(name, got[end], ref[name], tol[name])
    assert (a[:rows - n] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_gradient_against_differences(lib, causal):
    """(f(x + e t) - f(x - e t)) / 2e of f = sum of da * a in 64 bits against the kernel's gradient along t."""
    lengths, heads, kv_heads, D, dtype = [90, 41, 140], 4, 2, 64, torch.float16
    qkv, (q, k, v), da = inputs(lengths, heads, kv_heads, D, dtype)
    plan = lib.make_packed_plan(offsets_of(lengths))
    a, lse = lib.elsa_packed_attention(q, k, v, plan, heads, kv_heads, causal=causal, want_lse=True)
    grads = lib.elsa_packed_attention_backward(da, q, k, v, a, lse, plan, heads, kv_heads, causal=causal)
    _, tol = formula(q, k, v, lengths, heads, kv_heads, causal, D ** -0.5, da)
    for which, (name, grad) in enumerate(zip(("dq", "dk", "dv"), grads)):
        x = [t.double() for t in (q, k, v)]
        t = torch.randn(x[which].shape, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(which))

        def loss(e):
            y = list(x)
            y[which] = y[which] + e * t
            return float((formula(*y, lengths, heads, kv_heads, causal, D ** -0.5)[0]["a"] * da.double()).sum())

        e = 1e-4                                                      # the third difference leaves an error of e^2, 1e-8
        slope = (loss(e) - loss(-e)) / (2 * e)
        along = float((grad.double() * t).sum())
        assert abs(along - slope) <= float((tol[name] * t.abs()).sum()) + 1e-5 * abs(slope)
