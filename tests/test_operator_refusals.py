"""What elsa_layer_norm, elsa_rotary and the packed attention refuse, on the host before anything is launched."""
import ctypes

import pytest
import torch

FAKE = 0x10000          # a non-NULL, aligned value that is never dereferenced: validation fails first
WORK = 0x20000
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 1, 2, 4, 5, 6


@pytest.fixture(scope="module")
def lib():
    from paper_2409_09708_b200 import build
    build.build()
    from paper_2409_09708_b200 import binding
    return binding


def caller(fn, names, ok):
    def call(**kw):
        assert set(kw) <= set(names)
        a = dict(ok, **kw)
        return fn(*[a[n] for n in names])
    return call


def test_layer_norm(lib):
    names = "x residual gain bias rows dim eps dt s y stats stream".split()
    call = caller(lib._layer_norm, names, dict(x=FAKE, residual=FAKE, gain=FAKE, bias=FAKE, rows=4, dim=64, eps=1e-6, dt=0, s=FAKE, y=FAKE, stats=FAKE,
                                               stream=None))
    for n in ("x", "gain", "bias", "y", "s", "residual"):
        assert call(**{n: None}) == NULL, n
    for kw in (dict(rows=0), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(dim=0), dict(eps=-1.0), dict(eps=float("nan"))):
        assert call(**kw) == SHAPE, kw
    assert call(dt=2) == DTYPE
    for kw in (dict(dim=60), dict(x=FAKE + 2), dict(y=FAKE + 8), dict(gain=FAKE + 4), dict(bias=FAKE + 2), dict(s=FAKE + 2), dict(residual=FAKE + 2),
               dict(stats=FAKE + 4)):
        assert call(**kw) == ALIGN, kw


def test_layer_norm_backward(lib):
    names = "dy s stats gain ds rows dim dt dx dgain dbias work bytes stream".split()
    call = caller(lib._layer_norm_backward, names, dict(dy=FAKE, s=FAKE, stats=FAKE, gain=FAKE, ds=FAKE, rows=4, dim=64, dt=1, dx=FAKE, dgain=FAKE, dbias=FAKE,
                                                        work=WORK, bytes=1 << 20, stream=None))
    for n in ("dy", "s", "stats", "gain"):
        assert call(**{n: None}) == NULL, n
    assert call(dx=None, dgain=None, dbias=None) == NULL
    for kw in (dict(rows=0), dict(rows=(1 << 30) + 1), dict(dim=-8), dict(dim=16392)):
        assert call(**kw) == SHAPE, kw
    assert call(dt=-1) == DTYPE
    for kw in (dict(dim=20), dict(dy=FAKE + 2), dict(s=FAKE + 2), dict(ds=FAKE + 2), dict(dx=FAKE + 2), dict(dgain=FAKE + 2), dict(dbias=FAKE + 2),
               dict(gain=FAKE + 2), dict(stats=FAKE + 4), dict(work=WORK + 16)):
        assert call(**kw) == ALIGN, kw
    need = lib.elsa_layer_norm_backward_workspace_bytes(4, 64)
    assert need == 4 * 2 * 64 * 4
    assert call(work=None) == WORKSPACE and call(bytes=need - 1) == WORKSPACE
    for bad in ((0, 64), (4, 0), (4, 60), (4, 16392)):
        assert lib.elsa_layer_norm_backward_workspace_bytes(*bad) == 0


def test_rotary(lib):
    plan = lib.make_rotary_plan(64, [16, 16])
    names = "x xp positions plan rows heads inverse dt y yp stream".split()
    call = caller(lib._rotary, names, dict(x=FAKE, xp=256, positions=FAKE, plan=ctypes.byref(plan), rows=3, heads=4, inverse=0, dt=0, y=WORK, yp=256, stream=None))
    for n in ("x", "positions", "plan", "y"):
        assert call(**{n: None}) == NULL, n
    for kw in (dict(rows=0), dict(rows=(1 << 30) + 1), dict(heads=0), dict(xp=248), dict(yp=248), dict(heads=5), dict(y=FAKE, yp=264), dict(plan=ctypes.byref(lib.ElsaRotaryPlan()))):
        assert call(**kw) == SHAPE, kw
    for field, value in (("head_dim", 72), ("head_dim", 512), ("axes", 0), ("axes", 5)):
        other = lib.make_rotary_plan(64, [16, 16])
        setattr(other, field, value)
        assert call(plan=ctypes.byref(other)) == SHAPE, field
    other = lib.make_rotary_plan(64, [16, 16])
    other.axis[31] = 2
    assert call(plan=ctypes.byref(other)) == SHAPE
    assert call(heads=1 << 25, xp=1 << 40, yp=1 << 40) == SHAPE
    assert call(dt=7) == DTYPE
    for kw in (dict(x=FAKE + 8), dict(y=WORK + 2), dict(positions=FAKE + 2), dict(xp=260), dict(yp=257)):
        assert call(**kw) == ALIGN, kw


def test_packed_plan(lib):
    names = "offsets sequences rows plan bytes status stream".split()
    call = caller(lib._packed_plan, names, dict(offsets=FAKE, sequences=3, rows=500, plan=WORK, bytes=1 << 20, status=None, stream=None))
    assert call(offsets=None) == NULL and call(plan=None) == NULL
    assert call(sequences=0) == SHAPE and call(rows=0) == SHAPE and call(rows=(1 << 30) + 1) == SHAPE
    assert call(sequences=(1 << 30) + 1) == SHAPE and lib._packed_plan_bytes(5, (1 << 30) + 1) == 0
    assert call(offsets=FAKE + 2) == ALIGN and call(plan=WORK + 8) == ALIGN
    need = int(lib._packed_plan_bytes(500, 3))
    assert need == 64 + 16 * ((500 // 128 + 3) + (500 // 256 + 3)) and call(bytes=need - 1) == WORKSPACE
    assert lib._packed_plan_bytes(0, 3) == 0 and lib._packed_plan_bytes(5, 0) == 0
    assert lib._packed_plan_bytes(5, 100) == 64 + 16 * 10                   # no more tiles than rows
    for bad in ([], [0], [0, 5, 3], [-1, 4], [2, 1]):
        with pytest.raises(ValueError):
            lib.make_packed_plan(bad)
    with pytest.raises(ValueError):
        lib.make_packed_plan([0, 5], rows=4)
    for rows in (-1, 1 << 31, (1 << 32) + 5):
        with pytest.raises(ValueError):
            lib.make_packed_plan([0, 5], rows=rows)


def qkv_of(lib, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, q_pitch=256, k_pitch=128, v_pitch=128, rows=100, heads=4, kv_heads=2, head_dim=64, causal=0, scale=0.125)
    a.update(kw)
    return ctypes.byref(lib.ElsaPackedQkv(*[a[n] for n, _ in lib.ElsaPackedQkv._fields_]))


COMMON = [(dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(rows=0), SHAPE), (dict(rows=(1 << 30) + 1), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE),
          (dict(kv_heads=3), SHAPE), (dict(head_dim=48), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=256), SHAPE), (dict(scale=float("inf")), SHAPE),
          (dict(scale=float("nan")), SHAPE), (dict(q_pitch=248), SHAPE), (dict(k_pitch=120), SHAPE), (dict(v_pitch=0), SHAPE), (dict(q_pitch=260), ALIGN),
          (dict(k_pitch=132), ALIGN), (dict(q=FAKE + 8), ALIGN), (dict(v=FAKE + 2), ALIGN), (dict(heads=1 << 28, kv_heads=1, q_pitch=1 << 40), SHAPE)]


def test_packed_attention(lib):
    names = "qkv dt plan sequences a ap lse status stream".split()
    call = caller(lib._packed, names, dict(qkv=qkv_of(lib), dt=0, plan=FAKE, sequences=2, a=WORK, ap=256, lse=FAKE, status=None, stream=None))
    for kw, want in COMMON:
        assert call(qkv=qkv_of(lib, **kw)) == want, kw
    assert call(qkv=None) == NULL and call(plan=None) == NULL and call(a=None) == NULL
    assert call(sequences=0) == SHAPE and call(sequences=(1 << 30) + 1) == SHAPE and call(ap=255) == SHAPE
    assert call(dt=9) == DTYPE
    assert call(plan=FAKE + 4) == ALIGN and call(a=WORK + 2) == ALIGN and call(ap=257) == ALIGN and call(lse=FAKE + 2) == ALIGN


def test_packed_attention_backward(lib):
    names = "qkv dt plan sequences a ap lse da dap dq dqp dk dkp dv dvp work bytes status stream".split()
    call = caller(lib._packed_backward, names, dict(qkv=qkv_of(lib), dt=0, plan=FAKE, sequences=2, a=FAKE, ap=256, lse=FAKE, da=FAKE, dap=256, dq=FAKE, dqp=256,
                                                    dk=FAKE, dkp=128, dv=FAKE, dvp=128, work=WORK, bytes=1 << 20, status=None, stream=None))
    for kw, want in COMMON:
        assert call(qkv=qkv_of(lib, **kw)) == want, kw
    for n in ("a", "lse", "da", "dq", "dk", "dv"):
        assert call(**{n: None}) == NULL, n
        assert call(**{n: FAKE + 2}) == ALIGN, n
    for n, least in (("ap", 256), ("dap", 256), ("dqp", 256), ("dkp", 128), ("dvp", 128)):
        assert call(**{n: least - 8}) == SHAPE and call(**{n: least + 4}) == ALIGN, n
    need = int(lib._packed_ws(100, 4))
    assert need == 2 * (-(-100 * 4 * 4 // 256) * 256)
    assert call(work=None) == WORKSPACE and call(bytes=need - 1) == WORKSPACE and call(work=WORK + 64) == ALIGN
    assert lib._packed_ws(0, 4) == 0 and lib._packed_ws(4, 0) == 0


def test_tensors_of_the_wrong_kind(lib):
    """The binding: types, shapes and places that do not fit are refused before a pointer is taken."""
    x, g = torch.zeros(4, 64, dtype=torch.float16), torch.zeros(64, dtype=torch.float16)
    with pytest.raises(ValueError):
        lib.elsa_layer_norm(x, g, g)                                        # on the CPU
    with pytest.raises(TypeError):
        lib.elsa_layer_norm(x, g.bfloat16(), g)
    with pytest.raises(TypeError):
        lib.elsa_layer_norm(x.float(), g.float(), g.float())
    plan = lib.make_rotary_plan(64, [32])
    with pytest.raises(ValueError):
        lib.elsa_rotary(x, torch.zeros(4, 1, dtype=torch.int32), plan)
    fake = lib.PackedPlan(torch.zeros(3, dtype=torch.int32), 4, True, torch.zeros(64, dtype=torch.uint8))
    with pytest.raises(ValueError):
        lib.elsa_packed_attention(x, x, x, fake, 1)


@pytest.mark.gpu
def test_tensors_of_the_wrong_shape(lib):
    dev = "cuda"
    x, g = torch.zeros(4, 64, dtype=torch.float16, device=dev), torch.zeros(64, dtype=torch.float16, device=dev)
    y, _, stats = lib.elsa_layer_norm(x, g, g, want_stats=True)
    for bad in (lambda: lib.elsa_layer_norm(x, g[:32], g), lambda: lib.elsa_layer_norm(x, g, g, residual=x[:2]), lambda: lib.elsa_layer_norm(x, g, g, s=x),
                lambda: lib.elsa_layer_norm(x.t(), g[:4], g[:4]), lambda: lib.elsa_layer_norm(x, g, g, stats=stats[:2]),
                lambda: lib.elsa_layer_norm_backward(x, x, g, None), lambda: lib.elsa_layer_norm_backward(x, x[:3], g, stats),
                lambda: lib.elsa_layer_norm_backward(x, x, g, stats.double()), lambda: lib.elsa_layer_norm_backward(x, x, g, stats, ds=x[:1])):
        with pytest.raises(ValueError):
            bad()
    plan = lib.make_rotary_plan(64, [32])
    at = torch.zeros(4, 1, dtype=torch.int32, device=dev)
    for bad in (lambda: lib.elsa_rotary(x[:, :48], at, plan), lambda: lib.elsa_rotary(x, at[:2], plan), lambda: lib.elsa_rotary(x.t().contiguous().t(), at, plan),
                lambda: lib.elsa_rotary(x, at, plan, y=x[:2])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        lib.elsa_rotary(x, at.long(), plan)
    packed = lib.make_packed_plan([0, 1, 4])
    a, lse = lib.elsa_packed_attention(x, x, x, packed, 2, want_lse=True)
    for bad in (lambda: lib.elsa_packed_attention(x, x, x[:, :32], packed, 2), lambda: lib.elsa_packed_attention(x[:3], x, x, packed, 2),
                lambda: lib.elsa_packed_attention(x, x, x, packed, 3), lambda: lib.elsa_packed_attention(x, x, x, packed, 0),
                lambda: lib.elsa_packed_attention(x, x, x, packed, 2, a=x[:, :32]), lambda: lib.elsa_packed_attention(x, x, x, packed, 2, lse=lse[:1]),
                lambda: lib.elsa_packed_attention_backward(x, x, x, x, a, None, packed, 2),
                lambda: lib.elsa_packed_attention_backward(x[:, :32], x, x, x, a, lse, packed, 2)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        lib.elsa_packed_attention(x, x.bfloat16(), x, packed, 2)
    for bad in (torch.zeros(3, dtype=torch.int64, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)):
        with pytest.raises(ValueError):
            lib.make_packed_plan(bad, 4)
    assert lib.elsa_packed_attention(x, x, x, packed, 2)[1] is None


@pytest.mark.gpu
def test_sizes_that_fit_no_int(lib):
    """More rows than an int counts (expanded, so that they take no memory) are refused before anything is cut short."""
    x = torch.zeros(1, 64, dtype=torch.float16, device="cuda").expand((1 << 32) + 4, 64)
    g = torch.zeros(64, dtype=torch.float16, device="cuda")
    stats = torch.zeros(1, 2, device="cuda").expand(x.shape[0], 2)
    at = torch.zeros(1, 1, dtype=torch.int32, device="cuda").expand(x.shape[0], 1)
    packed = lib.make_packed_plan([0, 4])
    for bad in (lambda: lib.elsa_layer_norm(x, g, g, y=x), lambda: lib.elsa_layer_norm_backward(x, x, g, stats, dx=x),
                lambda: lib.elsa_rotary(x, at, lib.make_rotary_plan(64, [32]), y=x), lambda: lib.elsa_packed_attention(x, x, x, packed, 1)):
        with pytest.raises(ValueError, match="int"):
            bad()
