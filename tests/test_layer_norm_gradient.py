"""elsa_layer_norm and elsa_layer_norm_backward against the definitions in 64 bits.

Tolerances, h half a step of the type relative to the value (finfo.eps / 2), e = 2^-24:
  stats  mean: dim e mean|s|;  1 / sqrt(var + eps): relative (dim + 8) e plus what the mean's error adds, (dim e mean|s| rstd)^2
  y      h |y| + d (|xhat gain| + |bias|),  d = 3e-5: fp32 sums of up to 16384 values in chains of at most 200, products, the root
  dx     h |dx| + d rstd (|g| + mean|g| + |xhat| mean|g xhat|) + h-free |ds|
  dgain  h |dgain| + rows-deep chains of fp32 additions: e (rows / 8 + 600) sum |dy xhat| + d sum |dy xhat|;  dbias alike
"""
import pytest
import torch

from paper_2409_09708_b200 import synth

TYPES = [torch.bfloat16, torch.float16]
NAMES = ["bf16", "f16"]
EPS, D = 1e-6, 3e-5


@pytest.fixture(scope="module")
def lib():
    from paper_2409_09708_b200 import binding
    return binding


def near(name, got, ref, tol):
    got = got.double()
    assert torch.isfinite(got).all(), name
    over = (got - ref).abs() - tol - 1e-7
    worst = over.argmax()
    assert (over <= 0).all(), "%s: off by %g, allowed %g" % (name, (got - ref).abs().flatten()[worst], tol.flatten()[worst])


def check(lib, rows, dim, dtype, residual, ds, offset=0.0):
    h = torch.finfo(dtype).eps / 2
    x = synth.randn((rows, dim), 1, 1.0, dtype, "cuda")
    r = synth.randn((rows, dim), 2, 2.0, dtype, "cuda") + offset if residual else None
    gain, bias = synth.randn((dim,), 3, 0.3, dtype, "cuda") + 1.0, synth.randn((dim,), 4, 0.3, dtype, "cuda")
    dy = synth.randn((rows, dim), 5, 0.5, dtype, "cuda")
    dres = synth.randn((rows, dim), 6, 0.5, dtype, "cuda") if ds else None
    y, s, stats = lib.elsa_layer_norm(x, gain, bias, EPS, residual=r, want_stats=True)
    plain, _, none = lib.elsa_layer_norm(x, gain, bias, EPS, residual=r)
    assert none is None and torch.equal(plain, y)
    dx, dgain, dbias = lib.elsa_layer_norm_backward(dy, s, gain, stats, ds=dres)
    if residual:
        assert torch.equal(s, (x.float() + r.float()).to(dtype))
    else:
        assert s is x
    S, G, B, DY = s.double(), gain.double(), bias.double(), dy.double()
    mean = S.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((S - mean).square().mean(1, keepdim=True) + EPS)
    xhat, e = (S - mean) * rstd, 2.0 ** -24
    size = S.abs().mean(1, keepdim=True)
    near("mean", stats[:, :1], mean, dim * e * size)
    near("rstd", stats[:, 1:], rstd, rstd * ((dim + 8) * e + (dim * e * size * rstd) ** 2))
    # what the mean's own error does to xhat
    shift = torch.clamp(min(dim, 256) * e * size * rstd, max=1.0)
    near("y", y, xhat * G + B, h * (xhat * G + B).abs() + D * ((xhat * G).abs() + B.abs()) + shift * G.abs())
    g = DY * G
    c1, c2 = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
    ref = rstd * (g - c1 - xhat * c2) + (dres.double() if ds else 0.0)
    tol = h * ref.abs() + D * rstd * (g.abs() + g.abs().mean(1, keepdim=True) + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
    tol = tol + D * (dres.double().abs() if ds else 0.0) + shift * rstd * (c2.abs() + xhat.abs() * g.abs().mean(1, keepdim=True))
    near("dx", dx, ref, tol)
    chain = e * (rows / 8 + 600) + D
    near("dgain", dgain, (DY * xhat).sum(0), h * (DY * xhat).sum(0).abs() + chain * (DY * xhat).abs().sum(0) + (shift * DY.abs()).sum(0))
    near("dbias", dbias, DY.sum(0), h * DY.sum(0).abs() + chain * DY.abs().sum(0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("extra", [False, True], ids=["plain", "residual"])
@pytest.mark.parametrize("dim", [8, 24, 64, 72, 128, 192, 248, 256, 264, 384, 512, 520, 768, 1000, 1024, 1384, 2048, 2056, 4096, 4104, 8192,
                                 8200, 16384])
def test_widths(lib, dim, extra, dtype):
    check(lib, 77, dim, dtype, extra, extra)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [8, 128, 768, 1000, 4096])
@pytest.mark.parametrize("rows", [1, 2, 3, 31, 32, 33, 197, 5000])
def test_rows(lib, rows, dim):
    check(lib, rows, dim, torch.bfloat16, True, False)
    check(lib, rows, dim, torch.float16, False, True)


@pytest.mark.gpu
def test_many_rows(lib):
    check(lib, 50432, 768, torch.bfloat16, True, True)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 768, 2048])
def test_rows_far_from_zero(lib, dim):
    check(lib, 40, dim, torch.float16, True, True, offset=20.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 768, 1000])
def test_constant_rows(lib, dim):
    """No variance: y is the bias, and the gradient stays finite."""
    x = torch.full((9, dim), 3.0, dtype=torch.bfloat16, device="cuda")
    gain, bias = synth.randn((dim,), 3, 0.3, torch.bfloat16, "cuda"), synth.randn((dim,), 4, 0.3, torch.bfloat16, "cuda")
    y, s, stats = lib.elsa_layer_norm(x, gain, bias, EPS, want_stats=True)
    assert torch.equal(y, bias.expand(9, dim)) and torch.equal(stats[:, 0], torch.full((9,), 3.0, device="cuda"))
    dx, dgain, _ = lib.elsa_layer_norm_backward(torch.ones_like(x), s, gain, stats)
    assert torch.isfinite(dx).all() and (dgain == 0).all()


@pytest.mark.gpu
def test_wider_than_the_gradient_takes(lib):
    """The forward call has no limit of its own; the gradient refuses."""
    rows, dim = 5, 16392
    x, gain, bias = (synth.randn(s, i, 1.0, torch.float16, "cuda") for i, s in enumerate([(rows, dim), (dim,), (dim,)]))
    y, _, stats = lib.elsa_layer_norm(x, gain, bias, EPS, want_stats=True)
    X = x.double()
    rstd = 1 / torch.sqrt(X.var(1, correction=0, keepdim=True) + EPS)
    ref = (X - X.mean(1, keepdim=True)) * rstd * gain.double() + bias.double()
    near("y", y, ref, (2.0 ** -11 + D) * (ref.abs() + bias.double().abs()) + 1e-4 * gain.double().abs())
    near("rstd", stats[:, 1:], rstd, 1e-4 * rstd)
    with pytest.raises(lib.ElsaError):
        lib.elsa_layer_norm_backward(x, x, gain, stats)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [768, 1000])
def test_in_place_and_parts(lib, dim):
    rows, dtype = 333, torch.bfloat16
    x, r, dy, ds = (synth.randn((rows, dim), i, 1.0, dtype, "cuda") for i in range(4))
    gain, bias = synth.randn((dim,), 7, 0.3, dtype, "cuda"), synth.randn((dim,), 8, 0.3, dtype, "cuda")
    y, s, stats = lib.elsa_layer_norm(x, gain, bias, EPS, residual=r, want_stats=True)
    for target in (0, 1):
        two = [x.clone(), r.clone()]
        y2, s2, stats2 = lib.elsa_layer_norm(two[0], gain, bias, EPS, residual=two[1], s=two[target], want_stats=True)
        assert torch.equal(y, y2) and torch.equal(s, s2) and torch.equal(stats, stats2) and s2 is two[target]
    alone = lib.elsa_layer_norm(x, gain, bias, EPS)[0]
    same = x.clone()
    assert torch.equal(lib.elsa_layer_norm(same, gain, bias, EPS, y=same)[0], alone) and torch.equal(same, alone)
    dx, dgain, dbias = lib.elsa_layer_norm_backward(dy, s, gain, stats, ds=ds)
    for target in (0, 1):
        two = [dy.clone(), ds.clone()]
        got = lib.elsa_layer_norm_backward(two[0], s, gain, stats, ds=two[1], dx=two[target])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dgain) and torch.equal(got[2], dbias)
    for want in (("dx",), ("dgain",), ("dbias",), ("dx", "dbias")):
        got = dict(zip(("dx", "dgain", "dbias"), lib.elsa_layer_norm_backward(dy, s, gain, stats, ds=ds, want=want)))
        for name, ref in (("dx", dx), ("dgain", dgain), ("dbias", dbias)):
            assert got[name] is None if name not in want else torch.equal(got[name], ref)


@pytest.mark.gpu
def test_a_row_that_is_not_finite_stays_alone(lib):
    x = synth.randn((50, 1000), 1, 1.0, torch.float16, "cuda")
    gain, bias = synth.randn((1000,), 2, 0.3, torch.float16, "cuda"), synth.randn((1000,), 3, 0.3, torch.float16, "cuda")
    y, _, stats = lib.elsa_layer_norm(x, gain, bias, EPS, want_stats=True)
    x2 = x.clone()
    x2[17, 3] = float("inf")
    x2[30, 999] = float("nan")
    y2, _, stats2 = lib.elsa_layer_norm(x2, gain, bias, EPS, want_stats=True)
    keep = torch.ones(50, dtype=torch.bool, device="cuda")
    keep[[17, 30]] = False
    assert torch.equal(y[keep], y2[keep]) and torch.isnan(y2[~keep]).all()
    dx = lib.elsa_layer_norm_backward(x, x, gain, stats, want=("dx",))[0]
    dx2 = lib.elsa_layer_norm_backward(x, x2, gain, stats2, want=("dx",))[0]
    assert torch.equal(dx[keep], dx2[keep])


@pytest.mark.gpu
def test_graph_and_stream(lib):
    x, r, dy = (synth.randn((700, 768), i, 1.0, torch.bfloat16, "cuda") for i in range(3))
    gain, bias = synth.randn((768,), 7, 0.3, torch.bfloat16, "cuda"), synth.randn((768,), 8, 0.3, torch.bfloat16, "cuda")

    def step():
        y, s, stats = lib.elsa_layer_norm(x, gain, bias, EPS, residual=r, want_stats=True)
        return (y, s, stats) + lib.elsa_layer_norm_backward(dy, s, gain, stats, ds=dy)

    first = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = step()
    for t in third:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.gpu
def test_gradient_against_differences(lib):
    """(f(x + e t) - f(x - e t)) / 2e of f = sum of dy * y in 64 bits against the kernel's gradients along t."""
    rows, dim, dtype = 60, 200, torch.float16
    x, dy = synth.randn((rows, dim), 1, 1.0, dtype, "cuda"), synth.randn((rows, dim), 2, 1.0, dtype, "cuda")
    gain, bias = synth.randn((dim,), 3, 0.3, dtype, "cuda") + 1.0, synth.randn((dim,), 4, 0.3, dtype, "cuda")
    _, s, stats = lib.elsa_layer_norm(x, gain, bias, EPS, want_stats=True)
    grads = lib.elsa_layer_norm_backward(dy, s, gain, stats)
    for which, grad in enumerate(grads):
        t = torch.randn(grad.shape, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(which))

        def loss(e):
            p = [x.double(), gain.double(), bias.double()]
            p[which] = p[which] + e * t
            c = p[0] - p[0].mean(1, keepdim=True)
            return float(((c / torch.sqrt(c.square().mean(1, keepdim=True) + EPS) * p[1] + p[2]) * dy.double()).sum())

        slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
        # roundings of the stored gradient, half a step each, and fp32 inside
        allowed = float(((2.0 ** -11 + D) * grad.double().abs() * t.abs()).sum()) + D * float(dy.double().abs().sum())
        assert abs(float((grad.double() * t).sum()) - slope) <= allowed
