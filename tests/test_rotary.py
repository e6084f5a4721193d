"""Rotary positions against the definition in 64 bits: |err| <= h |ref| + 2e-6 (|a| + |b|), h half a step of the type (finfo.eps / 2):
angles are off by at most 2e-7, the special-function unit's sine and cosine by 5e-7 each, the two products and the sum by 2e-7."""
import math

import pytest
import torch

from paper_2409_09708_b200 import synth

TYPES = [torch.bfloat16, torch.float16]
NAMES = ["bf16", "f16"]


@pytest.fixture(scope="module")
def lib():
    from paper_2409_09708_b200 import binding
    return binding


def rates(sections, base, shared):
    """(axis, rate) of each pair."""
    total = sum(sections)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    if shared:
        return axis, [base ** (-p / total) for p in range(total)]
    return axis, [base ** (-i / n) for n in sections for i in range(n)]


def formula(x, positions, D, sections, base, shared, interleaved, inverse):
    axis, rate = rates(sections, base, shared)
    angle = positions.double()[:, axis] * torch.tensor(rate, dtype=torch.float64, device=x.device)
    angle = torch.remainder(angle, 2 * math.pi) * (-1 if inverse else 1)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    v = x.double().reshape(x.shape[0], -1, D)
    a, b = (v[..., 0::2], v[..., 1::2]) if interleaved else (v[..., :D // 2], v[..., D // 2:])
    out, size = [a * c - b * s, b * c + a * s], a.abs() + b.abs()
    join = (lambda p, q: torch.stack([p, q], dim=-1)) if interleaved else (lambda p, q: torch.cat([p, q], dim=-1))
    return join(*out).reshape(x.shape), join(size, size).reshape(x.shape)


def near(got, ref, size, dtype, extra=0.0):
    err = (got.double() - ref).abs()
    tol = torch.finfo(dtype).eps / 2 * ref.abs() + (2e-6 + extra) * size + 1e-7
    worst = (err - tol).argmax()
    assert (err <= tol).all(), "off by %g, allowed %g" % (err.flatten()[worst], tol.flatten()[worst])


CASES = [(16, [8], 1), (32, [8, 8], 3), (48, [8, 8, 8], 5), (64, [16, 16], 24), (64, [11, 21], 2), (64, [32, 0], 7), (80, [20, 20], 6),
         (96, [16, 16, 16], 4), (128, [16, 24, 24], 40), (128, [64], 1), (112, [14, 14, 14, 14], 9), (256, [43, 43, 42], 3)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("case", CASES, ids=["%d-%s-%d" % (d, "+".join(map(str, s)), h) for d, s, h in CASES])
def test_heads_and_axes(lib, case, interleaved, dtype):
    D, sections, heads = case
    for rows, shared, inverse in ((1, False, False), (37, True, True), (400, False, True)):
        qkv = synth.randn((rows, heads * D + 24), 3, 1.0, dtype, "cuda")
        x = qkv[:, 8:8 + heads * D]
        positions = torch.randint(-50, 300, (rows, len(sections)), dtype=torch.int32, device="cuda")
        plan = lib.make_rotary_plan(D, sections, base=10000.0, shared=shared, interleaved=interleaved)
        y = lib.elsa_rotary(x, positions, plan, inverse=inverse)
        ref, size = formula(x, positions, D, sections, 10000.0, shared, interleaved, inverse)
        near(y, ref, size, dtype)
        # in place, the columns beside stay
        keep = qkv.clone()
        assert lib.elsa_rotary(x, positions, plan, y=x, inverse=inverse) is x
        assert torch.equal(x, y) and torch.equal(qkv[:, :8], keep[:, :8]) and torch.equal(qkv[:, 8 + heads * D:], keep[:, 8 + heads * D:])


@pytest.mark.gpu
@pytest.mark.parametrize("base", [1.0, 100.0, 5e5])
def test_far_positions(lib, base):
    """Positions to the ends of int32.  The 64-bit reference itself is off by position * rate * 2^-53, 3e-7 at most."""
    D, sections, rows = 64, [16, 16], 500
    x = synth.randn((rows, 2 * D), 3, 1.0, torch.float16, "cuda")
    positions = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows, 2), dtype=torch.int64, device="cuda").to(torch.int32)
    positions[:3] = torch.tensor([[2 ** 31 - 1, -2 ** 31], [0, -1], [1, 0]], dtype=torch.int32)
    y = lib.elsa_rotary(x, positions, lib.make_rotary_plan(D, sections, base=base))
    ref, size = formula(x, positions, D, sections, base, False, False, False)
    near(y, ref, size, torch.float16, 1e-6)


@pytest.mark.gpu
def test_position_zero_changes_nothing_and_back_again(lib):
    x = synth.randn((300, 24 * 64), 3, 1.0, torch.bfloat16, "cuda")
    plan = lib.make_rotary_plan(64, [16, 16])
    assert torch.equal(lib.elsa_rotary(x, torch.zeros(300, 2, dtype=torch.int32, device="cuda"), plan), x)
    positions = torch.randint(0, 99, (300, 2), dtype=torch.int32, device="cuda")
    there = lib.elsa_rotary(x, positions, plan)
    back = lib.elsa_rotary(there, positions, plan, inverse=True)
    size = x.double().abs().reshape(300, 24, 2, 32).sum(2, keepdim=True).expand(-1, -1, 2, -1).reshape(300, -1)
    assert ((back.double() - x.double()).abs() <= 2.0 ** -8 * (x.double().abs() + 2 * size) + 4e-6 * size).all()


@pytest.mark.gpu
def test_more_than_32_bits_of_values(lib):
    rows, pitch = 180000, 12288
    big = torch.zeros((rows, pitch), dtype=torch.float16, device="cuda")
    x = big[:, -128:]
    x[-100:] = synth.randn((100, 128), 3, 1.0, torch.float16, "cuda")
    positions = torch.arange(rows, dtype=torch.int32, device="cuda")[:, None].contiguous()
    plan = lib.make_rotary_plan(64, [32])
    ref, size = formula(x[-100:], positions[-100:], 64, [32], 10000.0, False, False, False)
    lib.elsa_rotary(x, positions, plan, y=x)
    near(x[-100:], ref, size, torch.float16)
    assert (big[:, :-128] == 0).all()


@pytest.mark.gpu
def test_graph_and_stream(lib):
    x = synth.randn((197, 24 * 64), 3, 1.0, torch.float16, "cuda")
    positions = torch.randint(0, 99, (197, 2), dtype=torch.int32, device="cuda")
    plan = lib.make_rotary_plan(64, [16, 16])
    first = lib.elsa_rotary(x, positions, plan)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = lib.elsa_rotary(x, positions, plan)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = lib.elsa_rotary(x, positions, plan)
    del plan                                           # its rates went into the graph by value
    third.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, second) and torch.equal(first, third)


def test_plan_on_the_host(lib):
    """Turns per position of each pair, against 64-bit floating point.  What the reference itself may be off by, relative to a rate:
    its exponent -p / n is rounded (2^-53 of a number of at most 1, which the power turns into ln(base) 2^-53), the power and the
    quotient by 2 pi are within two units each (4 * 2^-53); the plan is within 2^-64 of a turn."""
    for D, sections, base, shared in ((64, [16, 16], 10000.0, False), (128, [16, 24, 24], 5e5, True), (16, [8], 1.0, False), (80, [0, 40], 100.0, False)):
        plan = lib.make_rotary_plan(D, sections, base, shared)
        axis, rate = rates(sections, base, shared)
        assert list(plan.axis[:D // 2]) == axis
        for t, r in zip(plan.turns[:D // 2], rate):
            assert abs(t / 2.0 ** 64 - r / (2 * math.pi)) <= (math.log(base) + 4) * 2.0 ** -53 * r + 2.0 ** -64
    for D, sections, base in ((60, [30], 10.0), (0, [0], 10.0), (272, [136], 10.0), (64, [16], 10.0), (64, [33, -1], 10.0), (64, [], 10.0),
                              (64, [8, 8, 8, 4, 4], 10.0), (64, [32], 0.5), (64, [32], float("nan")), (64, [32], float("inf"))):
        with pytest.raises(lib.ElsaError):
            lib.make_rotary_plan(D, sections, base)
