"""The plan of packed sequences where its offsets do not hold still, or come from a list while the stream that makes it is behind."""
import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2409_09708_b200 import binding
    return binding


def test_offsets_between_two_rows(lib):
    """Offsets that are no whole numbers are refused, not cut short: no place on the device is asked for."""
    for bad in ([0, 2.5, 5], torch.tensor([0.0, 2.25, 4.0]), np.array([0.5, 4.0]), [0, float("nan")]):
        with pytest.raises(ValueError, match="offsets"):
            lib.make_packed_plan(bad, rows=9)


def test_status_word_that_is_not_on_the_device(lib):
    """The kernel would write to it where the offsets are none: refused before anything is launched."""
    for status in (torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32).expand(4)):
        with pytest.raises(ValueError, match="dev_status"):
            lib.make_packed_plan([0, 5], rows=9, dev_status=status)


def test_a_list_that_leaves_rows_out(lib):
    for bad, rows in (([1, 5], 5), ([0, 4], 5)):
        with pytest.raises(ValueError, match="every row"):
            lib.make_packed_plan(bad, rows, full=True)


@pytest.mark.gpu
def test_full_offsets_on_the_device(lib):
    """Said to cover every row they are looked at, and outputs are not zeroed; left unsaid, rows of no sequence hold zeros."""
    qkv = torch.randn((300, 3 * 128), device="cuda", generator=torch.Generator("cuda").manual_seed(2)).half()
    q, k, v = qkv.split(128, dim=1)
    def on_device(*o):
        return torch.tensor(o, dtype=torch.int32, device="cuda")
    assert lib.make_packed_plan([0, 120, 300]).full and lib.make_packed_plan([0, 120, 300], full=True).full
    assert not lib.make_packed_plan(on_device(0, 120, 300), 300).full
    plan = lib.make_packed_plan(on_device(0, 120, 300), 300, full=True)
    assert plan.full
    assert torch.equal(lib.elsa_packed_attention(q, k, v, plan, 2)[0], lib.elsa_packed_attention(q, k, v, lib.make_packed_plan([0, 120, 300]), 2)[0])
    for bad in (on_device(0, 120, 299), on_device(1, 120, 300), on_device(0, 200, 100, 300), on_device(0, 301, 300)):
        with pytest.raises(ValueError, match="every row"):
            lib.make_packed_plan(bad, 300, full=True)


@pytest.mark.gpu
def test_offsets_that_change_while_the_plan_is_made(lib):
    """A plan from offsets that another stream rewrites meanwhile is worth nothing, but nothing outside it is written.  The two lists
    put the long sequences at opposite ends, so that a mixture counts fewer tiles than it lists."""
    sequences, rows = 5000, 40000
    lists = []
    for order in (1, -1):
        lengths = np.ones(sequences, dtype=np.int64)
        lengths[:sequences // 8] = 57
        offsets = np.concatenate([[0], np.cumsum(lengths[::order])])
        assert offsets[-1] <= rows
        lists.append(torch.tensor(offsets, dtype=torch.int32, device="cuda"))
    need = int(lib._packed_plan_bytes(rows, sequences))
    room = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    offsets = lists[0].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(side):
            for i in range(40):
                offsets.copy_(lists[i & 1])
        for _ in range(20):
            lib._check(lib._packed_plan(offsets.data_ptr(), sequences, rows, room.data_ptr(), need, None, lib._stream(None)))
    torch.cuda.synchronize()
    assert (room[need:] == 0x5a).all()


@pytest.mark.gpu
def test_plans_from_lists_on_a_stream_that_is_behind(lib):
    """Plans made from lists on a busy stream that is not current, each bound to the same name as the one before: every batch keeps
    its own boundaries, whatever the current stream does with memory that is free."""
    heads, D, rows = 2, 64, 400
    qkv = torch.randn((rows, 3 * heads * D), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).half()
    q, k, v = qkv.split(heads * D, dim=1)
    batches = [[0, n, rows - n // 2, rows] for n in range(20, 200, 20)]
    want = [lib.elsa_packed_attention(q, k, v, lib.make_packed_plan(b), heads)[0] for b in batches]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for fill in (False, True):
        got = []
        for b in batches:
            with torch.cuda.stream(side):
                torch.cuda._sleep(20_000_000)
            plan = lib.make_packed_plan(b, stream=side)
            got.append(lib.elsa_packed_attention(q, k, v, plan, heads, stream=side)[0])
            del plan
            if fill:
                others = [torch.full((len(b),), rows // 2, dtype=torch.int32, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        for x, y in zip(want, got):
            assert torch.equal(x, y)
    assert len(others) == 8
