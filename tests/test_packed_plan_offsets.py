"""The plan of packed sequences where its offsets do not hold still, or come from a list while the stream that makes it is behind."""
import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2409_09708_b200 import binding
    return binding


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
