"""Calls with `stream=` while the current stream is at work: what a call allocates for itself is that stream's memory, not the current one's."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


def _busy(times=30):
    """Some milliseconds of work on the current stream."""
    x = torch.zeros(1 << 26, device="cuda")
    torch.cuda.synchronize()
    for _ in range(times):
        x.add_(1)
    return x


@pytest.mark.parametrize("handle", [False, True])
def test_status_words_of_calls_beside_a_busy_stream(handle):
    fs = _fs()
    pool, side = fs.PagePool(8, 1, 1, 64, 4, 9), torch.cuda.Stream()
    fs.page_grow(pool, [0], [130])
    torch.cuda.synchronize()
    given = side.cuda_stream if handle else side
    busy = _busy()
    got = [fs.page_grow(pool, [1], [64 * 9], stream=given), fs.page_fork(pool, [1], [0], stream=given),
           fs.page_grow(pool, [1], [128], stream=given), fs.page_fork(pool, [0], [2], stream=given)]
    fs.page_free(pool, [0], stream=given)
    got.append(fs.page_compact(pool, stream=given))
    junk = [torch.full((1,), 99, dtype=torch.int32, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    # 3 pages taken of 8; 9 do not fit; a destination is not empty; 2 do fit; the partial page is copied, to page 5; page 2 is free then
    assert [int(s) for s in got] == [-1, -2, 2, 1, 1] and len(junk) == 64 and float(busy[0]) == 30
