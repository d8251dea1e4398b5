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


@pytest.mark.parametrize("handle", [False, True])
def test_results_written_beside_a_busy_stream(handle):
    """Blocks whose last owner's work is still queued on the current stream are not what a call on another stream writes to."""
    fs = _fs()
    side = torch.cuda.Stream()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    q = torch.randn((200, 8, 128), device="cuda", generator=g).to(torch.bfloat16)
    k = torch.randn((200, 2, 128), device="cuda", generator=g).to(torch.bfloat16)
    kv = torch.randn((1, 2, 2, 3000, 128), device="cuda", generator=g).to(torch.bfloat16)
    pool = fs.PagePool(4, 1, 2, 128, 1, 1)
    items = fs.paged_items([(0, 0, kv, 2800, 0, 200)])
    want = [fs.prompt_attention(q, k, k, [0, 200]), fs.paged_attention(pool, 0, q, items)]
    work = fs.paged_attention_workspace(pool, 8, 200)
    torch.cuda.synchronize()
    given = side.cuda_stream if handle else side
    busy = _busy()
    old = [torch.empty_like(q) for _ in range(4)] + [torch.empty_like(work) for _ in range(2)]
    for t in old:
        t.fill_(7)                                        # queued behind the work above
    del old, t
    got = [fs.prompt_attention(q, k, k, [0, 200], stream=given), fs.paged_attention(pool, 0, q, items, stream=given)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and float(busy[0]) == 30
