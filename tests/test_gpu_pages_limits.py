"""Page calls at the ends of their ranges."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


def test_growing_by_more_pages_than_32_bits_count():
    """128 and 256 sequences of 2^24 pages each: too few are free, whatever their sum wraps to, and nothing changes."""
    fs = _fs()
    n, width = 256, 1 << 24
    whole = fs.PagePool(300, 1, 1, 64, n, 2)
    table = torch.empty((n, width), dtype=torch.int32, device="cuda")  # (16 GiB; a call touches what it appends)
    table[:, :4] = -1
    pool = fs.PagePool.of(whole.codes, whole.scales, whole.ref, table, whole.length)
    most = width * 64
    assert int(fs.page_grow(pool, [0, 1], [130, 64])) == 4
    for seqs in (range(n), range(128), range(100, 229), [5], [0, 9]):
        assert int(fs.page_grow(pool, list(seqs), [most] * len(seqs))) == -1
        assert pool.length.tolist() == [130, 64] + [0] * 254 and int(pool.ref.sum()) == 4 and int((pool.ref != 0).sum()) == 4
    assert int(fs.page_grow(pool, [0, 1, 2], [most, 63, most])) == -2
    assert pool.length[:3].tolist() == [130, 64, 0] and bool((table[2:, :4] == -1).all())
    assert int(fs.page_grow(pool, list(range(2, 256)), [64] * 254)) == 254 and table[2:, 0].tolist() == list(range(4, 258))
    # as many as there are, and one more
    assert int(fs.page_grow(pool, [255], [64 * 44])) == -1
    assert int(fs.page_grow(pool, [255], [64 * 43])) == 42 and int((pool.ref == 0).sum()) == 0
    assert int(fs.page_grow(pool, [0], [192])) == 0
