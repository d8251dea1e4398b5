"""Argument sizes at which 32-bit products of the host side would wrap.  CPU only: pointers here are never followed."""
import ctypes as C

P = 1 << 20  # stands for a device pointer


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


def test_scratch_of_very_many_rows():
    """Heads times row blocks of 2^32 and more ended the process in a division by zero."""
    fs = _fs()
    f = fs.lib().fs_paged_attention_workspace_bytes
    for heads, kv_heads, rows in ((65536, 65536, 1 << 22), (1 << 21, 1 << 20, 1 << 18), (1 << 20, 1, 1 << 12), (1 << 16, 1 << 16, (1 << 31) - 1)):
        assert f(heads, kv_heads, 128, rows) >= rows * heads * 130 * 4 % (1 << 64)
    # one split from 256 blocks of 64 rows on; rows are padded to 16
    assert f(65536, 65536, 128, 1 << 22) == (1 << 38) * 130 * 4
    assert f(4, 4, 64, 1) == 64 * 4 * 16 * 66 * 4 and f(4, 4, 64, 64 * 64) == 4 * 64 * 64 * 66 * 4


def test_attention_over_pages_of_very_many_heads():
    fs = _fs()
    heads, kv_heads = 1 << 23, 1 << 15
    pool = C.byref(fs.PagePoolDesc(P, P, P, P, P, P, 8, 1, kv_heads, 128, 4, 3))
    kv = fs.KVCache(P, 8192, 4096, 2048, 128)
    items = (fs.PagedItem * 32)(*[fs.PagedItem(0, 0, kv, 1 << 20, 0, 0, 1024, None)] * 32)
    for dtype in (fs.FS_BF16, fs.FS_F32):
        assert fs.lib().fs_paged_attention(pool, 0, dtype, heads, items, 32, None, P, heads * 128, 2 * P, heads * 128, 0.0, P, 1 << 40, None) == fs.FS_ECAP
