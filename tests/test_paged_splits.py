"""Which contexts of attention over pages are split, by whether the call asks for scratch.  CPU only: pointers here are never followed, and
only calls that the host refuses are made."""
import ctypes as C

import pytest

P = 1 << 20  # stands for a device pointer


@pytest.mark.parametrize("dtype,rows,slots", [("FS_F32", 1, 320), ("FS_F32", 16, 960), ("FS_F32", 300, 960), ("FS_BF16", 1, 1792), ("FS_BF16", 17, 1280), ("FS_BF16", 40, 640)])
def test_contexts_that_are_split(dtype, rows, slots):
    """32-bit queries: from the fifth page on, where four waves have a second round (1000 slots in one split took up to twice as long)."""
    from paper_2507_02620_amd import flowspec as fs
    pool = C.byref(fs.PagePoolDesc(P, P, P, P, P, P, 64, 1, 2, 64, 4, 40))
    item = (fs.PagedItem * 1)(fs.PagedItem(0, slots, fs.KVCache(P, 1 << 20, 1 << 19, 1 << 18, 64), 1024, slots, 0, rows, None))
    assert fs.lib().fs_paged_attention(pool, 0, getattr(fs, dtype), 2, item, 1, None, P, 128, 2 * P, 128, 0.0, None, 0, None) == fs.FS_EWS
