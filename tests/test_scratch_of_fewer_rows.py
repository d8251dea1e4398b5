"""Scratch that a program asks for once, for the most rows that it has, serves calls of fewer rows: its size never falls as rows grow.  CPU only."""
import pytest


def _lib():
    from paper_2507_02620_amd import flowspec as fs
    return fs.lib()


@pytest.mark.parametrize("vocab", [1, 8192, 8193, 32000, 50257, 128256, 152064, 1 << 20])
def test_sampling(vocab):
    """Few rows are cut into short chunks, many into long ones, which take less scratch a row."""
    w = _lib().fs_sample_workspace_bytes
    sizes = [w(rows, vocab) for rows in [*range(1, 5600), 16384, 16385, 65535]]
    assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (32, 32), (28, 4), (8, 1), (3, 3), (40, 40), (600, 300)])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_over_pages(heads, kv_heads, hd):
    """Few rows are split further than many, and whole splits leave a remainder: five blocks of 64 rows are 12 splits of 320, four are 16 of 256."""
    for w in (_lib().fs_paged_attention_workspace_bytes, _lib().fs_shared_attention_workspace_bytes):
        sizes = [w(heads, kv_heads, hd, rows) for rows in [*range(1, 2100), 4096, 4097, 32768]]
        assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
