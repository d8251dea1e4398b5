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
