"""Sampling at the sizes where its launches change form: scratch, borders of the cuts, rounding."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


def test_one_scratch_for_all_batches_of_a_program():
    """Asked for once, for the most rows (long chunks), and used by smaller batches (short ones) as well."""
    fs, rows, vocab = _fs(), 65, 1 << 20
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn((rows, vocab), device="cuda", generator=g).mul_(2.5)
    u = torch.rand(rows, dtype=torch.float64, device="cuda", generator=g)
    work = fs.sample_workspace(rows, vocab)
    for n in (65, 64, 7, 1, 65):
        for how in ((0.8, 40, 0.9, 0.0), (1.0, 0, 0.9, 0.0)):
            print(f"[case] scratch for {rows} rows, {n} in use, {how}", flush=True)
            got = fs.sample_tokens(x[:n], u[:n], *how, workspace=work)
            want = [o[:n] for o in fs.sample_tokens(x, u, *how)]
            assert all(torch.equal(a, b) for a, b in zip(got, want))
