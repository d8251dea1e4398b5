"""Sampling at the sizes where its launches change form: scratch, borders of the cuts, rounding."""
import numpy as np
import pytest
import torch

from tests import cut_util

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


@pytest.mark.parametrize("vocab", [9000, 40000, 152064])
@pytest.mark.parametrize("near", [2e-5, 1e-6, 1e-3])
def test_min_p_just_below_one(vocab, near):
    """Scores that lie as near to the largest as min-p lies to 1: the border falls among thousands of them, in the narrowest bins."""
    fs, r = _fs(), np.random.default_rng(vocab)
    rows = 60 if vocab < 100000 else 12
    lg = -(r.uniform(0, near, (rows, vocab))).astype(np.float32)
    lg[:, 7] = 0
    m, u = (1 - r.uniform(0, near, rows)).astype(np.float32), r.random(rows)
    print(f"[case] min-p near 1, {rows}x{vocab}, within {near}", flush=True)
    dev = lambda a: torch.from_numpy(a).cuda()
    for how in ((1.0, 0, 1.0, m), (1.0, 0, 0.9, m), (1.0, vocab // 2, 1.0, m)):
        token, _, kept = (o.cpu().numpy() for o in fs.sample_tokens(dev(lg), dev(u), *how[:3], dev(m)))
        for i in range(rows):
            want = cut_util.sample(lg[i], u[i], *how[:3], m[i])
            assert (token[i], kept[i]) == (want[0], want[2]), (i, m[i], kept[i], want)


def _fused(row, temperature):
    """Weights if the score were not rounded before the largest is taken off it (one fused step for both)."""
    x, inv = row.astype(np.longdouble), np.longdouble(np.float32(1) / np.float32(temperature))
    m = (row * (np.float32(1) / np.float32(temperature))).astype(np.float32).max()
    return cut_util.weights((x * inv - np.longdouble(m)).astype(np.float32))


@pytest.mark.parametrize("vocab", [500, 6000, 20000, 60000])
def test_scores_are_rounded_before_the_largest_is_taken_off(vocab):
    """Logits so large that a score's own rounding moves its weight by a percent: every form of sampling and of acceptance has to round it alike."""
    from paper_2507_02620_amd import synth
    fs, r, rows, t = _fs(), np.random.default_rng(vocab), 16, 0.7
    lg = (3e5 + r.normal(0, 2, (rows, vocab))).astype(np.float32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    print(f"[case] large logits, {rows}x{vocab}", flush=True)
    other = 0
    for how in ((t, 0, 1.0, 0.0), (t, 0, 0.9, 0.0), (t, 40, 1.0, 0.0), (t, 0, 1.0, 0.05), (t, vocab // 3, 0.95, 0.0)):
        u = r.random(rows)
        token, _, kept = (o.cpu().numpy() for o in fs.sample_tokens(dev(lg), dev(u), *how))
        for i in range(rows):
            want = cut_util.sample(lg[i], u[i], *how)
            assert (token[i], kept[i]) == (want[0], want[2]), (i, how)
            if how[1:] == (0, 1.0, 0.0):
                w = _fused(lg[i], t)
                other += want[0] != cut_util.first_beyond(w, int(u[i] * 2.0 ** 48) * int(w.sum()) >> 48)
    assert other > 0                                      # (these inputs tell the two apart)
    tree = synth.random_tree(rows, 3, 8, vocab, 3)
    tok, par = dev(tree.token.astype(np.int32)), dev(tree.parent.astype(np.int32))
    for step in range(8):
        res, retain, work = fs.new_accept_buffers(rows, rows)
        fs.tree_accept_sample(dev(lg), t, tok, par, rows, 7, step, res, retain)
        free = fs.accept_result_to_host(res, retain, rows)
        fs.tree_accept_filtered(dev(lg), t, 0, 1.0, 0.0, tok, par, rows, 7, step, res, retain)
        cut = fs.accept_result_to_host(res, retain, rows)
        want = cut_util.accept(lg, (t, 0, 1.0, 0.0), tree.token.tolist(), tree.parent.tolist(), rows, 7, step)
        for got, kept in (free, cut):
            assert got.as_tuple() == want[0] and kept.tolist() == want[1], step
