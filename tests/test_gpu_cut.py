"""Sampling of tokens under temperature, top-k, top-p and min-p, and acceptance of a draft tree under the same cuts: whole numbers on both
sides, so tokens and counts have to be equal.  logprob is a logarithm in 64 bits of a quotient of whole numbers, rounded once: half a step of
2^-24 of its size, and the two libraries' 64-bit logarithms, 2^-48."""
import numpy as np
import pytest
import torch

from paper_2507_02620_amd import synth
from tests import cut_util

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HOW = [(1.0, 0, 1.0, 0.0), (0.8, 50, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.7, 20, 0.95, 0.0), (1.2, 0, 1.0, 0.05), (0.9, 200, 0.5, 0.02), (0.0, 7, 0.3, 0.5),
       (1.7, 3000, 0.99, 1e-4), (30.0, 0, 0.6, 0.0), (1.0, 1, 1.0, 0.0)]


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


def _logits(r, rows, vocab, std=2.0):
    x = r.normal(0, std, (rows, vocab)).astype(np.float32)
    for i in range(rows):
        at = r.integers(0, vocab, min(vocab, 12))
        x[i, at] += (r.uniform(0, 14) / np.sqrt(1 + np.arange(len(at)))).astype(np.float32)
    return x


def _check(lg, dtype, u, how, **kw):
    """how: (temperature, top_k, top_p, min_p), each a number or an array with an entry per row."""
    fs = _fs()
    x = torch.from_numpy(lg).cuda().to(DTYPES[dtype])
    rows = lg.shape[0]
    given = [torch.from_numpy(np.ascontiguousarray(v)).cuda() if isinstance(v, np.ndarray) else v for v in how]
    got = fs.sample_tokens(x, torch.from_numpy(np.ascontiguousarray(u)).cuda(), *given, **kw)
    token, logprob, kept = (t.cpu().numpy() for t in got)
    seen = x.float().cpu().numpy()
    for i in range(rows):
        want = cut_util.sample(seen[i], float(u[i]), *(v[i] if isinstance(v, np.ndarray) else v for v in how))
        assert (token[i], kept[i]) == (want[0], want[2]), (i, token[i], kept[i], want)
        if np.isfinite(want[1]):
            assert abs(logprob[i] - want[1]) <= abs(want[1]) * (2.0 ** -24 + 2.0 ** -48), (i, logprob[i], want[1])
        else:
            assert logprob[i] == want[1]
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 3, 63, 64, 65, 255, 1000, 1024, 4095, 4097, 10007, 32000])
def test_tokens(dtype, vocab):
    r = np.random.default_rng(vocab)
    rows = 7 if vocab <= 4097 else 3
    for how in HOW:
        print(f"[case] sample {dtype} {rows}x{vocab} {how}", flush=True)
        _check(_logits(r, rows, vocab), dtype, r.random(rows), how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(1, 152064), (2, 152063), (5, 65537), (37, 8192), (260, 1500), (70, 40000)])
def test_large_and_many(dtype, rows, vocab):
    r = np.random.default_rng(rows)
    print(f"[case] sample {dtype} {rows}x{vocab}", flush=True)
    lg = _logits(r, rows, vocab)
    how = (r.choice(np.array([0, 0.6, 1, 1.3, 8], np.float32), rows), r.choice(np.array([0, 0, 1, 20, 1000, vocab], np.int32), rows),
           r.choice(np.array([1, 0.95, 0.5, 0], np.float32), rows), r.choice(np.array([0, 0.05, 1], np.float32), rows))
    _check(lg, dtype, r.random(rows), how)
    _check(lg, dtype, r.random(rows), (0.7, 50, 0.95, 0.0))
    _check(lg, dtype, r.random(rows), (2.5, 0, 0.999, 0.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(65535, 30), (550, 124003), (560, 122880)])
def test_most_rows(dtype, rows, vocab):
    """The most rows that a call takes, and so many chunks that long ones are taken; some of the rows are compared."""
    fs, r = _fs(), np.random.default_rng(rows)
    print(f"[case] sample {dtype} {rows}x{vocab}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    x = (torch.randn((rows, vocab), device="cuda", generator=g) * 2.5).to(DTYPES[dtype])
    u = r.random(rows)
    some = np.unique(np.concatenate([[0, 1, rows - 1], r.integers(0, rows, 60 if vocab < 100 else 9)]))
    t, k = r.choice(np.array([0, 0.6, 1, 1.3], np.float32), rows), r.choice(np.array([0, 1, 20, 700, 2000], np.int32), rows)
    p, m = r.choice(np.array([1, 0.95, 0.5], np.float32), rows), r.choice(np.array([0, 0.05], np.float32), rows)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    work = fs.sample_workspace(rows, vocab)
    seen = x[torch.from_numpy(some).cuda()].float().cpu().numpy()
    for how in ((t, k, p, m), (0.8, 40, 0.9, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.01)):
        token, _, kept = (o.cpu().numpy() for o in fs.sample_tokens(x, dev(u), *(dev(v) if isinstance(v, np.ndarray) else v for v in how), workspace=work))
        for j, i in enumerate(some):
            want = cut_util.sample(seen[j], float(u[i]), *(v[i] if isinstance(v, np.ndarray) else v for v in how))
            assert (token[i], kept[i]) == (want[0], want[2]), (i, how)


def _special(vocab, r):
    inf, nan = np.inf, np.nan
    rows = [np.zeros(vocab), np.full(vocab, -inf), np.full(vocab, nan), np.where(np.arange(vocab) % 3 == 1, 1.0, -inf), np.full(vocab, -3e38), np.full(vocab, 3e38)]
    for v, n in ((inf, 1), (inf, 3), (nan, 5), (-inf, vocab - 1)):
        x = r.normal(0, 2, vocab)
        x[r.permutation(vocab)[:min(n, vocab)]] = v
        rows.append(x)
    x = np.zeros(vocab)
    x[::2] = -0.0                                    # -0 is 0: the lower index comes first
    rows.append(x)
    rows.append(r.integers(-2, 3, vocab) * 0.5)        # few values, each many times
    rows.append(r.normal(0, 1e-6, vocab))              # nearly equal
    rows.append(r.normal(0, 1e-42, vocab))             # below the normal numbers
    rows.append(r.normal(0, 30, vocab))                # most weigh nothing
    rows.append(-np.arange(vocab) * 0.01)
    rows.append(np.where(np.arange(vocab) == vocab // 2, inf, -inf))
    return np.stack(rows).astype(np.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 300, 6000, 50000])
def test_ties_infinities_and_rows_of_nothing(dtype, vocab):
    r = np.random.default_rng(vocab)
    lg = _special(vocab, r)
    for how in HOW[:6] if vocab > 10000 else HOW + [(1.0, 2, 0.5, 0.0), (1.0, 0, 0.0, 0.0), (2.0 ** 100, 0, 0.5, 0.0), (2.0 ** -100, 3, 0.5, 0.0), (1.0, 0, 0.5, 2.0),
                                                    (0.5, vocab - 1, 1.0, -1.0), (1.0, -5, 7.0, 0.0), (1e6, vocab // 2 + 1, 0.75, 0.0)]:
        print(f"[case] special {dtype} {vocab} {how}", flush=True)
        _check(lg, dtype, r.random(lg.shape[0]), how)


def test_uniform_numbers_at_and_beyond_the_ends():
    r = np.random.default_rng(3)
    u = np.array([0.0, 2.0 ** -60, 2.0 ** -48, 0.5, 1 - 2.0 ** -53, 1.0, 1.5, -0.25, np.nan, np.inf, -np.inf])
    lg = np.repeat(_logits(r, 1, 900), len(u), axis=0)
    for how in HOW[:5]:
        _check(lg, "f32", u, how)
    top = _check(np.zeros((len(u), 900), np.float32), "f32", u, (1.0, 0, 1.0, 0.0))[0].cpu().numpy()
    assert top[0] == 0 == top[7] == top[8] and top[4] == top[5] == top[6] == top[9] == 899


def test_settings_out_of_range_leave_their_rows_without_a_token():
    r = np.random.default_rng(4)
    f = lambda *v: np.array(v, np.float32)
    t = f(1, -1, np.nan, np.inf, 2.0 ** 101, 1e-35, 1, 1, 1, 0)
    p = f(0.9, 0.9, 0.9, 0.9, 0.9, 0.9, np.nan, 0.9, np.inf, 0.9)
    m = f(0, 0, 0, 0, 0, 0, 0, np.nan, np.inf, 0)
    got = _check(_logits(r, 10, 700), "f32", r.random(10), (t, np.full(10, 40, np.int32), p, m))
    assert (got[0].cpu().numpy() >= 0).tolist() == [True] + [False] * 7 + [True] * 2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_rows_and_given_buffers(dtype):
    fs, r = _fs(), np.random.default_rng(8)
    big = torch.from_numpy(_logits(r, 9, 1111)).cuda().to(DTYPES[dtype])
    big[:, 1003:] = float("inf")                       # behind the rows: never read
    big[:, :3] = float("nan")
    x, u = big[:, 3:1003], torch.from_numpy(r.random(9)).cuda()
    out = [torch.full((11,), 77, dtype=d, device="cuda") for d in (torch.int32, torch.float32, torch.int32)]
    work = torch.full((fs._lib.fs_sample_workspace_bytes(9, 1000),), 255, dtype=torch.uint8, device="cuda")
    fs.sample_tokens(x, u, 0.9, 30, 0.9, 0.01, *(o[1:10] for o in out), workspace=work)
    want = fs.sample_tokens(x.contiguous(), u, 0.9, 30, 0.9, 0.01)
    for o, w in zip(out, want):
        assert torch.equal(o[1:10], w) and float(o[0]) == float(o[10]) == 77
    one = fs.sample_tokens(big[4:5, 3:1003], u[4:5], 0.9, 30, 0.9, 0.01)
    assert [float(a[0]) for a in one] == [float(w[4]) for w in want]
    assert fs.sample_tokens(x[:0], u[:0])[0].numel() == 0


@pytest.mark.parametrize("rows,vocab", [(1, 152064), (16, 32000), (300, 2000)])
def test_replayed_from_a_graph(rows, vocab):
    """Scratch of the capture is used by every replay and by nothing else; logits, numbers and settings change between replays."""
    fs, r = _fs(), np.random.default_rng(rows)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    x, u = dev(_logits(r, rows, vocab)), dev(r.random(rows))
    t, k = dev(np.ones(rows, np.float32)), dev(np.zeros(rows, np.int32))
    work, other = fs.sample_workspace(rows, vocab), fs.sample_workspace(rows, vocab)
    out = fs.sample_tokens(x, u, t, k, 0.9, 0.0, workspace=work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fs.sample_tokens(x, u, t, k, 0.9, 0.0, *out, workspace=work)
    for i in range(4):
        x.copy_(dev(_logits(r, rows, vocab)))
        u.copy_(dev(r.random(rows)))
        t.fill_([0.7, 0.0, 1.5, 1.0][i])
        k.fill_([40, 0, 0, 5000][i])
        graph.replay()
        got = [o.clone() for o in out]
        want = fs.sample_tokens(x, u, t, k, 0.9, 0.0, workspace=other)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_streams_at_once():
    fs, r = _fs(), np.random.default_rng(11)
    jobs = []
    for i in range(2):
        x, u = torch.from_numpy(_logits(r, 24, 60000)).cuda(), torch.from_numpy(r.random(24)).cuda()
        jobs.append((x, u, fs.sample_tokens(x, u, 0.9, 0, 0.9), torch.cuda.Stream(), []))
    torch.cuda.synchronize()
    for _ in range(8):
        for x, u, _, s, got in jobs:
            got.append(fs.sample_tokens(x, u, 0.9, 0, 0.9, stream=s))
    torch.cuda.synchronize()
    for _, _, want, _, got in jobs:
        assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))


# ---- acceptance ------------------------------------------------------------------------------------------------------------------

def _accept(lg, how, token, parent, n_ver, seed, step):
    fs = _fs()
    res, retain, _ = fs.new_accept_buffers(len(token), 1)
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    fs.tree_accept_filtered(d(lg), *how, d(np.asarray(token, np.int32)), d(np.asarray(parent, np.int32)), n_ver, seed, step, res, retain)
    out, ret = fs.accept_result_to_host(res, retain, len(token))
    return out.as_tuple(), ret.tolist()


@pytest.mark.parametrize("seed", range(14))
def test_accepted_trees(seed):
    r = np.random.default_rng(seed)
    T = int(r.choice([1, 2, 9, 64, 65, 200]))
    vocab = int(r.choice([2, 7, 50, 1000, 20000]))
    tree = synth.random_tree(T, int(r.choice([3, 8, 30])), int(r.choice([0, 2, 4])), vocab, seed, forest=bool(seed % 4 == 0))
    n_ver = int(r.integers(0, T + 1))
    lg = _logits(r, max(n_ver, 1), vocab, 1.5)
    if seed % 2:                                       # long accepted paths likely
        for row, t in synth.resolve_plants(synth.plant_path(tree, n_ver, seed, 0, 0.3, 5.0), tree, vocab):
            lg[row, t] += 6.0
    if seed % 3 == 0 and T > 3:
        tree.token[T // 2] = vocab + 3                  # not a token of the vocabulary
        tree.token[T - 1] = tree.token[T - 2]            # perhaps the same token twice under one node
    for i, how in enumerate(HOW):
        if how[0] == 0:
            continue
        print(f"[case] accept T={T} n_ver={n_ver} vocab={vocab} {how}", flush=True)
        want = cut_util.accept(lg, how, tree.token.tolist(), tree.parent.tolist(), n_ver, 99 + seed, i)
        got = _accept(lg, how, tree.token, tree.parent, n_ver, 99 + seed, i)
        assert got[0] == want[0] and got[1] == want[1], (got, want)


@pytest.mark.parametrize("T,n_ver,vocab", [(1, 1, 152064), (20, 3, 152064), (40, 20, 60001), (1024, 1024, 64)])
def test_accepted_trees_draw_from_large_vocabularies(T, n_ver, vocab):
    r = np.random.default_rng(T)
    lg = _logits(r, n_ver, vocab)
    par = np.array([-1] + [int(r.integers(0, max(1, min(i, n_ver)))) for i in range(1, T)], np.int32) if T < 1000 else np.arange(-1, T - 1, dtype=np.int32)
    tok = r.integers(0, vocab, T).astype(np.int32)
    if T == 1024:
        lg[np.arange(T - 1), tok[1:]] += 20
    for step, how in enumerate([(1.0, 0, 0.9, 0.0), (0.8, 40, 1.0, 0.0), (1.5, 0, 0.99, 1e-3), (1.0, 0, 1.0, 0.0)]):
        want = cut_util.accept(lg, how, tok.tolist(), par.tolist(), n_ver, 5, step)
        assert _accept(lg, how, tok, par, n_ver, 5, step) == (want[0], want[1])
        assert T < 1000 or want[0][0] > 20  # (the definition itself walks 43 nodes down at least)


@pytest.mark.parametrize("seed", range(6))
def test_without_cuts_it_is_the_acceptance_at_a_temperature(seed):
    fs, r = _fs(), np.random.default_rng(seed)
    T, vocab = int(r.choice([8, 64, 300])), int(r.choice([40, 5000, 70000]))
    tree = synth.random_tree(T, 8, 4, vocab, seed)
    n_ver = int(r.integers(1, min(T, 64) + 1))
    lg = _logits(r, n_ver, vocab, 1.0)
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    for step in range(4):
        res, retain, _ = fs.new_accept_buffers(T, 1)
        fs.tree_accept_sample(d(lg), 0.8, d(tree.token.astype(np.int32)), d(tree.parent.astype(np.int32)), n_ver, seed, step, res, retain)
        out, ret = fs.accept_result_to_host(res, retain, T)
        assert _accept(lg, (0.8, 0, 1.0, 0.0), tree.token, tree.parent, n_ver, seed, step) == (out.as_tuple(), ret.tolist())


def test_a_broken_tree_is_reported():
    lg = np.zeros((2, 50), np.float32)
    assert _accept(lg, HOW[3], [1, 2, 3], [-1, 2, 0], 2, 1, 1)[0][0] == -1


def test_rows_of_nothing_under_a_tree():
    """A verified row that rules every token out: no child is accepted, and the draw's default is the last token."""
    lg = np.full((2, 300), -np.inf, np.float32)
    for how in (HOW[0], HOW[3]):
        want = cut_util.accept(lg, how, [5, 6, 7], [-1, 0, 0], 2, 1, 1)
        assert _accept(lg, how, [5, 6, 7], [-1, 0, 0], 2, 1, 1) == (want[0], want[1]) and want[0][1] == 299


def test_acceptance_replayed_from_a_graph():
    fs, r = _fs(), np.random.default_rng(2)
    T, vocab, n_ver = 40, 60000, 30
    tree = synth.random_tree(T, 8, 4, vocab, 1)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    x, tok, par = dev(_logits(r, n_ver, vocab)), dev(tree.token.astype(np.int32)), dev(tree.parent.astype(np.int32))
    work = fs.sample_workspace(n_ver, vocab)
    res, retain, _ = fs.new_accept_buffers(T, 1)
    run = lambda a, b, w: fs.tree_accept_filtered(x, 0.9, 0, 0.9, 0.0, tok, par, n_ver, 3, 4, a, b, workspace=w)
    run(res, retain, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(res, retain, work)
    for i in range(4):
        x.copy_(dev(_logits(r, n_ver, vocab, 1.0 + i)))
        retain.zero_()
        graph.replay()
        got = res.clone(), retain.clone()
        res2, retain2, _ = fs.new_accept_buffers(T, 1)
        run(res2, retain2, fs.sample_workspace(n_ver, vocab))
        assert torch.equal(got[0], res2) and torch.equal(got[1], retain2)
