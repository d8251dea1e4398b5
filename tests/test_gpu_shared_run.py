"""Several continuations of one prompt as they are used: the prompt settles in pages, sequences fork from it, first tokens are sampled, draft trees
behind them are verified over the shared pages, accepted under the same cuts, and the caches behind the pages are pruned; twice."""
import numpy as np
import pytest
import torch

from paper_2507_02620_amd import synth
from tests import cut_util

pytestmark = pytest.mark.gpu

HOW = [(0.8, 50, 0.95, 0.0), (1.0, 0, 0.9, 0.02), (1.3, 0, 1.0, 0.0)]


@pytest.mark.parametrize("dtype,hq,hkv,hd,d,ffn", [("f32", 4, 2, 64, 256, 688), ("bf16", 8, 2, 64, 512, 1408), ("bf16", 4, 4, 128, 512, 1408)])
def test_continuations_of_one_prompt(dtype, hq, hkv, hd, d, ffn):
    from paper_2507_02620_amd import flowspec as fs
    from tests.gpu_util import TOL, Pair, max_rel_err, to_dev
    print(f"[case] continuations {dtype} {hq}/{hkv}x{hd}", flush=True)
    n, l_glo, vocab, T = 4, 300, 1500, 24
    cfg = synth.StageConfig("run", dtype, 2, d, hq, hkv, hd, ffn, vocab, l_glo, T, T, 8, 3)
    pair = Pair(cfg.with_(seg_len=n * T), seed=7, head=True, max_seg=n * T)
    pool = fs.PagePool(24, 2, hkv, hd, n, 8)
    fs.page_grow(pool, [0], [l_glo])
    fs.paged_store(pool, [(0, 0, pair.kv, 0, l_glo)])
    fs.page_fork(pool, [0] * (n - 1), list(range(1, n)))
    r = np.random.default_rng(3)
    # the prompt's last logits, once for each continuation, under settings of its own
    first = pair.gpu.tree_logits(to_dev(synth.hidden(cfg, 1, 2, 7), pair.tdtype))[0].repeat(n, 1)
    u = r.random(n)
    t, k = np.array([0.8, 1.0, 0.0, 1.5], np.float32), np.array([40, 0, 3, 0], np.int32)
    token, logprob, kept = fs.sample_tokens(first, torch.from_numpy(u).cuda(), torch.from_numpy(t).cuda(), torch.from_numpy(k).cuda(), 0.95)
    for i in range(n):
        want = cut_util.sample(first[i].cpu().numpy(), u[i], t[i], k[i], 0.95, 0.0)
        assert (int(token[i]), int(kept[i])) == (want[0], want[2])
    # one tail for all steps; what is settled stays the prompt's whole pages
    tails = [torch.full((2, 2, hkv, 3 * T + 44, hd), float("nan"), dtype=pair.tdtype, device="cuda") for _ in range(n)]
    for tail in tails:
        tail[:, :, :, :l_glo - 256] = pair.kv[:, :, :, 256:l_glo]
    lengths = [l_glo] * n
    root = token.cpu().numpy()
    for step in range(2):
        trees = [synth.random_tree(T - 3 * i, 8, 3, vocab, 11 + step, stream=i) for i in range(n)]
        for i, tree in enumerate(trees):
            tree.token[0] = root[i]
        items = [(i, 256, tails[i], lengths[i], 0, tree.size, tree.parent) for i, tree in enumerate(trees)]
        hid = to_dev(np.concatenate([synth.hidden(cfg, tree.size, 50 + 10 * step + i, 7) for i, tree in enumerate(trees)]), pair.tdtype)
        before = [tail.clone() for tail in tails]
        out = pair.gpu.tree_verify_shared(pool, items, [(n, 256)], hid)
        plain = pair.gpu.tree_verify_paged(pool, [(i, 256, before[i], *it[3:]) for i, it in enumerate(items)], hid)
        err = max_rel_err(out.float().cpu().numpy(), plain.float().cpu().numpy())
        print(f"  step {step}: {hid.shape[0]} rows, distance from the call without groups {err:.2e}", flush=True)
        assert err < TOL[dtype]
        # what the other sequences' rows of the table name in place of the shared pages is not read
        table = pool.table.clone()
        pool.table[1:, :4] = -1
        again = pair.gpu.tree_verify_shared(pool, [(i, 256, before[i], *it[3:]) for i, it in enumerate(items)], [(n, 256)], hid)
        pool.table.copy_(table)
        assert torch.equal(again, out)
        at = 0
        for i, tree in enumerate(trees):
            m = tree.size
            logits = pair.gpu.tree_logits(out[at:at + m])[0]
            at += m
            for c in range(1, m):                       # drafts that are often right
                if c % 2:
                    logits[tree.parent[c], tree.token[c]] += 4
            how = HOW[(i + step) % len(HOW)]
            res, retain, _ = fs.new_accept_buffers(m, 1)
            dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
            fs.tree_accept_filtered(logits, *how, dev(tree.token), dev(tree.parent), m, 5, step, res, retain)
            got, kept_nodes = fs.accept_result_to_host(res, retain, m)
            want = cut_util.accept(logits.cpu().numpy(), how, tree.token.tolist(), tree.parent.tolist(), m, 5, step)
            assert got.as_tuple() == want[0] and kept_nodes.tolist() == want[1]
            new_len = torch.zeros(2, dtype=torch.int32, device="cuda")
            front, n_acc = lengths[i] - 256, want[0][0]
            held = tails[i][:, :, :, front:front + m].clone()
            # the accepted path moves to the front of the drafts' slots, ordered by the acceptance on the device
            pair.gpu.kv_compact(tails[i], front, front + m, retain, res=res, new_len=new_len)
            path = want[1][:n_acc]
            assert torch.equal(tails[i][:, :, :, front:front + n_acc], held[:, :, :, path])
            lengths[i] += n_acc
            root[i] = want[0][1]
        print(f"  lengths now {lengths}", flush=True)
    fs.page_free(pool, list(range(n)))
    assert int(pool.ref.abs().sum()) == 0


def test_two_graphs_with_scratch_of_their_own():
    """A graph of one step's shared attention and sampling beside another one's, replayed on two streams: nothing of one is in the other."""
    from paper_2507_02620_amd import flowspec as fs
    from tests.test_gpu_shared_attention import Shared
    from tests.test_gpu_paged_attention import _words
    r = np.random.default_rng(5)
    sets = []
    for j in range(2):
        c = Shared([(700, 640, 2, 9), (690, 640, 0, 20), (640, 640, 0, 5)], [(3, 640)], 8, 2, 128, torch.bfloat16, 31 + j)
        x = torch.from_numpy(r.normal(0, 2, (6, 40000)).astype(np.float32)).cuda()
        u = torch.from_numpy(r.random(6)).cuda()
        items, groups, anc = fs.paged_items(c.items()), fs.prefix_groups(c.groups), _words(c.masks)
        works = fs.shared_attention_workspace(c.pool, 8, c.q.shape[0]), fs.sample_workspace(6, 40000)
        out, tok = torch.empty_like(c.q), fs.sample_tokens(x, u, 0.9, 0, 0.9)

        def run(c=c, x=x, u=u, items=items, groups=groups, anc=anc, works=works, out=out, tok=tok):
            fs.shared_attention(c.pool, 0, c.q, items, groups, out=out, anc=anc, workspace=works[0])
            fs.sample_tokens(x, u, 0.9, 0, 0.9, 0.0, *tok, workspace=works[1])
        run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        sets.append((graph, [out, *tok], [t.clone() for t in (out, *tok)], torch.cuda.Stream(), run))
    for i in range(4):
        for _, got, _, _, _ in sets:
            for t in got:
                t.fill_(3)
        torch.cuda.synchronize()
        for graph, _, _, s, _ in sets:
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for _, got, want, _, _ in sets:
            assert all(torch.equal(a, b) for a, b in zip(got, want)), i


@pytest.mark.parametrize("handle", [False, True])
def test_results_beside_a_busy_stream(handle):
    """Memory that the calls allocate themselves is that of the stream they are given."""
    from paper_2507_02620_amd import flowspec as fs
    from tests.test_gpu_given_stream import _busy
    from tests.test_gpu_shared_attention import Shared
    c = Shared([(700, 640, 2, 9), (690, 640, 0, 20), (640, 640, 0, 5)], [(3, 640)], 8, 2, 128, torch.bfloat16, 3)
    r = np.random.default_rng(5)
    x, u = torch.from_numpy(r.normal(0, 2, (40, 30000)).astype(np.float32)).cuda(), torch.from_numpy(r.random(40)).cuda()
    dev = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
    token, parent = dev(r.integers(0, 30000, 40)), dev([-1] + [i // 2 for i in range(39)])
    buf = fs.new_accept_buffers(40, 1)[:2], fs.new_accept_buffers(40, 1)[:2]

    def calls(b, **kw):
        out = [c.run(chain=True, **kw), *fs.sample_tokens(x, u, 0.9, 0, 0.9, **kw)]
        fs.tree_accept_filtered(x, 0.9, 0, 0.9, 0.0, token, parent, 40, 1, 2, *b, **kw)
        return out

    want = calls(buf[0])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy = _busy()
    old = [torch.empty_like(want[0]) for _ in range(4)] + [fs.sample_workspace(40, 30000) for _ in range(3)] + [torch.empty(40, dtype=torch.int32, device="cuda") for _ in range(6)]
    for t in old:
        t.fill_(7)                                        # queued behind the work above
    del old, t
    got = calls(buf[1], stream=side.cuda_stream if handle else side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(buf[0][0], buf[1][0]) and float(busy[0]) == 30
