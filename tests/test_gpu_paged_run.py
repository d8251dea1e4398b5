"""The operators over pages and prompts as they are used together: a context moves into pages, sequences fork, segments are verified over
them, the cache behind the pages is pruned, the pool is made dense — against the oracle run on what the pages stand for."""
import math

import numpy as np
import pytest
import torch

from paper_2507_02620_amd import synth
from tests.paged_util import PAGE, attend, check, quantise, values

pytestmark = pytest.mark.gpu


def _paged_prefix(pool, seq, n, layer, hd):
    """[2, heads, n, hd] that the first n settled tokens of a sequence stand for."""
    ids = pool.table[seq].cpu().numpy()
    parts = [np.stack(values(pool.codes, pool.scales, int(ids[i]), layer, hd)) for i in range(-(-n // PAGE))]
    return np.concatenate(parts, axis=2)[:, :, :n]


@pytest.mark.parametrize("cfg,n_paged", [
    (synth.StageConfig("p-f32", "f32", 2, 256, 4, 2, 64, 688, 0, 150, 40, 16, 6, 3), 128),
    (synth.StageConfig("p-gqa", "bf16", 2, 512, 8, 2, 64, 1408, 0, 300, 40, 16, 6, 3, qkv_bias=True), 300),
    (synth.StageConfig("p-128", "bf16", 2, 512, 4, 4, 128, 1408, 0, 250, 48, 24, 40, 2), 192),
], ids=lambda x: getattr(x, "name", str(x)))
def test_a_serving_round_over_pages(cfg, n_paged):
    from oracle import oracle
    from paper_2507_02620_amd import flowspec as fs
    from tests.gpu_util import TOL, Pair, max_rel_err, to_dev
    print(f"[case] round {cfg.name}", flush=True)
    pair = Pair(cfg.with_(seg_len=4 * cfg.seg_len), seed=3, max_seg=4 * cfg.seg_len)
    L, hd, l_glo = cfg.n_layers, cfg.head_dim, cfg.l_glo
    pool = fs.PagePool(24, L, cfg.n_kv_heads, hd, 5, 8)
    # the context of sequence 0 settles; sequence 4 takes pages before it, sequences 1 and 2 fork from it
    fs.page_grow(pool, [4, 0], [200, n_paged])
    fs.paged_store(pool, [(0, 0, pair.kv, 0, n_paged)])
    fs.page_fork(pool, [0, 0], [1, 2])
    cap = l_glo - n_paged + cfg.tree_size + 8
    reqs = []
    for r in range(3):
        tail = torch.full((L, 2, cfg.n_kv_heads, cap, hd), float("nan"), dtype=pair.tdtype, device="cuda")
        tail[:, :, :, :l_glo - n_paged] = pair.kv[:, :, :, n_paged:l_glo]
        orc = oracle.Stage(cfg, pair.layers, None, None, l_glo + cfg.tree_size + 8)
        for l in range(L):
            pre = pair.kv[l].double().cpu().numpy()[:, :, :l_glo].copy()
            pre[:, :, :n_paged] = _paged_prefix(pool, r, n_paged, l, hd)
            orc.load_prefix(l, pre)
        tree = synth.random_tree(cfg.tree_size, cfg.max_depth, cfg.max_branch, 1000, 3, stream=r)
        reqs.append((tail, orc, tree, synth.hidden(cfg, cfg.tree_size, 5 + r, 3)))

    def step(seg, l_glo, n_paged, trees):
        items, rows, want = [], [], []
        for r, (off, n) in seg.items():
            tail, orc, _, _ = reqs[r]
            parent, hid = trees[r]
            items.append((r, n_paged, tail, l_glo[r], off, n, parent[:off + n]))
            rows.append(hid[off:off + n])
            want.append(orc.verify(l_glo[r], l_glo[r] + off, hid[off:off + n], off, parent[:off + n]))
        got = pair.gpu.tree_verify_paged(pool, fs.paged_items(items), to_dev(np.concatenate(rows), pair.tdtype)).float().cpu().numpy()
        at = 0
        for w in want:
            err = max_rel_err(got[at:at + len(w)], w)
            print(f"  {len(w)} rows, max-rel-err {err:.2e}", flush=True)
            assert err < TOL[cfg.dtype]
            at += len(w)

    trees = {r: (reqs[r][2].parent, reqs[r][3]) for r in range(3)}
    lg = {r: l_glo for r in range(3)}
    half = cfg.tree_size // 2
    step({0: (0, half), 1: (0, 7), 2: (0, 1)}, lg, n_paged, trees)
    # the pool becomes dense between two segments: nothing that is read changes
    fs.page_free(pool, [4])
    assert int(fs.page_compact(pool)) > 0
    step({0: (half, cfg.tree_size - half), 1: (7, 9)}, lg, n_paged, trees)
    # acceptance on request 0: a path of the tree stays, the cache behind the pages is pruned in place
    par = reqs[0][2].parent
    node = max(range(cfg.tree_size), key=lambda i: (synth_depth(par, i), -i))
    path = []
    while node >= 0:
        path.insert(0, node)
        node = int(par[node])
    retain = np.array(path, np.int32)
    new_len = torch.zeros(2, dtype=torch.int32, device="cuda")
    tail, orc = reqs[0][0], reqs[0][1]
    front = l_glo - n_paged
    pair.gpu.kv_compact(tail, front, front + cfg.tree_size, retain, n_acc=len(path), new_len=new_len)
    assert new_len.tolist() == [front + len(path)] * 2
    oracle.kv_compact(orc.kv, l_glo, l_glo + cfg.tree_size, retain, len(path))
    # the accepted tokens complete a page where there are enough of them: it settles, and the next segment reads it there
    lg[0] = l_glo + len(path)
    settled = n_paged
    if n_paged % PAGE == 0 and lg[0] - n_paged >= PAGE:
        settled = n_paged + PAGE
        assert int(fs.page_grow(pool, [0], [settled])) == 1
        fs.paged_store(pool, [(0, n_paged // PAGE, tail, 0, PAGE)])
        for l in range(L):
            orc.kv[l][:, :, :settled] = _paged_prefix(pool, 0, settled, l, hd)
        tail[:, :, :, :cap - PAGE] = tail[:, :, :, PAGE:].clone()
    tree2 = synth.random_tree(16, 5, 3, 1000, 3, stream=9)
    step({0: (0, 16)}, lg, settled, {0: (tree2.parent, synth.hidden(cfg, 16, 9, 3))})
    fs.page_free(pool, [0, 1, 2])
    assert int((pool.ref != 0).sum()) == 0 and int(pool.length.abs().sum()) == 0 and bool((pool.table == -1).all())
    if cfg.name == "p-128":
        assert settled == n_paged + PAGE  # (the last segment read a page that the accepted tokens had completed)


def synth_depth(parent, i):
    d = 0
    while parent[i] >= 0:
        i, d = int(parent[i]), d + 1
    return d


def test_prompts_to_pages_to_next_tokens():
    """Packed prompts through attention, their K and V into pages, children forked, one token each attended over the pages."""
    from paper_2507_02620_amd import flowspec as fs
    hq, hkv, hd, lens = 8, 2, 128, [300, 64, 129]
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    cu = np.cumsum([0] + lens)
    n = int(cu[-1])
    cache = torch.randn((1, 2, hkv, n, hd), device="cuda", generator=g).to(torch.bfloat16)
    q = torch.randn((n, hq, hd), device="cuda", generator=g).to(torch.bfloat16)
    k, v = cache[0, 0].transpose(0, 1), cache[0, 1].transpose(0, 1)
    got = fs.prompt_attention(q, k, v, cu)
    scale = 1 / math.sqrt(hd)
    for a, b in zip(cu[:-1], cu[1:]):
        seen = torch.tril(torch.ones((b - a, b - a), dtype=torch.bool, device="cuda"))
        for h in range(hq):
            check(got[a:b, h], *attend(q[a:b, h].double(), k[a:b, h // 4].double(), v[a:b, h // 4].double(), seen, scale, torch.bfloat16), "prompt")
    pool = fs.PagePool(32, 1, hkv, hd, 6, 8)
    assert int(fs.page_grow(pool, [0, 1, 2], lens)) == 9
    fs.paged_store(pool, [(s, 0, cache, int(cu[s]), lens[s]) for s in range(3)])
    assert int(fs.page_fork(pool, [0, 2, 0], [3, 4, 5])) == 3
    tails = [torch.randn((1, 2, hkv, 4, hd), device="cuda", generator=g).to(torch.bfloat16) for _ in range(6)]
    src = [0, 1, 2, 0, 2, 0]
    qt = torch.randn((6, hq, hd), device="cuda", generator=g).to(torch.bfloat16)
    got = fs.paged_attention(pool, 0, qt, [(i, lens[s], tails[i], lens[s] + 2, 0, 1) for i, s in enumerate(src)])
    for i, s in enumerate(src):
        rows = [[], []]
        for p in range(2):
            for h in range(hkv):
                tiles = []
                for j in range(0, lens[s], PAGE):
                    w, sc = quantise(cache[0, p, h, cu[s] + j:cu[s] + min(j + PAGE, lens[s])].double().cpu().numpy())
                    tiles.append(w * sc)
                rows[p].append(torch.cat([torch.from_numpy(np.concatenate(tiles)[:lens[s]]).cuda(), tails[i][0, p, h, :3].double()]))
        seen = torch.ones((1, lens[s] + 3), dtype=torch.bool, device="cuda")
        for h in range(hq):
            check(got[i:i + 1, h], *attend(qt[i:i + 1, h].double(), rows[0][h // 4], rows[1][h // 4], seen, scale, torch.bfloat16), "token")


def test_stage_refuses_pools_of_another_shape_and_full_caches():
    from paper_2507_02620_amd import flowspec as fs
    from tests.gpu_util import Pair, to_dev
    cfg = synth.StageConfig("p-ref", "f32", 1, 256, 4, 2, 64, 688, 0, 64, 16, 16, 5, 3)
    pair = Pair(cfg, seed=1)
    hid = to_dev(synth.hidden(cfg, 4), torch.float32)
    par = [-1, 0, 1, 2]

    def run(pool, tail=None, n_paged=64, l_glo=64, parent=par):
        tail = pair.kv if tail is None else tail
        return pair.gpu.tree_verify_paged(pool, fs.paged_items([(0, n_paged, tail, l_glo, 0, 4, parent)]), hid)

    good = fs.PagePool(2, 1, 2, 64, 1, 2)
    for pool in (fs.PagePool(2, 2, 2, 64, 1, 2), fs.PagePool(2, 1, 4, 64, 1, 2), fs.PagePool(2, 1, 2, 128, 1, 2)):
        with pytest.raises(fs.FlowSpecError) as e:
            run(pool)
        assert e.value.code == fs.FS_EINVAL
    for kw, code in ((dict(tail=pair.kv[:, :, :, :3]), fs.FS_ECAP), (dict(n_paged=65), fs.FS_EINVAL), (dict(parent=[-1, 0, 3, 1]), fs.FS_ETOPO),
                     (dict(n_paged=129, l_glo=200), fs.FS_ECAP)):
        with pytest.raises(fs.FlowSpecError) as e:
            run(good, **kw)
        assert e.value.code == code
