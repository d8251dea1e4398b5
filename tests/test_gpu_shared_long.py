"""Attention over long shared prefixes, which is partial sums of groups and requests joined by a second launch: what short prefixes, each request by
itself in one launch, do not reach.  Every test says which kernels it means to run, so that a change of that rule shows."""
import re

import numpy as np
import pytest
import torch

from paper_2507_02620_amd import synth
from tests import cut_util
from tests.paged_util import check
from tests.test_gpu_paged_attention import _words
from tests.test_gpu_shared_attention import Shared

pytestmark = pytest.mark.gpu

#: row tiles of a workgroup over shared pages and over what follows: (requests, groups) for heads 8/2, 2048 slots and more shared
FORMS = {
    (2, 2): ([(2300, 2240, 4, 9), (2118, 2118, 0, 3), (2060, 2048, 2, 20)], [(3, 2048)]),
    (2, 1): ([(2300, 2240, 4, 3), (2118, 2118, 0, 1), (2060, 2048, 2, 4), (700, 640, 0, 2)], [(3, 2048), (1, 0)]),
    (1, 1): ([(2300, 2240, 4, 1), (2118, 2118, 0, 2), (2500, 2500, 0, 1)], [(2, 2048), (1, 64)]),
}


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


def _joined(fn, form, dtype):
    """Runs fn, which has to be the two launches in that form."""
    from tests.gpu_util import kernel_names
    names = [n for n in kernel_names(fn) if "shared" in n or "paged" in n]
    form = (1, 1) if dtype == torch.float32 else form
    assert any(re.search(r"shared_attn_kernel.*(, %d, %d>|Li%dELi%dEE)" % (form + form), n) for n in names), names  # (bf16 names come mangled)
    assert any("shared_merge_kernel" in n for n in names) and not any("shared_each" in n or "paged" in n for n in names), names


def _case(form, dtype, seed=5, **kw):
    return Shared(*FORMS[form], 8, 2, 128, dtype, seed, **kw)


DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
ALL_FORMS = pytest.mark.parametrize("form", FORMS, ids=str)


@DTYPES
@ALL_FORMS
def test_layers_strides_scale_and_given_buffers(dtype, form):
    fs = _fs()
    c = _case(form, dtype, layers=3, gap=8, n_pages=120)
    print(f"[case] long shared {dtype} {form}", flush=True)
    n = c.q.shape[0]
    wide = torch.full((n, 8 * 128 + 16), 7.0, dtype=dtype, device="cuda")
    out = wide[:, :1024].unflatten(1, (8, 128))
    q = torch.zeros((n, 8 * 128 + 32), dtype=dtype, device="cuda")[:, :1024].unflatten(1, (8, 128))
    q.copy_(c.q)
    dense = c.q
    work = fs.shared_attention_workspace(c.pool, 8, n).fill_(255)
    c.q = q
    _joined(lambda: c.run(out=out, workspace=work), form, dtype)
    for layer in range(3):
        for chain in (False, True):
            c.q = q
            out.fill_(3)
            c.run(layer, chain, out=out, workspace=work, scale=0.11)
            c.q = dense
            check(out, *c.want(layer, chain, scale=0.11), (layer, chain))
        assert float(wide[:, 1024:].float().min()) == 7 == float(wide[:, 1024:].float().max())


@DTYPES
@ALL_FORMS
def test_replayed_from_a_graph_and_on_other_streams(dtype, form):
    fs = _fs()
    c = _case(form, dtype, 21)
    items, groups, anc = fs.paged_items(c.items()), fs.prefix_groups(c.groups), _words(c.masks)
    work, out = fs.shared_attention_workspace(c.pool, 8, c.q.shape[0]), torch.empty_like(c.q)
    run = lambda o, w, **kw: fs.shared_attention(c.pool, 0, c.q, items, groups, out=o, anc=anc, workspace=w, **kw)
    _joined(lambda: run(out, work), form, dtype)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out, work)
    for i in range(4):
        c.q.mul_(0.7 + 0.2 * i)
        work.fill_(255)
        graph.replay()
        got = out.clone()
        assert torch.equal(got, run(None, None))
    check(got, *c.want(), "replayed")
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    several = [run(None, None, stream=s) for _ in range(6) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, got) for o in several)


@ALL_FORMS
def test_two_graphs_with_scratch_of_their_own(form):
    """Two graphs replayed on two streams at once: nothing of one's partial sums is in the other's."""
    fs = _fs()
    sets = []
    for j in range(2):
        c = _case(form, torch.bfloat16, 31 + j)
        items, groups, anc = fs.paged_items(c.items()), fs.prefix_groups(c.groups), _words(c.masks)
        work, out = fs.shared_attention_workspace(c.pool, 8, c.q.shape[0]), torch.empty_like(c.q)

        def run(c=c, items=items, groups=groups, anc=anc, work=work, out=out):
            for _ in range(5):                            # (long enough that the graphs meet)
                fs.shared_attention(c.pool, 0, c.q, items, groups, out=out, anc=anc, workspace=work)
        _joined(run, form, torch.bfloat16)
        check(out, *c.want(), j)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        sets.append((graph, out, out.clone(), torch.cuda.Stream(), work, run))
    for _ in range(4):
        for _, out, _, _, work, _ in sets:
            out.fill_(3)
            work.fill_(255)
        torch.cuda.synchronize()
        for graph, _, _, s, _, _ in sets:
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out, want) for _, out, want, _, _, _ in sets)


@pytest.mark.parametrize("handle", [False, True])
@ALL_FORMS
def test_results_beside_a_busy_stream(form, handle):
    """The partial sums of a call that allocates them itself are in memory of the stream it is given."""
    from tests.test_gpu_given_stream import _busy
    fs = _fs()
    c = _case(form, torch.bfloat16, 3)
    _joined(lambda: c.run(), form, torch.bfloat16)
    want = c.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy = _busy()
    old = [torch.empty_like(want) for _ in range(4)] + [fs.shared_attention_workspace(c.pool, 8, c.q.shape[0]) for _ in range(3)]
    for t in old:
        t.fill_(7)                                        # queued behind the work above
    del old, t
    got = c.run(stream=side.cuda_stream if handle else side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and float(busy[0]) == 30


def test_one_scratch_for_all_batches_of_a_program():
    """Asked for once, for the most rows, and used for fewer, which are split further; 4 KV heads: 320 rows are 12 splits, 256 are 16."""
    fs = _fs()
    for rows in (256, 320, 65, 1):
        c = Shared([(6500, 6400, 0, (rows + 1) // 2), (6464, 6464, 0, rows // 2)], [(2, 6400)], 4, 4, 64, torch.bfloat16, rows)
        work = fs.shared_attention_workspace(c.pool, 4, 320)
        print(f"[case] scratch for 320 rows, {rows} in use", flush=True)
        check(c.run(workspace=work), *c.want(), rows)
        got = fs.paged_attention(c.pool, 0, c.q, c.items(), anc=_words(c.masks), workspace=fs.paged_attention_workspace(c.pool, 4, 320))
        check(got, *c.want(), rows)


STAGES = [("f32", 4, 2, 64, 256, 688), ("bf16", 8, 2, 64, 512, 1408), ("bf16", 8, 2, 128, 512, 1408)]
#: rows of the requests, for four query heads to a KV head (f32: two)
ROWS = {(2, 2): [16, 24, 9], (2, 1): [1, 4, 3], (1, 1): [1, 2, 1]}


@pytest.mark.parametrize("cfg", STAGES, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-{c[3]}")
@pytest.mark.parametrize("form", ROWS, ids=str)
def test_the_stage(cfg, form):
    """tree_verify_shared against tree_verify_paged over the same pages: the partial sums lie in the stage's own scratch, and results go to the
    output projection in its layout.  Sums are split otherwise, so both are held to the distance that the stage has from its oracle."""
    from tests.gpu_util import TOL, Pair, max_rel_err, to_dev
    fs = _fs()
    dtype, hq, hkv, hd, d, ffn = cfg
    l_glo, rows = 2400, ROWS[form]
    print(f"[case] stage, long shared {cfg} {rows}", flush=True)
    pair = Pair(synth.StageConfig("s", dtype, 2, d, hq, hkv, hd, ffn, 0, l_glo, 40, 64, 6, 3), seed=4)
    pool = fs.PagePool(60, 2, hkv, hd, 4, 40)
    fs.page_grow(pool, [0], [l_glo])
    fs.paged_store(pool, [(0, 0, pair.kv, 0, l_glo)])
    fs.page_fork(pool, [0, 0], [1, 2])
    reqs, hid = [], []
    for i, m in enumerate(rows):
        paged = l_glo if i != 1 else 2304
        tail = torch.zeros((2, 2, hkv, 96 + 40 + max(rows), hd), dtype=pair.tdtype, device="cuda")
        tail[:, :, :, :l_glo - paged] = pair.kv[:, :, :, paged:l_glo]
        tree = synth.random_tree(m, 6, 3, 1000, 3, stream=i)
        reqs.append((i, paged, tail, l_glo, 0, m, tree.parent))
        hid.append(synth.hidden(pair.cfg, m, 5 + i, 3))
    x = to_dev(np.concatenate(hid), pair.tdtype)
    want = pair.gpu.tree_verify_paged(pool, reqs, x)
    tails = [q[2].clone() for q in reqs]
    for q in reqs:
        q[2][:, :, :, l_glo - q[1]:] = float("nan")
    _joined(lambda: pair.gpu.tree_verify_shared(pool, reqs, [(3, 2304)], x), form, pair.tdtype)
    got = pair.gpu.tree_verify_shared(pool, reqs, [(3, 2304)], x)
    assert max_rel_err(got.float().cpu().numpy(), want.float().cpu().numpy()) < TOL[dtype]
    for q, t in zip(reqs, tails):
        used = l_glo - q[1] + q[5]
        assert max_rel_err(q[2][:, :, :, :used].float().cpu().numpy(), t[:, :, :, :used].float().cpu().numpy()) < TOL[dtype]
    pool.table[1:, :36] = -1                               # the first item's row of the table counts
    assert torch.equal(pair.gpu.tree_verify_shared(pool, reqs, [(3, 2304)], x), got)
    # the same from a graph: the scratch is the stage's, and nothing of a call is left for the next
    torch.cuda.synchronize()
    items, groups, out = fs.paged_items(reqs), fs.prefix_groups([(3, 2304)]), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pair.gpu.tree_verify_shared(pool, items, groups, x, out)
    for i in range(3):
        x.mul_(1.0 - 0.1 * i)
        graph.replay()
        got = out.clone()
        assert torch.equal(got, pair.gpu.tree_verify_shared(pool, reqs, [(3, 2304)], x))


@pytest.mark.parametrize("dtype,hq,hkv,hd,d,ffn", STAGES)
def test_continuations_of_one_long_prompt(dtype, hq, hkv, hd, d, ffn):
    """Prompt to pages, forks, draft trees verified over the shared pages, accepted under cuts, the caches behind the pages pruned; twice."""
    from tests.gpu_util import TOL, Pair, max_rel_err, to_dev
    fs = _fs()
    n, l_glo, shared, vocab, T = 4, 2330, 2304, 1500, 24
    print(f"[case] continuations of a long prompt {dtype} {hq}/{hkv}x{hd}", flush=True)
    cfg = synth.StageConfig("run", dtype, 2, d, hq, hkv, hd, ffn, vocab, l_glo, T, T, 8, 3)
    pair = Pair(cfg.with_(seg_len=n * T), seed=7, head=True, max_seg=n * T)
    pool = fs.PagePool(44, 2, hkv, hd, n, 40)
    fs.page_grow(pool, [0], [l_glo])
    fs.paged_store(pool, [(0, 0, pair.kv, 0, l_glo)])
    fs.page_fork(pool, [0] * (n - 1), list(range(1, n)))
    tails = [torch.full((2, 2, hkv, 3 * T + 44, hd), float("nan"), dtype=pair.tdtype, device="cuda") for _ in range(n)]
    for tail in tails:
        tail[:, :, :, :l_glo - shared] = pair.kv[:, :, :, shared:l_glo]
    lengths, root = [l_glo] * n, [3, 5, 7, 9]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
    for step in range(2):
        trees = [synth.random_tree(T - 3 * i, 8, 3, vocab, 11 + step, stream=i) for i in range(n)]
        for i, tree in enumerate(trees):
            tree.token[0] = root[i]
        items = [(i, shared, tails[i], lengths[i], 0, tree.size, tree.parent) for i, tree in enumerate(trees)]
        hid = to_dev(np.concatenate([synth.hidden(cfg, tree.size, 50 + 10 * step + i, 7) for i, tree in enumerate(trees)]), pair.tdtype)
        before = [tail.clone() for tail in tails]
        _joined(lambda: pair.gpu.tree_verify_shared(pool, items, [(n, shared)], hid), (2, 2), pair.tdtype)
        out = pair.gpu.tree_verify_shared(pool, items, [(n, shared)], hid)
        plain = pair.gpu.tree_verify_paged(pool, [(i, shared, before[i], *it[3:]) for i, it in enumerate(items)], hid)
        assert max_rel_err(out.float().cpu().numpy(), plain.float().cpu().numpy()) < TOL[dtype]
        at = 0
        for i, tree in enumerate(trees):
            m = tree.size
            logits = pair.gpu.tree_logits(out[at:at + m])[0]
            at += m
            for c in range(1, m, 2):                       # drafts that are often right
                logits[tree.parent[c], tree.token[c]] += 4
            how = [(0.8, 50, 0.95, 0.0), (1.0, 0, 0.9, 0.02)][(i + step) % 2]
            res, retain, _ = fs.new_accept_buffers(m, 1)
            fs.tree_accept_filtered(logits, *how, dev(tree.token), dev(tree.parent), m, 5, step, res, retain)
            got, kept = fs.accept_result_to_host(res, retain, m)
            want = cut_util.accept(logits.cpu().numpy(), how, tree.token.tolist(), tree.parent.tolist(), m, 5, step)
            assert got.as_tuple() == want[0] and kept.tolist() == want[1]
            front, n_acc = lengths[i] - shared, want[0][0]
            held = tails[i][:, :, :, front:front + m].clone()
            pair.gpu.kv_compact(tails[i], front, front + m, retain, res=res, new_len=torch.zeros(2, dtype=torch.int32, device="cuda"))
            assert torch.equal(tails[i][:, :, :, front:front + n_acc], held[:, :, :, want[1][:n_acc]])
            lengths[i] += n_acc
            root[i] = want[0][1]
        print(f"  lengths now {lengths}", flush=True)


@pytest.mark.parametrize("dtype,slots", [(torch.bfloat16, 384), (torch.float32, 128)])
def test_short_prefixes_are_each_by_itself(dtype, slots):
    """The other way, in one launch that touches no scratch."""
    from tests.gpu_util import kernel_names
    fs = _fs()
    c = Shared([(slots + 20, slots, 2, 3), (slots + 9, slots + 9, 0, 2), (slots, slots, 0, 4)], [(3, slots)], 8, 2, 128, dtype, 21)
    work = fs.shared_attention_workspace(c.pool, 8, 9).fill_(255)
    names = [n for n in kernel_names(lambda: c.run(workspace=work)) if "shared" in n or "paged" in n]
    assert names and all("shared_each_kernel" in n for n in names), names
    assert int(work.min()) == 255
    check(c.run(workspace=work), *c.want(), "short")
