"""Attention of requests whose contexts begin alike against the formula in 64 bits over what the pages stand for, and the stage's forward
over it."""
import numpy as np
import pytest
import torch

from tests.paged_util import PAGE, check
from tests.test_gpu_paged_attention import Case, _words

pytestmark = pytest.mark.gpu


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


class Shared(Case):
    """A pool in which the items of a group name the same pages at the front of their rows of the table; groups: (items, shared tokens)."""

    def __init__(self, reqs, groups, *a, **kw):
        super().__init__(reqs, *a, **kw)
        at = 0
        for n, shared in groups:
            self.table[at:at + n, :shared // PAGE] = self.table[at, :shared // PAGE]
            at += n
        assert at == len(reqs)
        self.groups = groups
        self.pool.table.copy_(torch.from_numpy(self.table))

    def run(self, layer=0, chain=False, **kw):
        return self.fs.shared_attention(self.pool, layer, self.q, self.items(), self.groups, anc=None if chain else _words(self.masks), **kw)


SHAPES = [(4, 4, 64), (8, 2, 128), (7, 1, 64), (2, 2, 128), (14, 2, 128)]
#: ((l_glo, n_paged, seg_off, rows) of each request, groups)
CASES = [
    ([(64, 64, 0, 1), (64, 64, 0, 1)], [(2, 64)]),
    ([(130, 128, 0, 1), (140, 128, 0, 3), (128, 128, 2, 1)], [(3, 128)]),
    ([(64, 64, 0, 1)], [(1, 64)]),
    ([(200, 192, 0, 2), (10, 0, 0, 1), (70, 64, 0, 1)], [(1, 128), (1, 0), (1, 64)]),
    ([(300, 300, 1, 17), (290, 256, 0, 5), (256, 256, 0, 1), (70, 64, 3, 4), (65, 65, 0, 2)], [(3, 256), (2, 64)]),
    ([(1000, 960, 5, 9), (1024, 1024, 0, 16), (960, 960, 0, 0), (1100, 1088, 0, 24)], [(4, 960)]),
    ([(64, 64, 0, 0), (90, 80, 0, 2)], [(2, 64)]),                            # the group's first item has no rows of its own
    ([(2000, 1984, 0, 1)] * 16, [(16, 1984)]),
    ([(600 + 9 * i, 600 + 9 * i, i % 4, 1 + i % 5) for i in range(32)], [(32, 576)]),
    ([(600 + 9 * i, (600 + 9 * i) // 64 * 64, i % 4, 16) for i in range(12)], [(5, 512), (7, 192)]),
    ([(320, 320, 0, 100), (320, 320, 0, 130)], [(2, 320)]),
    ([(100, 64, 0, 1), (90, 0, 0, 2)], [(2, 0)]),                             # nothing shared
    ([(3000, 2944, 0, 33), (2900, 2880, 7, 30)], [(2, 2880)]),
    ([(64, 64, 0, 1), (70, 64, 0, 1), (500, 448, 0, 90)], [(2, 64), (1, 0)]),   # a request with more rows than the group has
    ([(64, 64, 0, 1), (2500, 2496, 0, 1), (900, 100, 0, 2)], [(3, 64)]),       # long behind what is shared, settled or not
    ([(130 + i, 128, 0, 1 + i % 2) for i in range(32)], [(2, 64)] * 16),
    ([(130 + i, 128, 0, 1) for i in range(32)], [(1, 64)] * 32),
    ([(4096 + i, 4096 + i, 0, 20) for i in range(4)], [(4, 4096)]),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,hd", SHAPES)
@pytest.mark.parametrize("k", range(len(CASES)))
def test_shared_attention(dtype, hq, hkv, hd, k):
    reqs, groups = CASES[k]
    print(f"[case] shared {dtype} {hq}/{hkv}x{hd} {groups} {reqs}", flush=True)
    c = Shared(reqs, groups, hq, hkv, hd, dtype, k * 100 + hq)
    check(c.run(), *c.want(), "tree")
    check(c.run(chain=True), *c.want(chain=True), "chain")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_first_items_row_of_the_table_counts(dtype):
    """What the others' rows of the table name in place of the shared pages does not matter."""
    c = Shared([(200, 192, 0, 3), (250, 192, 0, 2), (192, 192, 0, 1)], [(3, 128)], 4, 2, 128, dtype, 5)
    want = c.run()
    c.pool.table[1, :2] = -1
    c.pool.table[2, :2] = c.pool.desc.n_pages + 5
    assert torch.equal(c.run(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 12, 70])
def test_layers_strides_scale_and_given_buffers(dtype, rows):
    fs = _fs()
    c = Shared([(300, 256, 4, rows), (270, 270, 0, 3)], [(2, 256)], 4, 2, 128, dtype, 5, layers=3, gap=8, n_pages=11)
    n = c.q.shape[0]
    wide = torch.full((n, 4 * 128 + 16), 7.0, dtype=dtype, device="cuda")
    q = torch.zeros((n, 4 * 128 + 32), dtype=dtype, device="cuda")[:, :512].unflatten(1, (4, 128))
    q.copy_(c.q)
    dense, c.q = c.q, q
    work = fs.shared_attention_workspace(c.pool, 4, n).fill_(255)
    for layer in range(3):
        c.run(layer, out=wide[:, :512].unflatten(1, (4, 128)), workspace=work, scale=0.11)
        c.q = dense
        check(wide[:, :512].unflatten(1, (4, 128)), *c.want(layer, scale=0.11), layer)
        c.q = q
        assert float(wide[:, 512:].float().min()) == 7 == float(wide[:, 512:].float().max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [2, 40])
def test_rows_that_see_nothing_of_their_own(dtype, rows):
    """Rows whose mask leaves only what is shared; draft slots that are not seen hold what is not a number."""
    c = Shared([(128, 128, 0, rows), (128, 128, 3, rows)], [(2, 128)], 4, 2, 64, dtype, 9)
    for m in c.masks:
        m[:] = False
    for t in c.tails:
        t.fill_(float("nan"))
    check(c.run(), *c.want(), "shared slots alone")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 40])
def test_values_that_are_not_finite(dtype, rows):
    c = Shared([(128, 128, 0, rows), (150, 128, 0, rows), (70, 64, 0, 2), (64, 64, 0, 1)], [(2, 128), (2, 64)], 4, 2, 64, dtype, 9)
    c.pool.codes[int(c.table[0, 1]), 0, 1, 0, 70] = 127       # a value of a shared page
    c.tails[2][0, 0, 1, 3, 5] = float("inf")                 # a key that the third request sees
    check(c.run(), *c.want(), "NaN and inf")


@pytest.mark.parametrize("rows", [1, 40])
def test_a_table_entry_that_is_no_page(rows):
    c = Shared([(200, 192, 0, rows), (192, 192, 0, 2), (70, 64, 0, 2), (64, 64, 0, 1)], [(2, 128), (2, 64)], 4, 2, 64, torch.bfloat16, 9)
    want = c.run()
    c.pool.table[0, 1] = 999
    got = c.run()
    assert bool(torch.isnan(got[:rows + 2]).all()) and torch.equal(got[rows + 2:], want[rows + 2:])
    c.pool.table[0, 1] = int(c.table[0, 1])
    c.pool.table[1, 2] = -7                                   # a page of the second request's own
    got = c.run()
    assert bool(torch.isnan(got[rows:rows + 2]).all()) and torch.equal(got[:rows], want[:rows]) and torch.equal(got[rows + 2:], want[rows + 2:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 7, 40])
def test_long_shared_parts_are_read_by_the_first_items_row_and_masked(dtype, rows):
    """The same where groups are worked on together: table rows of the others, pages that are none, values that are not finite, rows without slots of their own."""
    c = Shared([(2048, 2048, 0, rows), (2048, 2048, 3, rows), (2100, 2048, 0, 2), (70, 64, 0, 2), (64, 64, 0, 1)], [(3, 2048), (2, 64)], 4, 2, 64, dtype, 9)
    for m in c.masks[:2]:
        m[:] = False
    for t in c.tails[:2]:
        t.fill_(float("nan"))
    want = c.run()
    check(want, *c.want(), "long")
    c.pool.table[1:3, :32] = -1
    assert torch.equal(c.run(), want)
    c.pool.table[0, 20] = c.pool.desc.n_pages                  # one past the last page
    got, n = c.run(), 2 * rows + 2
    assert bool(torch.isnan(got[:n]).all()) and torch.equal(got[n:], want[n:])
    c.pool.table[0, 20] = int(c.table[0, 20])
    c.pool.codes[int(c.table[0, 31]), 0, 1, 0, 70] = 127       # a value of a shared page
    c.pool.codes[int(c.table[0, 7]), 0, 0, 1, 70] = 127         # a key of another
    c.table[1:3, :32] = c.table[0, :32]
    c.pool.table.copy_(torch.from_numpy(c.table))
    check(c.run(), *c.want(), "NaN")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_replayed_from_a_graph_and_on_other_streams(dtype):
    fs = _fs()
    c = Shared([(400, 384, 2, 20), (390, 384, 0, 20), (384, 384, 0, 5)], [(3, 384)], 8, 2, 128, dtype, 21)
    items, groups, anc = fs.paged_items(c.items()), fs.prefix_groups(c.groups), _words(c.masks)
    work, out = fs.shared_attention_workspace(c.pool, 8, c.q.shape[0]), torch.empty_like(c.q)
    run = lambda o, w, **kw: fs.shared_attention(c.pool, 0, c.q, items, groups, out=o, anc=anc, workspace=w, **kw)
    run(out, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out, work)
    for i in range(4):
        c.q.mul_(0.7 + 0.2 * i)
        graph.replay()
        got = out.clone()
        assert torch.equal(got, run(None, None))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    several = [run(None, None, stream=s) for _ in range(6) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, got) for o in several)


@pytest.mark.parametrize("cfg", [("f32", 4, 2, 64, 256, 688), ("bf16", 8, 2, 64, 512, 1408), ("bf16", 4, 4, 128, 512, 1408)], ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-{c[3]}")
@pytest.mark.parametrize("rows", [[3, 5, 1], [16, 24, 9]])
def test_the_stage_over_a_shared_prefix(cfg, rows):
    """tree_verify_shared against tree_verify_paged over the same pages: the sums are split otherwise, so bf16 roundings of P and of the layers'
    activations may fall otherwise; both are held to the distance that the stage has from its oracle."""
    from paper_2507_02620_amd import synth
    from tests.gpu_util import TOL, Pair, max_rel_err, to_dev
    fs = _fs()
    dtype, hq, hkv, hd, d, ffn = cfg
    pair = Pair(synth.StageConfig("s", dtype, 2, d, hq, hkv, hd, ffn, 0, 300, 40, 64, 6, 3), seed=4)
    pool = fs.PagePool(20, 2, hkv, hd, 4, 8)
    fs.page_grow(pool, [0], [300])
    fs.paged_store(pool, [(0, 0, pair.kv, 0, 300)])
    fs.page_fork(pool, [0, 0], [1, 2])
    reqs, hid = [], []
    for i, m in enumerate(rows):
        paged = 300 if i != 1 else 256
        tail = torch.zeros((2, 2, hkv, 44 + 40 + max(rows), hd), dtype=pair.tdtype, device="cuda")
        tail[:, :, :, :300 - paged] = pair.kv[:, :, :, paged:300]
        tree = synth.random_tree(m, 6, 3, 1000, 3, stream=i)
        reqs.append((i, paged, tail, 300, 0, m, tree.parent))
        hid.append(synth.hidden(pair.cfg, m, 5 + i, 3))
    x = to_dev(np.concatenate(hid), pair.tdtype)
    want = pair.gpu.tree_verify_paged(pool, reqs, x)
    tails = [q[2].clone() for q in reqs]
    for q in reqs:
        q[2][:, :, :, 300 - q[1]:] = float("nan")
    got = pair.gpu.tree_verify_shared(pool, reqs, [(3, 256)], x)
    torch.cuda.synchronize()
    assert max_rel_err(got.float().cpu().numpy(), want.float().cpu().numpy()) < TOL[dtype]
    for q, t in zip(reqs, tails):
        used = 300 - q[1] + q[5]
        assert max_rel_err(q[2][:, :, :, :used].float().cpu().numpy(), t[:, :, :, :used].float().cpu().numpy()) < TOL[dtype]
    assert torch.equal(pair.gpu.tree_verify_shared(pool, reqs, [(3, 0)], x), pair.gpu.tree_verify_paged(pool, reqs, x))
