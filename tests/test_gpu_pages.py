"""8-bit pages: quantising cache rows into them against the definition in 64 bits, and the bookkeeping of the sequences that share a
pool against the same steps on the host."""
import numpy as np
import pytest
import torch

from tests.paged_util import PAGE, HostPool, quantise, values

pytestmark = pytest.mark.gpu


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


def _state(pool):
    return pool.ref.cpu().numpy(), pool.table.cpu().numpy(), pool.length.cpu().numpy()


def _same(pool, host):
    ref, table, length = _state(pool)
    assert np.array_equal(ref, host.ref) and np.array_equal(table, host.table) and np.array_equal(length, host.length)


def _fill(pool, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    pool.codes.random_(0, 256, generator=g)
    pool.scales.uniform_(0, 1, generator=g)
    return pool.codes.clone(), pool.scales.clone()


def _moved(pool, was, moves):
    codes, scales = was[0].clone(), was[1].clone()
    for a, b in moves:
        codes[b], scales[b] = was[0][a], was[1][a]
    assert torch.equal(pool.codes, codes) and torch.equal(pool.scales, scales)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,hd,layers,lens", [(1, 64, 1, [1]), (2, 128, 2, [64]), (3, 64, 2, [65, 0, 127]), (4, 128, 1, [63, 200])])
def test_store(dtype, heads, hd, layers, lens):
    fs = _fs()
    print(f"[case] store {dtype} heads={heads} hd={hd} layers={layers} lens={lens}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(heads * 1000 + hd)
    pool = fs.PagePool(16, layers, heads, hd, len(lens) + 1, 5)
    caps = [max(n, 1) + 9 for n in lens]
    # rows of different sizes over many powers of two, an all-zero head, exact ties between codes, padded strides
    kvs = []
    for i, cap in enumerate(caps):
        big = torch.randn((layers, 2, heads, cap, hd + 8), device="cuda", generator=g)
        big *= torch.exp2(torch.randint(-20, 20, (layers, 2, heads, 1, 1), device="cuda", generator=g).float())
        big[0, 0, 0, :, :4] = torch.tensor([448.0, 17.0, 19.0, -17.0], device="cuda") * 2.0 ** (i - 3)
        if heads > 1:
            big[0, 1, 1] = 0
        kvs.append(big.to(dtype)[..., :hd])
    grown = [s + 1 for s, n in enumerate(lens) if n]
    fs.page_grow(pool, grown, [lens[s - 1] for s in grown])
    before = pool.codes.clone()
    written = torch.full((sum(-(-n // PAGE) for n in lens),), 7, dtype=torch.int32, device="cuda")
    fs.paged_store(pool, [(s + 1, 0, kv, 3, n) for s, (kv, n) in enumerate(zip(kvs, lens))], written=written)
    torch.cuda.synchronize()
    assert bool((written == 1).all())
    table, at = pool.table.cpu().numpy(), 0
    for s, n in enumerate(lens):
        for i in range(-(-n // PAGE)):
            page = int(table[s + 1, i])
            for layer in range(layers):
                got = values(pool.codes, pool.scales, page, layer, hd)
                for part in range(2):
                    for h in range(heads):
                        rows = kvs[s][layer, part, h, 3 + i * PAGE:3 + min(n, (i + 1) * PAGE)].double().cpu().numpy()
                        want, scale = quantise(rows)
                        assert float(pool.scales[page, layer, part, h]) == scale
                        assert np.array_equal(got[part][h], want * scale), (page, layer, part, h)
            at += 1
    unused = torch.from_numpy(np.setdiff1d(np.arange(16), table[table >= 0])).cuda()
    assert torch.equal(pool.codes[unused], before[unused])


def test_store_of_values_that_are_not_finite():
    fs = _fs()
    for dtype in (torch.bfloat16, torch.float32):
        pool = fs.PagePool(2, 1, 1, 64, 1, 2)
        kv = torch.randn((1, 2, 1, 64, 64), device="cuda").to(dtype)
        kv[0, 0, 0, 5, 7], kv[0, 0, 0, 6, 7], kv[0, 1, 0, 63, 63] = float("inf"), float("-inf"), float("nan")
        fs.page_grow(pool, [0], [64])
        fs.paged_store(pool, [(0, 0, kv, 0, 64)])
        k, v = values(pool.codes, pool.scales, 0, 0, 64)
        for got, part in ((k, 0), (v, 1)):
            want, scale = quantise(kv[0, part, 0].double().cpu().numpy())
            assert np.array_equal(got[0], want * scale, equal_nan=True)


def test_store_writes_only_a_sequences_own_pages():
    fs = _fs()
    pool = fs.PagePool(8, 1, 2, 64, 3, 4)
    kv = torch.randn((1, 2, 2, 256, 64), device="cuda").to(torch.bfloat16)
    fs.page_grow(pool, [0], [100])
    fs.paged_store(pool, [(0, 0, kv, 0, 100)])
    fs.page_fork(pool, [0], [1])                       # shares page 0, has a copy of page 1
    was = pool.codes.clone()
    written = torch.full((4,), 7, dtype=torch.int32, device="cuda")
    # the shared page, the own one, an entry that is no page (behind the sequence's last)
    fs.paged_store(pool, [(1, 0, kv, 100, 128), (2, 2, kv, 0, 65)], written=written)
    assert written.tolist() == [0, 1, 0, 0]
    own = int(pool.table[1, 1])
    keep = [p for p in range(8) if p != own]
    assert torch.equal(pool.codes[keep], was[keep]) and not torch.equal(pool.codes[own], was[own])


@pytest.mark.parametrize("n_pages,seed", [(1, 0), (7, 1), (100, 2), (5000, 3), (9001, 4)])
def test_bookkeeping_follows_the_host(n_pages, seed):
    """Random grows, forks, frees and compactions, failing ones among them; contents follow their pages."""
    fs = _fs()
    print(f"[case] bookkeeping pages={n_pages}", flush=True)
    r = np.random.default_rng(seed)
    n_seqs, width = 12, max(2, min(n_pages // 3, 700))
    pool, host = fs.PagePool(n_pages, 1, 1, 64, n_seqs, width), HostPool(n_pages, n_seqs, width)
    seen = set()
    for step in range(40):
        op = r.choice(["grow", "grow", "fork", "fork", "free", "compact"])
        was = _fill(pool, step)
        moves = []
        if op == "grow":
            seqs = r.permutation(n_seqs)[:r.integers(1, 5)]
            to = [int(r.integers(0 if r.random() < 0.1 else host.length[s], width * PAGE + 1)) for s in seqs]
            want, got = host.grow(seqs, to), int(fs.page_grow(pool, seqs, to))
        elif op == "fork":
            order = r.permutation(n_seqs)
            k = int(r.integers(1, 5))
            dst, src = order[:k], r.choice(order[k:], k)
            if r.random() < 0.8:
                fs.page_free(pool, dst)
                host.free(dst)
            (want, moves), got = host.fork(src, dst), int(fs.page_fork(pool, src, dst))
        elif op == "free":
            seqs = r.permutation(n_seqs)[:r.integers(1, 4)]
            fs.page_free(pool, seqs)
            host.free(seqs)
            want = got = 0
        else:
            moves = host.compact()
            want, got = len(moves), int(fs.page_compact(pool))
        assert got == want, (step, op)
        seen.add((op, min(want, 1)))
        _same(pool, host)
        _moved(pool, was, moves)
    if n_pages == 100:
        assert {("grow", -1), ("fork", -2), ("fork", 1), ("compact", 1)} <= seen


def test_fork_of_many_children_and_out_of_pages():
    fs = _fs()
    pool, host = fs.PagePool(300, 2, 3, 128, 257, 4), HostPool(300, 257, 4)
    assert int(fs.page_grow(pool, [0], [130])) == host.grow([0], [130]) == 3
    was = _fill(pool, 1)
    src, dst = [0] * 256, list(range(1, 257))
    want, moves = host.fork(src, dst)
    assert int(fs.page_fork(pool, src, dst)) == want == 256
    _same(pool, host)
    _moved(pool, was, moves)
    fs.page_free(pool, dst)
    host.free(dst)
    _same(pool, host)
    assert int(fs.page_grow(pool, [1, 2], [256, 256])) == 8
    host.grow([1, 2], [256, 256])
    before = [x.copy() for x in _state(pool)]
    assert int(fs.page_grow(pool, list(range(3, 77)), [256] * 74)) == -1  # 289 free, 296 asked for
    assert int(fs.page_grow(pool, [3, 0], [64, 129])) == -2                 # sequence 0 has 130
    assert all(np.array_equal(a, b) for a, b in zip(before, _state(pool)))


@pytest.mark.parametrize("layers,heads,hd", [(1, 1, 64), (3, 5, 128)])
def test_copy_between_pools_and_within_one(layers, heads, hd):
    fs = _fs()
    a, b = fs.PagePool(9, layers, heads, hd, 1, 1), fs.PagePool(300, layers, heads, hd, 1, 1)
    wa, wb = _fill(a, 1), _fill(b, 2)
    src, dst = [8, 0, 8, 3], [299, 7, 0, 8]
    fs.page_copy(b, a, src, dst)
    assert torch.equal(a.codes, wa[0])
    wb[0][dst], wb[1][dst] = wa[0][src], wa[1][src]
    assert torch.equal(b.codes, wb[0]) and torch.equal(b.scales, wb[1])
    fs.page_copy(a, a, [1, 1], [2, 3])
    wa[0][[2, 3]], wa[1][[2, 3]] = wa[0][[1, 1]], wa[1][[1, 1]]
    assert torch.equal(a.codes, wa[0]) and torch.equal(a.scales, wa[1])
    many = list(range(1, 257))
    fs.page_copy(b, b, [0] * 256, many)
    wb[0][many], wb[1][many] = wb[0][0].clone(), wb[1][0].clone()
    assert torch.equal(b.codes, wb[0]) and torch.equal(b.scales, wb[1])


def test_a_captured_reordering_of_children_replays():
    """Free, fork, compact in a graph on a side stream, replayed with the program's own eager work in between."""
    fs = _fs()
    pool, host = fs.PagePool(64, 1, 2, 64, 6, 6), HostPool(64, 6, 6)
    stream, status = torch.cuda.Stream(), torch.zeros(3, dtype=torch.int32, device="cuda")
    with torch.cuda.stream(stream):
        fs.page_grow(pool, [0, 1], [130, 260])
        fs.page_fork(pool, [0, 0, 1], [2, 3, 4])
    host.grow([0, 1], [130, 260])
    host.fork([0, 0, 1], [2, 3, 4])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        fs.page_free(pool, [2, 3])
        fs.page_fork(pool, [1, 1], [2, 3], status[0:1])
        fs.page_compact(pool, status[1:2])
    for step in range(4):
        was = _fill(pool, step)
        host.free([2, 3])
        n, moves = host.fork([1, 1], [2, 3])
        graph.replay()
        torch.cuda.synchronize()
        codes = was[0].clone()
        for x, y in moves:
            codes[y] = codes[x]
        moved = host.compact()
        out = codes.clone()
        for x, y in moved:
            out[y] = codes[x]
        assert status.tolist()[:2] == [n, len(moved)]
        _same(pool, host)
        assert torch.equal(pool.codes, out)
        if step == 1:  # the program's own work between the replays
            fs.page_free(pool, [4])
            host.free([4])
            fs.page_grow(pool, [5], [64])
            host.grow([5], [64])
            torch.cuda.synchronize()
