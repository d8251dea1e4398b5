"""Attention over pages of batches with more workgroups than compute units, where the slots behind the pages have no waves of their own."""
import numpy as np
import pytest
import torch

from tests.paged_util import check
from tests.test_gpu_paged_attention import Case

pytestmark = pytest.mark.gpu

#: (l_glo, n_paged, seg_off, rows) of each request: up to 16 rows of a KV head (one row tile), 17 to 32 (two), some with fewer; contexts that end
#: with a page, in one or before the first, drafts that begin in a page's range, requests without rows between others
ONE_TILE = [(300, 256, 3, 1), (64, 64, 0, 16), (70, 70, 2, 5), (0, 0, 0, 1), (130, 100, 40, 9), (5, 0, 0, 3), (64, 64, 0, 0), (200, 192, 1, 13), (129, 128, 0, 1),
            (500, 500, 31, 2), (1, 1, 0, 1)]
TWO_TILES = [(300, 256, 3, 17), (64, 64, 0, 32), (70, 70, 2, 31), (0, 0, 0, 18), (130, 100, 40, 25), (5, 0, 0, 3), (200, 192, 1, 30), (64, 64, 0, 0), (129, 128, 0, 1),
             (500, 500, 31, 20), (1, 1, 0, 24)]


def _workgroups(reqs, hkv):
    return hkv * sum(m > 0 for _, _, _, m in reqs)


@pytest.mark.parametrize("dtype,hd", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 128)])
@pytest.mark.parametrize("reqs", [ONE_TILE, TWO_TILES], ids=["one tile", "two tiles"])
def test_as_many_heads_as_requests_fill_the_chip(dtype, hd, reqs):
    assert _workgroups(reqs, 32) > 256
    print(f"[case] batch {dtype} 32/32x{hd} {len(reqs)} requests", flush=True)
    c = Case(reqs, 32, 32, hd, dtype, hd + len(reqs[0]))
    check(c.run(), *c.want(), "tree")
    check(c.run(chain=True), *c.want(chain=True), "chain")


@pytest.mark.parametrize("hq,hkv,most,hd", [(24, 12, 8, 128), (24, 12, 16, 64), (36, 9, 8, 128)])
def test_many_requests_of_grouped_heads(hq, hkv, most, hd):
    """32 requests; rows of several query heads stacked."""
    r = np.random.default_rng(hq + most)
    reqs = []
    for i in range(32):
        l = int(r.integers(0, 400))
        reqs.append((l, int(r.integers(0, l + 1)) if i % 3 == 0 else l // 64 * 64, int(r.integers(0, 20)), most if i == 7 else int(r.integers(1, most + 1))))
    assert _workgroups(reqs, hkv) > 256 and 1 <= (hq // hkv * most + 15) // 16 <= 2
    print(f"[case] batch bf16 {hq}/{hkv}x{hd} 32 requests of up to {most} rows", flush=True)
    c = Case(reqs, hq, hkv, hd, torch.bfloat16, hq)
    first = c.run()
    check(first, *c.want(), "tree")
    check(c.run(chain=True), *c.want(chain=True), "chain")
    assert torch.equal(first, c.run())


@pytest.mark.parametrize("reqs", [ONE_TILE, TWO_TILES], ids=["one tile", "two tiles"])
def test_what_a_row_does_not_see_counts_for_nothing(reqs):
    """Slots behind the segments, draft slots that no row sees and rows that see nothing, in such a batch."""
    c = Case(reqs, 32, 32, 64, torch.bfloat16, 3)
    for t, (l, p, o, m) in zip(c.tails, c.reqs):
        t[:, :, :, l - p + o + m:] = float("nan")
    hidden = [i for i, (l, p, o, m) in enumerate(reqs) if o > 0 and m > 1]
    assert len(hidden) >= 3
    for i in hidden:
        l, p, o, m = reqs[i]
        c.masks[i][:, 0] = False
        c.tails[i][0, :, ::2, l - p] = float("inf")
        c.tails[i][0, :, 1::2, l - p] = float("nan")
    c.masks[3][0] = False                                   # (nothing before it: the row sees no slot at all)
    assert reqs[3][0] == 0
    got = c.run()
    check(got, *c.want(), "unseen")
    row = sum(m for _, _, _, m in reqs[:3])
    assert bool((got[row] == 0).all())


def test_one_token_as_heads_of_one_row():
    """[heads, 1, head_dim] transposed: dense, with a stride of its own for the single row."""
    c = Case([(200, 192, 0, 1)], 8, 2, 128, torch.bfloat16, 9)
    q, out = (torch.empty((8, 1, 128), dtype=torch.bfloat16, device="cuda").transpose(0, 1) for _ in range(2))
    q.copy_(c.q)
    assert q.stride(0) == 128 and torch.equal(q, c.q)
    c.q = q
    check(c.run(out=out), *c.want(), "transposed")
    assert torch.equal(c.fs.prompt_attention(q, q[:, :2], q[:, 2:4], [0, 1], out=torch.empty_like(out)), q[:, 2:4].repeat_interleave(4, dim=1))
