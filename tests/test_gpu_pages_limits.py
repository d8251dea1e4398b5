"""Page calls at the ends of their ranges."""
import math

import numpy as np
import pytest
import torch

from tests.paged_util import quantise, values

pytestmark = pytest.mark.gpu


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


def test_growing_by_more_pages_than_32_bits_count():
    """128 and 256 sequences of 2^24 pages each: too few are free, whatever their sum wraps to, and nothing changes."""
    fs = _fs()
    n, width = 256, 1 << 24
    whole = fs.PagePool(300, 1, 1, 64, n, 2)
    table = torch.empty((n, width), dtype=torch.int32, device="cuda")  # (16 GiB; a call touches what it appends)
    table[:, :4] = -1
    pool = fs.PagePool.of(whole.codes, whole.scales, whole.ref, table, whole.length)
    most = width * 64
    assert int(fs.page_grow(pool, [0, 1], [130, 64])) == 4
    for seqs in (range(n), range(128), range(100, 229), [5], [0, 9]):
        assert int(fs.page_grow(pool, list(seqs), [most] * len(seqs))) == -1
        assert pool.length.tolist() == [130, 64] + [0] * 254 and int(pool.ref.sum()) == 4 and int((pool.ref != 0).sum()) == 4
    assert int(fs.page_grow(pool, [0, 1, 2], [most, 63, most])) == -2
    assert pool.length[:3].tolist() == [130, 64, 0] and bool((table[2:, :4] == -1).all())
    assert int(fs.page_grow(pool, list(range(2, 256)), [64] * 254)) == 254 and table[2:, 0].tolist() == list(range(4, 258))
    # as many as there are, and one more
    assert int(fs.page_grow(pool, [255], [64 * 44])) == -1
    assert int(fs.page_grow(pool, [255], [64 * 43])) == 42 and int((pool.ref == 0).sum()) == 0
    assert int(fs.page_grow(pool, [0], [192])) == 0


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_finite_values_stay_finite_in_a_page(dtype, hd):
    """At the scale 2^120 a value from 248 * 2^120 on lies nearest to 2^128, which no 32-bit number is; 240 * 2^120 is within half a step, 2^-4 of
    the value, as well.  Smaller values of the tile, infinities and tiles without such values are as ever."""
    fs = _fs()
    pool = fs.PagePool(2, 1, 2, hd, 1, 2)
    g = torch.Generator(device="cuda")
    g.manual_seed(hd)
    kv = (torch.randn((1, 2, 2, 70, hd), device="cuda", generator=g) * 2.0 ** 125).to(dtype)
    kv = torch.where(kv.abs() < 2.0 ** 127, kv, torch.ones_like(kv))
    unit = 2.0 ** 120
    edge = [240.0, 247.0, 248.0, -248.0, 255.0, -255.0, 232.0, 1.0, 2.0 ** -9]
    if dtype == torch.float32:
        edge += [248.0 - 2.0 ** -16, 256.0 - 2.0 ** -16, -256.0 + 2.0 ** -16]
    for part in range(2):
        kv[0, part, 0, 5, :len(edge)] = torch.tensor([e * unit for e in edge], dtype=torch.float64).to(dtype).cuda()
        kv[0, part, 0, 6, :3] = torch.tensor([math.inf, -math.inf, math.nan], dtype=dtype)
        kv[0, part, 1, 69, 3] = 247 * unit                 # the second page of head 1: the scale is 2^120, nothing rounds to 2^128
        kv[0, part, 0, 64:] = 447 * 2.0 ** 119             # the second page of head 0: just under the largest scale
    fs.page_grow(pool, [0], [70])
    fs.paged_store(pool, [(0, 0, kv, 0, 70)])
    cut = kv.double()
    cut = torch.where(torch.isfinite(cut), cut.clamp(-240 * unit, 240 * unit), cut).cpu().numpy()
    for page in range(2):
        got = values(pool.codes, pool.scales, int(pool.table[0, page]), 0, hd)
        for part in range(2):
            for h in range(2):
                rows = kv[0, part, h, 64 * page:min(70, 64 * page + 64)].double().cpu().numpy()
                top = np.abs(rows[np.isfinite(rows)]).max()
                want, scale = quantise(cut[0, part, h, 64 * page:64 * page + 64] if top >= 248 * unit else rows)
                assert np.array_equal(got[part][h], want * scale, equal_nan=True), (page, part, h)
                fine = np.isfinite(rows)
                mine = got[part][h][:rows.shape[0]]
                assert np.isfinite(mine[fine]).all() and (np.abs(mine[fine]) < 2.0 ** 128).all() and np.isnan(mine[~fine]).all()
                assert (np.abs(mine[fine] - rows[fine]) <= np.maximum(2.0 ** -4 * np.abs(rows[fine]), scale * 2.0 ** -10)).all()
