"""Attention over whole prompts against the formula in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests.paged_util import attend, check

pytestmark = pytest.mark.gpu


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


def _want(q, k, v, cu, scale):
    n, hq, _ = q.shape
    G = hq // k.shape[1]
    o, tol = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for a, b in zip(cu[:-1], cu[1:]):
        seen = torch.tril(torch.ones((b - a, b - a), dtype=torch.bool, device="cuda"))
        for h in range(hq):
            if b > a:
                o[a:b, h], tol[a:b, h] = attend(q[a:b, h].double(), k[a:b, h // G].double(), v[a:b, h // G].double(), seen, scale, q.dtype)
    return o, tol


def _make(n, hq, hkv, hd, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda h, s: (torch.randn((n, h, hd), device="cuda", generator=g) * s).to(dtype)
    return r(hq, std), r(hkv, std), r(hkv, 1.0)


LENS = [[1], [2, 1, 3], [15, 16, 17], [31, 32, 33], [63, 64, 65, 0, 1], [127, 128, 129], [255, 257], [500, 13], [1025],
        [513], [577, 512, 3], [640, 129, 641]]  # (the last ones: two groups of waves on alternate tiles)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 4, 64), (6, 2, 128), (7, 1, 64), (4, 4, 128)])
@pytest.mark.parametrize("lens", LENS, ids=lambda l: "-".join(map(str, l)))
def test_prompts(dtype, hq, hkv, hd, lens):
    fs = _fs()
    cu = np.cumsum([0] + lens)
    print(f"[case] prompt {dtype} {hq}/{hkv}x{hd} {lens}", flush=True)
    q, k, v = _make(int(cu[-1]), hq, hkv, hd, dtype, sum(lens) + hq)
    got = fs.prompt_attention(q, k, v, cu)
    check(got, *_want(q, k, v, cu, 1 / math.sqrt(hd)), (lens,))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale,std", [(0.3, 1.0), (1.0, 4.0), (1e-3, 1.0)])
def test_scale_and_peaked_rows(dtype, scale, std):
    fs = _fs()
    cu = [0, 190, 450]
    q, k, v = _make(450, 2, 1, 128, dtype, 5, std)
    check(fs.prompt_attention(q, k, v, cu, scale=scale), *_want(q, k, v, cu, scale), (scale, std))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_outside_the_sequences_are_left_alone(dtype):
    """Tokens before the first and behind the last sequence are neither read nor written; strides are those of cache views."""
    fs = _fs()
    cu = np.array([3, 3, 80, 85, 300])
    n, hq, hkv, hd = 310, 4, 2, 64
    q, k, v = _make(n, hq, hkv, hd, dtype, 9)
    for t in (q, k, v):
        t[:3] = float("nan")
        t[300:] = float("nan")
    kv = torch.full((1, 2, hkv, n + 7, hd + 16), float("nan"), dtype=dtype, device="cuda")  # a cache of rows with gaps
    kv[0, 0, :, :n, :hd], kv[0, 1, :, :n, :hd] = k.transpose(0, 1), v.transpose(0, 1)
    out = torch.full((hq, n, hd), 7.0, dtype=dtype, device="cuda").transpose(0, 1)
    fs.prompt_attention(q, kv[0, 0, :, :n, :hd].transpose(0, 1), kv[0, 1, :, :n, :hd].transpose(0, 1), cu, out=out)
    want, tol = _want(q, k, v, cu, 0.125)
    check(out[3:300], want[3:300], tol[3:300], "strided")
    assert bool((out[:3] == 7).all()) and bool((out[300:] == 7).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("last", [200, 600])  # one group of waves, two
@pytest.mark.parametrize("at", [0, 5, 63, 64, 150, 199])
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(dtype, bad, at, last):
    fs = _fs()
    cu = [0, last, last + 90]
    q, k, v = _make(last + 90, 2, 2, 128, dtype, 11)
    v[at, 0, 17] = bad
    k[at, 1, 3] = bad
    got = fs.prompt_attention(q, k, v, cu)
    want, tol = _want(q, k, v, cu, 1 / math.sqrt(128))
    # rows from `at` on of head 1 have an infinite or undefined score: only that the others are right is claimed
    check(got[:, 0], want[:, 0], tol[:, 0], "values")
    check(got[:at, 1], want[:at, 1], tol[:at, 1], "keys before")
    check(got[last:, 1], want[last:, 1], tol[last:, 1], "keys of the next sequence")


def test_many_sequences():
    """More sequences than one launch's arguments hold."""
    fs = _fs()
    r = np.random.default_rng(3)
    lens = r.integers(0, 9, 1000)
    cu = np.concatenate([[0], np.cumsum(lens)])
    for dtype in (torch.bfloat16, torch.float32):
        q, k, v = _make(int(cu[-1]), 2, 1, 64, dtype, 4)
        got = fs.prompt_attention(q, k, v, cu)
        seq = torch.from_numpy(np.repeat(np.arange(1000), lens)).cuda()
        at = torch.arange(int(cu[-1]), device="cuda")
        seen = (seq[:, None] == seq[None]) & (at[:, None] >= at[None])
        for h in range(2):
            o, tol = attend(q[:, h].double(), k[:, 0].double(), v[:, 0].double(), seen, 0.125, dtype)
            check(got[:, h], o, tol, "many")


def test_on_another_stream_and_captured():
    fs = _fs()
    cu = [0, 100, 333]
    q, k, v = _make(333, 4, 2, 128, torch.bfloat16, 21)
    eager = fs.prompt_attention(q, k, v, cu)
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    out = torch.zeros_like(q)
    with torch.cuda.graph(graph, stream=stream):
        fs.prompt_attention(q, k, v, cu, out=out)
    for i in range(3):
        out.fill_(i)
        if i == 2:
            q.mul_(0.5)
            eager = fs.prompt_attention(q, k, v, cu)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_far_rows_of_a_large_tensor():
    """Offsets beyond 2^31 elements: two short prompts at the far end of strided rows."""
    fs = _fs()
    n, hd = 300, 64
    big = torch.empty((n, 1 << 23), dtype=torch.bfloat16, device="cuda")  # 4.7 GiB, rows 16 MiB apart
    q, k, v = (big[:, o:o + 2 * hd].view(n, 2, hd) for o in (0, 1 << 20, 1 << 22))
    for i, t in enumerate((q, k, v)):
        t.copy_(torch.randn((n, 2, hd), device="cuda"))
    cu = [250, 260, 300]
    got = fs.prompt_attention(q, k, v, cu)
    want, tol = _want(q, k, v, cu, 0.125)
    check(got[250:], want[250:], tol[250:], "far")


@pytest.mark.parametrize("dtype,lens", [(torch.float32, [5300, 40, 5200, 1]), (torch.bfloat16, [41100, 300])])
def test_more_blocks_than_a_launch_has_levels(dtype, lens):
    """Sequences of more than 320 blocks (16 rows in f32, 128 in bf16): some rows against the formula, the last ones and the ends of blocks
    among them; every row is written."""
    fs = _fs()
    cu = np.concatenate([[0], np.cumsum(lens)])
    q, k, v = _make(int(cu[-1]), 1, 1, 64, dtype, 31)
    out = torch.full_like(q, float("nan"))
    fs.prompt_attention(q, k, v, cu, out=out)
    assert not bool(out.isnan().any())
    r = np.random.default_rng(1)
    for a, b in zip(cu[:-1], cu[1:]):
        n = int(b - a)
        rows = np.unique(np.concatenate([r.integers(0, n, 40), [0, n - 1], [x for x in (15, 16, 127, 128, 2559, 2560, 5119, 5120, 40959, 40960) if x < n]]).astype(np.int64))
        idx = torch.from_numpy(rows).cuda()
        seen = torch.arange(n, device="cuda")[None] <= idx[:, None]
        check(out[a:b, 0][idx], *attend(q[a:b, 0][idx].double(), k[a:b, 0].double(), v[a:b, 0].double(), seen, 0.125, dtype), n)
