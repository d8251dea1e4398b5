"""What sampling under cuts and attention over a shared prefix refuse, on the host, before any GPU work.  CPU only: pointers here are never followed."""
import ctypes as C

import pytest

from tests.test_paged_refusals import P, _kv, _pool


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


def _sample(dtype=0, logits=P, ld=100, rows=2, vocab=100, how=None, u=P, token=P, logprob=P, kept=P, work=P, size=1 << 40, **settings):
    fs = _fs()
    f = dict(temperature=None, top_k=None, top_p=None, min_p=None, temperature_all=1.0, top_k_all=0, top_p_all=1.0, min_p_all=0.0)
    f.update(settings)
    s = fs.Sampling(*(f[n] for n, _ in fs.Sampling._fields_))
    return fs.lib().fs_sample_tokens(dtype, logits, ld, rows, vocab, None if how is False else C.byref(s), u, token, logprob, kept, work, size, None)


@pytest.mark.parametrize("kw", [dict(logits=None), dict(logits=P + 2), dict(dtype=1, logits=P + 1), dict(ld=99), dict(rows=-1), dict(vocab=0), dict(how=False),
                                dict(u=None), dict(u=P + 4), dict(token=None), dict(token=P + 2), dict(logprob=P + 1), dict(kept=P + 2), dict(temperature=P + 2),
                                dict(temperature_all=-1.0), dict(temperature_all=float("nan")), dict(temperature_all=float("inf")), dict(temperature_all=2.0 ** -101),
                                dict(temperature_all=2.0 ** 101), dict(top_p_all=float("nan")), dict(min_p_all=float("nan")), dict(top_k=P + 1)])
def test_sample_arguments(kw):
    assert _sample(**kw) == _fs().FS_EINVAL


def test_sample_limits():
    fs = _fs()
    assert _sample(dtype=2) == fs.FS_EDTYPE
    assert _sample(vocab=(1 << 20) + 1, ld=1 << 21) == _sample(rows=65536) == fs.FS_ECAP
    need = fs.lib().fs_sample_workspace_bytes(2, 100)
    assert need > 0 and _sample(size=need - 1) == _sample(work=None) == _sample(work=P + 128) == fs.FS_EWS
    assert _sample(rows=0, logits=None, u=None, token=None, work=None) == fs.FS_OK
    w = fs.lib().fs_sample_workspace_bytes
    assert w(0, 10) == w(3, 0) == w(-1, 10) == w(1, (1 << 20) + 1) == w(65536, 10) == 0 and w(1, 1 << 20) > 0
    assert w(1024, 152064) < 1 << 28                   # (a stage's tree of the largest size)


def _accept(logits=P, vocab=100, t=1.0, k=5, p=0.9, m=0.0, token=P, parent=P, T=8, n_ver=4, res=P, retain=P, work=P, size=1 << 40):
    return _fs().lib().fs_tree_accept_filtered(logits, vocab, t, k, p, m, token, parent, T, n_ver, 1, 2, res, retain, work, size, None)


@pytest.mark.parametrize("kw", [dict(logits=None), dict(logits=P + 2), dict(vocab=0), dict(t=0.0), dict(t=-1.0), dict(t=float("nan")), dict(t=2.0 ** -101), dict(t=float("inf")),
                                dict(p=float("nan")), dict(m=float("nan")), dict(token=None), dict(parent=None), dict(T=0), dict(n_ver=-1), dict(n_ver=9),
                                dict(res=None), dict(retain=None), dict(retain=P + 2)])
def test_accept_arguments(kw):
    assert _accept(**kw) == _fs().FS_EINVAL


def test_accept_limits():
    fs = _fs()
    assert _accept(T=1025) == _accept(vocab=(1 << 20) + 1) == fs.FS_ECAP
    assert _accept(work=None) == _accept(work=P + 64) == _accept(size=fs.lib().fs_sample_workspace_bytes(4, 100) - 1) == fs.FS_EWS


def _shared(groups, items=None, pool=None, layer=0, dtype=1, heads=4, q=P, ldq=512, out=2 * P, ldo=512, scale=0.0, work=P, size=1 << 40, n_groups=None, anc=None):
    fs = _fs()
    items = items or [(0, 128, 200, 8), (1, 128, 150, 8)]
    arr = (fs.PagedItem * len(items))(*[fs.PagedItem(s, p, _kv(), 200, l, 0, m, None) for s, p, l, m in items])
    g = (fs.PrefixGroup * max(len(groups), 1))(*[fs.PrefixGroup(*v) for v in groups])
    return fs.lib().fs_shared_attention(pool or _pool(), layer, dtype, heads, arr, len(items), g, len(groups) if n_groups is None else n_groups, anc, q, ldq, out, ldo,
                                        scale, work, size, None)


@pytest.mark.parametrize("groups", [[], [(2, 63)], [(2, -64)], [(2, 192)], [(1, 64)], [(3, 64)], [(0, 0), (2, 64)], [(-1, 0), (3, 0)], [(1, 64), (1, 64), (1, 64)], [(2, 1 << 30)]])
def test_groups(groups):
    assert _shared(groups) == _fs().FS_EINVAL


def test_shared_attention_arguments():
    fs = _fs()
    g = [(2, 128)]
    for kw in (dict(layer=2), dict(layer=-1), dict(heads=3), dict(q=None), dict(q=P + 8), dict(out=P), dict(out=None), dict(ldq=504), dict(ldo=516), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(anc=P + 4), dict(pool=_pool(head_dim=96)), dict(n_groups=0), dict(n_groups=5)):
        assert _shared(g, **kw) == fs.FS_EINVAL, kw
    assert _shared(g, dtype=3) == fs.FS_EDTYPE
    assert _shared([(33, 64)], items=[(0, 64, 64, 1)] * 33) == fs.FS_ECAP
    assert _shared(g, items=[(0, 128, 400, 8), (1, 128, 150, 8)]) == fs.FS_ECAP     # more slots behind the pages than the cache has
    n = fs.lib().fs_shared_attention_workspace_bytes
    assert _shared(g, work=None) == _shared(g, work=P + 64) == _shared(g, size=256) == fs.FS_EWS
    assert n(4, 2, 128, 16) >= fs.lib().fs_paged_attention_workspace_bytes(4, 2, 128, 16) > 0
    assert n(4, 3, 128, 16) == n(4, 2, 96, 16) == n(4, 2, 128, 0) == 0
    assert _shared(g, items=[(0, 128, 200, 0), (1, 128, 150, 0)]) == fs.FS_OK       # no rows


def test_the_stage_refuses_groups_without_a_stage_or_a_list():
    fs = _fs()
    g = (fs.PrefixGroup * 1)(fs.PrefixGroup(1, 0))
    it = (fs.PagedItem * 1)(fs.PagedItem(0, 0, _kv(), 200, 0, 0, 1, None))
    assert fs.lib().fs_tree_verify_shared(None, _pool(), it, 1, g, 1, P, P, None) == fs.FS_EINVAL
    assert fs.lib().fs_tree_verify_shared(C.c_void_p(P), _pool(), it, 1, g, 0, P, P, None) == fs.FS_EINVAL
    assert C.sizeof(fs.PrefixGroup) == 8 and C.sizeof(fs.Sampling) == 48
