"""What the entry points over pages and prompts refuse, on the host, before any GPU work.  CPU only: pointers here are never followed."""
import ctypes as C

import numpy as np
import pytest


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


P = 1 << 20  # stands for a device pointer


def _pool(**kw):
    fs = _fs()
    f = dict(codes=P, scales=P, ref=P, table=P, length=P, work=P, n_pages=8, n_layers=2, n_kv_heads=2, head_dim=128, n_seqs=4, max_pages=3)
    f.update(kw)
    return C.byref(fs.PagePoolDesc(*(f[n] for n, _ in fs.PagePoolDesc._fields_)))


def _kv(base=P, layer=8192, kv=4096, head=2048, tok=128):
    return _fs().KVCache(base, layer, kv, head, tok)


def _i32(*v):
    a = np.array(v, dtype=np.int32)
    return a.ctypes.data_as(C.c_void_p), a


@pytest.mark.parametrize("kw", [dict(codes=None), dict(codes=P + 8), dict(scales=P + 2), dict(ref=None), dict(table=None), dict(length=None), dict(work=None),
                                dict(n_pages=0), dict(n_pages=(1 << 24) + 1), dict(n_layers=0), dict(n_kv_heads=0), dict(head_dim=96), dict(n_seqs=0),
                                dict(max_pages=0)])
def test_pools(kw):
    fs = _fs()
    L = fs.lib()
    p, (s, _), (n, _) = _pool(**kw), _i32(0), _i32(64)
    item = (fs.StoreItem * 1)(fs.StoreItem(0, 0, _kv(), 0, 64))
    assert L.fs_page_grow(p, s, n, 1, P, None) == fs.FS_EINVAL
    assert L.fs_page_fork(p, s, n, 1, P, None) == fs.FS_EINVAL
    assert L.fs_page_free(p, s, 1, None) == fs.FS_EINVAL
    assert L.fs_page_compact(p, P, None) == fs.FS_EINVAL
    assert L.fs_page_copy(p, _pool(), s, s, 1, None) == fs.FS_EINVAL and L.fs_page_copy(_pool(), p, s, s, 1, None) == fs.FS_EINVAL
    assert L.fs_paged_store(p, fs.FS_BF16, item, 1, None, None) == fs.FS_EINVAL


def test_lists_of_sequences_and_pages():
    fs = _fs()
    L, p = fs.lib(), _pool()

    def grow(seqs, toks, status=P, n=None):
        (s, _a), (t, _b) = _i32(*seqs), _i32(*toks)
        return L.fs_page_grow(p, s, t, len(seqs) if n is None else n, status, None)

    assert grow([4], [64]) == grow([-1], [64]) == grow([1, 1], [64, 64]) == grow([0], [-1]) == grow([0], [64], None) == grow([0], [1], n=-1) == fs.FS_EINVAL
    assert grow([0], [193]) == grow([0] * 257, [1] * 257) == fs.FS_ECAP
    assert grow([], []) == fs.FS_OK

    def fork(src, dst, status=P):
        (s, _a), (d, _b) = _i32(*src), _i32(*dst)
        return L.fs_page_fork(p, s, d, len(src), status, None)

    assert fork([0], [0]) == fork([0, 1], [2, 2]) == fork([0, 2], [2, 3]) == fork([9], [1]) == fork([0], [4]) == fork([0], [1], None) == fs.FS_EINVAL
    assert fork([0] * 257, list(range(257))) == fs.FS_ECAP

    def free(seqs):
        s, _a = _i32(*seqs)
        return L.fs_page_free(p, s, len(seqs), None)

    assert free([1, 1]) == free([4]) == free([-2]) == fs.FS_EINVAL and free([]) == fs.FS_OK
    assert L.fs_page_compact(p, None, None) == fs.FS_EINVAL

    def copy(src, dst, to=p, frm=p):
        (s, _a), (d, _b) = _i32(*src), _i32(*dst)
        return L.fs_page_copy(to, frm, s, d, len(src), None)

    other = _pool(codes=2 * P)
    assert copy([0], [8]) == copy([8], [0]) == copy([0], [0]) == copy([0, 1], [2, 2]) == copy([0, 1], [1, 2]) == copy([-1], [0]) == fs.FS_EINVAL
    assert copy([0, 1], [2, 2], other) == copy([0], [1], _pool(codes=2 * P, head_dim=64)) == copy([0], [1], _pool(n_layers=1)) == fs.FS_EINVAL
    assert copy([0] * 257, [1] * 257) == fs.FS_ECAP and copy([], []) == fs.FS_OK


def test_store():
    fs = _fs()
    L = fs.lib()

    def store(*items, dtype=fs.FS_BF16, n=None):
        arr = (fs.StoreItem * max(len(items), 1))(*items)
        return L.fs_paged_store(_pool(), dtype, arr, len(items) if n is None else n, None, None)

    S = fs.StoreItem
    assert store(S(0, 0, _kv(), 0, 64), dtype=2) == fs.FS_EDTYPE
    assert store() == store(S(4, 0, _kv(), 0, 64)) == store(S(-1, 0, _kv(), 0, 1)) == store(S(0, -1, _kv(), 0, 1)) == store(S(0, 0, _kv(), -1, 1)) == fs.FS_EINVAL
    assert store(S(0, 0, _kv(), 0, -1)) == store(S(0, 0, _kv(base=None), 0, 1)) == store(S(0, 0, _kv(base=P + 2), 0, 1)) == fs.FS_EINVAL
    assert store(S(0, 0, _kv(tok=64), 0, 1)) == store(S(0, 0, _kv(tok=132), 0, 1)) == store(S(0, 0, _kv(head=-8), 0, 1)) == store(S(0, 0, _kv(layer=4), 0, 1)) == fs.FS_EINVAL
    assert store(S(0, 0, _kv(), 0, 193)) == store(S(0, 3, _kv(), 0, 1)) == store(*[S(0, 0, _kv(), 0, 0)] * 33) == fs.FS_ECAP
    assert store(S(0, 0, _kv(), 0, 100), S(0, 1, _kv(), 0, 1)) == fs.FS_EINVAL  # page 1 twice
    assert store(S(0, 0, _kv(base=None), 0, 0)) == fs.FS_OK


def test_paged_attention():
    fs = _fs()
    L = fs.lib()
    need = L.fs_paged_attention_workspace_bytes(4, 2, 128, 2)
    assert need >= 2 * 16 * 130 * 4 and L.fs_paged_attention_workspace_bytes(5, 2, 128, 1) == 0 == L.fs_paged_attention_workspace_bytes(4, 2, 96, 1)

    def item(seq=0, n_paged=128, kv=None, cap=200, l_glo=150, off=0, l_s=2):
        return fs.PagedItem(seq, n_paged, kv or _kv(), cap, l_glo, off, l_s, None)

    def run(*items, pool=None, layer=0, dtype=fs.FS_BF16, hq=4, anc=None, q=P, ldq=512, out=2 * P, ldo=512, scale=0.0, ws=P, nb=need):
        arr = (fs.PagedItem * max(len(items), 1))(*items)
        return L.fs_paged_attention(pool or _pool(), layer, dtype, hq, arr, len(items), anc, q, ldq, out, ldo, scale, ws, nb, None)

    E = fs.FS_EINVAL
    assert run(item(), dtype=5) == fs.FS_EDTYPE
    assert run() == run(item(), layer=2) == run(item(), layer=-1) == run(item(), hq=3) == run(item(), hq=0) == E
    assert run(item(), scale=-1.0) == run(item(), scale=float("nan")) == run(item(), scale=float("inf")) == E
    assert run(item(seq=4)) == run(item(seq=-1)) == run(item(n_paged=151)) == run(item(n_paged=-1)) == run(item(l_s=-1)) == run(item(off=-1)) == E
    assert run(item(kv=_kv(base=None))) == run(item(kv=_kv(base=P + 8))) == run(item(kv=_kv(tok=100))) == run(item(), item(kv=_kv(head=4096))) == E
    assert run(item(), q=None) == run(item(), out=None) == run(item(), out=P) == run(item(), q=P + 8) == run(item(), anc=P + 4) == E
    assert run(item(), ldq=504) == run(item(), ldo=516) == run(item(), ldq=0) == E
    assert run(item(n_paged=256, l_glo=300)) == run(item(cap=23)) == run(item(l_glo=(1 << 31) - 9, cap=(1 << 31) - 1)) == run(item(off=1023, cap=9999)) == run(*[item()] * 33) == fs.FS_ECAP
    long = item(n_paged=0, l_glo=1000, cap=2000)
    assert run(long, ws=None) == run(long, ws=P + 16) == run(long, nb=64) == fs.FS_EWS
    assert run(item(l_s=0)) == fs.FS_OK
    assert L.fs_tree_verify_paged(None, _pool(), (fs.PagedItem * 1)(item()), 1, P, P, None) == E


def test_prompt_attention():
    fs = _fs()
    L = fs.lib()

    def rows(base=P, tok=512, head=128):
        return fs.Rows(base, tok, head)

    def run(cu=(0, 5, 9), q=None, k=None, v=None, out=None, dtype=fs.FS_BF16, hq=4, hkv=2, hd=128, scale=0.0, n=None):
        c, _a = _i32(*cu)
        r = [C.byref(x) for x in (q or rows(), k or rows(2 * P), v or rows(3 * P), out or rows(4 * P))]
        return L.fs_prompt_attention(dtype, hq, hkv, hd, c, len(cu) - 1 if n is None else n, *r, scale, None)

    E = fs.FS_EINVAL
    assert run(dtype=3) == fs.FS_EDTYPE
    assert run(cu=(0, 5, 4)) == run(cu=(-1, 5)) == run(n=-1) == run(hq=3) == run(hkv=0) == run(hd=80) == run(scale=-0.5) == run(scale=float("nan")) == E
    assert run(q=rows(None)) == run(k=rows(P + 8)) == run(v=rows(tok=516)) == run(q=rows(head=-8)) == run(q=rows(tok=1 << 25)) == E
    assert run(out=rows(4 * P, tok=64)) == run(out=rows(4 * P, head=0)) == run(out=rows(P)) == run(out=rows(2 * P)) == E
    assert run(out=rows(4 * P, tok=256, head=128)) == run(out=rows(4 * P, tok=128, head=1016)) == E    # rows that overlap
    assert run(cu=(0, 1 << 28)) == fs.FS_ECAP
    assert run(cu=(0,)) == run(cu=(3, 3, 3)) == fs.FS_OK
    assert L.fs_prompt_attention(fs.FS_F32, 1, 1, 64, None, 1, None, None, None, None, 0.0, None) == E


def test_bindings_refuse_operands_that_are_not_on_the_current_device():
    import torch
    fs = _fs()
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    pool = fs.PagePool(2, 1, 2, 64, 1, 2, device="cpu")
    with pytest.raises((fs.FlowSpecError, AssertionError, RuntimeError)):
        fs.prompt_attention(x, x, x, [0, 4])
    with pytest.raises((fs.FlowSpecError, AssertionError, RuntimeError)):
        fs.page_free(pool, [0])
    half = torch.zeros((4, 2, 64), dtype=torch.float16)
    with pytest.raises(fs.FlowSpecError) as e:
        fs.prompt_attention(half, half, half, [0, 4])
    assert e.value.code == fs.FS_EDTYPE


def test_the_largest_argument_counts_match_the_header():
    import os
    import re
    fs = _fs()
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "flowspec.h")).read()
    for name in ("FS_PAGE_TOKENS", "FS_MAX_SEQ_LIST", "FS_PAGE_WORK", "FS_MAX_BATCH"):
        assert int(re.search(r"#define\s+%s\s+(\d+)" % name, hdr).group(1)) == getattr(fs, name)
