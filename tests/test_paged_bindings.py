"""What the bindings over pages and prompts refuse before the library sees an address.  CPU only: where operands stand for device memory,
their device number is a stand-in and the library only notes that it was called."""
import struct
import types

import numpy as np
import pytest
import torch

GIVEN = types.SimpleNamespace(cuda_stream=77, device_index=0)


def _fs():
    from paper_2507_02620_amd import flowspec as fs
    return fs


@pytest.fixture
def device(monkeypatch):
    """Every tensor is on device 0 but those in `away`; returns (away, calls of the library)."""
    fs = _fs()
    away, calls = {}, []

    class Lib:
        def __getattr__(self, name):
            def call(*a):
                calls.append((name, a))
                return 512 if name.endswith("workspace_bytes") else 0
            return call

    monkeypatch.setattr(fs, "_lib", Lib())
    monkeypatch.setattr(fs, "_raw_stream", lambda d: 5)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: away.get(t.data_ptr(), 0))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=5, device_index=0))
    return away, calls


REFUSED = (AssertionError, _fs().FlowSpecError)


def _pool(fs, layers=1, heads=2, hd=64):
    return fs.PagePool(4, layers, heads, hd, 4, 2, device="cpu")


def _paged(fs, dtype=torch.float32, rows=2):
    kv, q = torch.zeros(1, 2, 2, 8, 64, dtype=dtype), torch.zeros(rows, 4, 64, dtype=dtype)
    return kv, q, torch.zeros(rows, 16, dtype=torch.int64), lambda: fs.paged_items([(0, 0, kv, 4, 0, rows)])


@pytest.mark.parametrize("stream", [GIVEN, 77], ids=["stream", "handle"])
def test_operands_in_host_memory_with_a_given_stream(stream):
    fs = _fs()
    pool, word = _pool(fs), torch.zeros(1, dtype=torch.int32)
    kv, q, anc, items = _paged(fs)
    out, work = torch.empty_like(q), torch.empty(512, dtype=torch.uint8)
    for run in (lambda: fs.page_grow(pool, [0], [64], word, stream=stream), lambda: fs.page_fork(pool, [0], [1], word, stream=stream),
                lambda: fs.page_free(pool, [0], stream=stream), lambda: fs.page_compact(pool, word, stream=stream),
                lambda: fs.page_copy(pool, pool, [0], [1], stream=stream), lambda: fs.paged_store(pool, [(0, 0, kv, 0, 4)], stream=stream),
                lambda: fs.paged_attention(pool, 0, q, items(), out=out, workspace=work, stream=stream),
                lambda: fs.prompt_attention(q, q, q, [0, 2], out=out, stream=stream)):
        with pytest.raises(fs.FlowSpecError) as e:
            run()
        assert e.value.code == fs.FS_EINVAL


def test_operands_on_another_device_than_the_given_stream(device):
    fs = _fs()
    other = types.SimpleNamespace(cuda_stream=78, device_index=1)
    pool, (kv, q, anc, items) = _pool(fs), _paged(fs)
    for run in (lambda s: fs.page_free(pool, [0], stream=s), lambda s: fs.prompt_attention(q, q, q, [0, 2], out=torch.empty_like(q), stream=s)):
        run(GIVEN)
        with pytest.raises(fs.FlowSpecError) as e:
            run(other)
        assert e.value.code == fs.FS_EINVAL


@pytest.mark.parametrize("where", [-1, 1])
def test_masks_and_caches_on_another_device_than_the_pool(device, where):
    fs = _fs()
    away, calls = device
    pool, (kv, q, anc, items) = _pool(fs), _paged(fs)
    work = torch.empty(512, dtype=torch.uint8)
    fs.paged_attention(pool, 0, q, items(), anc=anc, workspace=work)
    fs.paged_store(pool, [(0, 0, kv, 0, 4)])
    for t in (anc, kv, work):
        away.clear()
        away[t.data_ptr()] = where
        calls.clear()
        with pytest.raises(REFUSED):
            fs.paged_attention(pool, 0, q, items(), anc=anc, workspace=work)
        if t is kv:
            with pytest.raises(REFUSED):
                fs.paged_store(pool, [(0, 0, kv, 0, 4)])
        assert not calls


def _stage(fs, dtype):
    st = fs.Stage.__new__(fs.Stage)
    st.desc = fs.StageDesc(1, 256, 4, 2, 64, 688, 0, fs.FS_F32 if dtype == torch.float32 else fs.FS_BF16, 1e-5, 1e4, 64, 16, 16, 0)
    st.dtype, st.device, st._handle, st.workspace = dtype, torch.device("cpu"), None, torch.empty(8)
    return st


@pytest.mark.parametrize("dtype,other", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_the_stage_over_pages_takes_caches_and_rows_of_its_own_shape(device, dtype, other):
    fs = _fs()
    away, calls = device
    st, pool, par = _stage(fs, dtype), _pool(fs), [-1, 0, 1]
    kv = lambda l=1, h=2, hd=64, t=dtype: torch.zeros(l, 2, h, 8, hd, dtype=t)
    items = lambda c: fs.paged_items([(0, 0, c, 4, 0, 3, par)])
    hid = lambda n=3, m=256, t=dtype: torch.zeros(n, m, dtype=t)
    out = st.tree_verify_paged(pool, items(kv()), hid())
    assert out.shape == (3, 256) and out.dtype is dtype
    st.tree_verify_paged(pool, [(0, 0, kv(), 4, 0, 2, par), (1, 0, kv(), 4, 1, 1, par)], hid(), hid())  # (a list as paged_items takes it)
    assert [n for n, _ in calls] == ["fs_tree_verify_paged"] * 2
    calls.clear()
    wrong = [(items(kv(t=other)), hid(), None), (items(kv(l=2)), hid(), None), (items(kv(h=1)), hid(), None), (items(kv(hd=128)), hid(), None),
             (items(kv()), hid(2), None), (items(kv()), hid(m=128), None), (items(kv()), hid(t=other), None), (items(kv()), hid(3, 512)[:, :256], None),
             (items(kv()), hid(), hid(2)), (items(kv()), hid(), hid(t=other)), (items(kv()), hid(), hid(3, 512)[:, ::2])]
    for i, (it, x, y) in enumerate(wrong):
        with pytest.raises(REFUSED):
            st.tree_verify_paged(pool, it, x, y)
        assert not calls, i
    for t in (0, 1, 2, 3):
        c, x, y = kv(), hid(), hid()
        away.clear()
        away[(c, x, y, st.workspace)[t].data_ptr()] = 1
        with pytest.raises(REFUSED):
            st.tree_verify_paged(pool, items(c), x, y)
        assert not calls, t


def test_a_pool_over_the_callers_tensors():
    """A page's codes are whole columns of 64 tokens, and all tensors are on one device."""
    fs = _fs()

    def make(width=64 * 64, at=None):
        i32 = lambda n, *shape: torch.zeros(shape, dtype=torch.int32, device="meta" if n == at else "cpu")
        return fs.PagePool.of(torch.zeros((4, 1, 2, 2, width), dtype=torch.uint8), torch.zeros((4, 1, 2, 2), device="meta" if at == 0 else "cpu"),
                              i32(1, 4), i32(2, 3, 2), i32(3, 3))

    assert make().desc.head_dim == 64
    for width in (64 * 64 + 16, 64 * 64 - 16):
        with pytest.raises(AssertionError):
            make(width)
    for at in range(4):
        with pytest.raises(AssertionError):
            make(at=at)


def test_scratch_with_gaps_or_repeats(device):
    """Its size is taken as bytes from its address on."""
    fs = _fs()
    pool, (kv, q, anc, items) = _pool(fs), _paged(fs)
    fs.paged_attention(pool, 0, q, items(), workspace=torch.empty(128))
    for work in (torch.empty(1).expand(4096), torch.empty(4096, dtype=torch.uint8)[::2]):
        with pytest.raises(REFUSED):
            fs.paged_attention(pool, 0, q, items(), workspace=work)


def test_host_lists(device):
    """Whole numbers of 32 bits, one after another, whatever holds them; none is cut to fit."""
    fs = _fs()
    away, calls = device
    pool = _pool(fs)
    for good in ([1, 3], (1, 3), np.array([1, 3]), np.array([1, 9, 3, 9], np.int32)[::2], np.array([1, 3], np.uint8), torch.tensor([1, 3]), [np.int64(1), 3]):
        calls.clear()
        fs.page_free(pool, good)
        assert calls[0][1][1] == np.array([1, 3], np.int32).tobytes() and calls[0][1][2] == 2
    long = np.arange(300)
    calls.clear()
    fs.page_copy(pool, pool, long, long.astype(np.int16))
    assert calls[0][1][2] == calls[0][1][3] == long.astype(np.int32).tobytes() and calls[0][1][4] == 300
    fs.page_free(pool, [])
    calls.clear()
    for bad in ([[0, 1], [2, 3]], np.zeros((2, 2), np.int32), np.int32(1), [1.5], np.array([1.0]), np.array([(1 << 32) + 1]), [1 << 31], np.array([1 << 31], np.uint32),
                [-(1 << 31) - 1], [1 << 70], np.array([2 ** 63], np.uint64), ["1"], [None], [True, 0.5],
                long + (1 << 32), long[None], long * 1.0, long.astype(np.uint32) - 1):
        with pytest.raises((AssertionError, TypeError, struct.error)):
            fs.page_free(pool, bad)
    x = torch.zeros(8, 2, 64)
    with pytest.raises((AssertionError, struct.error)):
        fs.prompt_attention(x, x, x, np.array([0, (1 << 32) + 8]))
    assert not calls


def test_the_stride_of_a_single_row_or_head_may_be_anything(device):
    """[heads, 1, head_dim] transposed is one dense row whose stride torch gives as head_dim; views can have any other."""
    fs = _fs()
    away, calls = device
    pool, (kv, _, anc, _) = _pool(fs), _paged(fs, rows=1)
    items = fs.paged_items([(0, 0, kv, 4, 0, 1)])
    flat, work = torch.zeros(4 * 64), torch.empty(512, dtype=torch.uint8)
    for q in (torch.zeros(4, 1, 64).transpose(0, 1), flat.as_strided((1, 4, 64), (1, 64, 1)), flat.as_strided((1, 4, 64), (0, 64, 1))):
        for out in (None, q.clone(), torch.zeros(4, 1, 64).transpose(0, 1)):
            calls.clear()
            fs.paged_attention(pool, 0, q, items, out=out, workspace=work)
            args = calls[0][1]
            assert args[8] == args[10] == 256
    kv1 = torch.zeros(5 * 64).as_strided((5, 1, 64), (64, 3, 1))
    calls.clear()
    fs.prompt_attention(torch.zeros(5, 2, 64), kv1, kv1, [0, 5])
    assert (calls[0][1][7].stride_tok, calls[0][1][7].stride_head) == (64, 64)
    q = flat.as_strided((1, 4, 64), (3, 64, 1))
    calls.clear()
    fs.prompt_attention(q, q, q, [0, 1])
    assert all((r.stride_tok, r.stride_head) == (256, 64) for r in calls[0][1][6:10])


def test_scales(device):
    fs = _fs()
    away, calls = device
    pool, (kv, q, anc, items) = _pool(fs), _paged(fs)
    for run, name in ((lambda s: fs.prompt_attention(q, q, q, [0, 2], scale=s), "fs_prompt_attention"),
                      (lambda s: fs.paged_attention(pool, 0, q, items(), scale=s, workspace=torch.empty(128)), "fs_paged_attention")):
        for good, given in ((None, 0.0), (0.125, 0.125), (2.0 ** -126, 2.0 ** -126)):
            calls.clear()
            run(good)
            assert calls[-1][0] == name and given in calls[-1][1]
        for bad in (0.0, -1.0, float("nan"), 1e-50, -1e-50):
            with pytest.raises(fs.FlowSpecError) as e:
                run(bad)
            assert e.value.code == fs.FS_EINVAL


def test_lists_in_device_memory(device, monkeypatch):
    """Reading one would wait for everything that is queued."""
    fs = _fs()
    away, calls = device
    pool, seqs = _pool(fs), torch.tensor([1])
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: t is seqs))
    with pytest.raises(TypeError):
        fs.page_free(pool, seqs)
    assert not calls
