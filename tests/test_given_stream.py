"""Memory that a call allocates itself comes from the stream the call is given: a block of another stream's pool may still have that
stream's work queued on it, and a fill there is not ordered against the kernels here.  CPU only: the library, the streams and the
device of the tensors are stand-ins, the order of allocations and calls is what is looked at."""
import contextlib
import types

import pytest
import torch


class _Recorder:
    """What was allocated or filled under which stream, and for which streams memory was kept."""

    def __init__(self, monkeypatch, fs):
        self.under, self.made, self.filled, self.kept, self.calls = [None], [], [], {}, []
        self.given = types.SimpleNamespace(cuda_stream=77, device_index=0)
        self.current = types.SimpleNamespace(cuda_stream=5, device_index=0)

        @contextlib.contextmanager
        def stream(s):
            self.under.append(s)
            yield
            self.under.pop()

        def watch(owner, name):
            real = getattr(owner, name)

            def made(*a, **kw):
                t = real(*a, **kw)
                self.made.append((t.data_ptr(), self.under[-1]))
                if name == "zeros":
                    self.filled.append(self.under[-1])
                return t
            monkeypatch.setattr(owner, name, made)

        real_zero = torch.Tensor.zero_

        def zero_(t):
            self.filled.append(self.under[-1])
            return real_zero(t)

        for name in ("empty", "zeros", "empty_like"):
            watch(torch, name)
        watch(torch.Tensor, "new_empty")
        monkeypatch.setattr(torch.Tensor, "zero_", zero_)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: self.kept.setdefault(t.data_ptr(), []).append(s))
        monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
        monkeypatch.setattr(torch.cuda, "stream", stream)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h, *a, **kw: self.given if h == 77 else None)
        self.default = types.SimpleNamespace(cuda_stream=0, device_index=0)
        monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: self.default)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: self.current)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
        monkeypatch.setattr(fs, "_raw_stream", lambda d: 5)
        rec = self

        class Lib:
            def __getattr__(self, name):
                def call(*a):
                    rec.calls.append(name)
                    return 512 if name.endswith("workspace_bytes") else 0
                return call
        monkeypatch.setattr(fs, "_lib", Lib())

    def start(self):
        self.made.clear()
        self.filled.clear()
        self.kept.clear()
        self.calls.clear()


@pytest.fixture
def rec(monkeypatch):
    from paper_2507_02620_amd import flowspec as fs
    return _Recorder(monkeypatch, fs)


def _pool(fs):
    return fs.PagePool(4, 1, 2, 64, 4, 2, device="cpu")


def _stage(fs):
    st = fs.Stage.__new__(fs.Stage)
    st.desc = fs.StageDesc(1, 256, 4, 2, 64, 688, 50, fs.FS_F32, 1e-5, 1e4, 64, 16, 16, 0)
    st.dtype, st.device, st._handle = torch.float32, torch.device("cpu"), None
    st.workspace = torch.empty(8)
    return st


def _page_calls(fs, pool):
    return {"grow": lambda s: fs.page_grow(pool, [0], [64], stream=s), "fork": lambda s: fs.page_fork(pool, [0], [1], stream=s),
            "compact": lambda s: fs.page_compact(pool, stream=s)}


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("call", ["grow", "fork", "compact"])
def test_status_words(rec, call, handle):
    from paper_2507_02620_amd import flowspec as fs
    run = _page_calls(fs, _pool(fs))[call]
    rec.start()
    run(77 if handle else rec.given)
    assert [n for n in rec.calls] == ["fs_page_" + call]
    assert rec.made and all(s is rec.given for _, s in rec.made)    # and not of the current stream's memory
    assert all(s is rec.given for s in rec.filled)                  # no fill that the kernel does not follow
    rec.start()
    run(None)
    assert all(s is None for _, s in rec.made)


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("call", ["page_grow", "page_fork"])
def test_an_empty_list_takes_no_pages(rec, call, own):
    """The word of an earlier call does not stand for this one's; the library itself leaves it alone."""
    from paper_2507_02620_amd import flowspec as fs
    pool, run = _pool(fs), getattr(fs, call)
    for stream in (None, rec.given, 77):
        word = None if own else torch.full((3,), -1, dtype=torch.int32)[1:2]
        rec.start()
        got = run(pool, [], [], word, stream=stream)
        assert int(got) == 0 and (own or got is word) and rec.calls == ["fs_" + call]
        assert rec.filled == [None if stream is None else rec.given]
    assert word is None or int(word._base[0]) == int(word._base[2]) == -1
    rec.start()
    run(pool, [0], [1], word)
    assert not rec.filled


def test_the_default_streams_handle(rec):
    """0 is a stream like any other; torch makes another one of it."""
    from paper_2507_02620_amd import flowspec as fs
    pool, x = _pool(fs), torch.zeros(2, 4, 64)
    for run in (lambda: fs.page_grow(pool, [0], [64], stream=0), lambda: fs.page_fork(pool, [], [], stream=0), lambda: fs.prompt_attention(x, x, x, [0, 2], stream=0)):
        rec.start()
        run()
        assert rec.made and all(s is rec.default for _, s in rec.made) and all(s is rec.default for s in rec.filled)


def _attention_calls(fs, pool):
    kv, q = torch.zeros(1, 2, 2, 8, 64), torch.zeros(2, 4, 64)
    wide = torch.zeros(2, 4, 80)[:, :, :64]                       # (not contiguous: another way to allocate)
    items = fs.paged_items([(0, 0, kv, 4, 0, 2)])
    return {"paged": lambda s: fs.paged_attention(pool, 0, q, items, stream=s), "prompt": lambda s: fs.prompt_attention(q, q, q, [0, 2], stream=s),
            "prompt of a view": lambda s: fs.prompt_attention(wide, q, q, [0, 2], stream=s)}


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("call", ["paged", "prompt", "prompt of a view"])
def test_results_and_scratch_of_attention(rec, call, handle):
    from paper_2507_02620_amd import flowspec as fs
    run = _attention_calls(fs, _pool(fs))[call]
    rec.start()
    out = run(77 if handle else rec.given)
    assert len(rec.made) == (2 if call == "paged" else 1)
    assert all(s is rec.given for _, s in rec.made)
    assert rec.kept[out.data_ptr()] == [rec.current]              # the caller reads it there
    rec.start()
    run(None)
    assert all(s is None for _, s in rec.made) and not rec.kept


def _stage_paged(fs, pool, hidden):
    items = fs.paged_items([(0, 0, torch.zeros(1, 2, 2, 8, 64), 4, 0, 2, [-1, 0])])
    return lambda s: _stage(fs).tree_verify_paged(pool, items, hidden, stream=s)


@pytest.mark.parametrize("handle", [False, True])
def test_result_of_the_stage_over_pages(rec, handle):
    from paper_2507_02620_amd import flowspec as fs
    run = _stage_paged(fs, _pool(fs), torch.zeros(2, 256))
    rec.start()
    out = run(77 if handle else rec.given)
    assert (out.data_ptr(), rec.given) in rec.made and (out.data_ptr(), None) not in rec.made
    assert rec.kept[out.data_ptr()] == [rec.current]


def _older_calls(fs):
    st, hid, par = _stage(fs), torch.zeros(2, 256), [-1, 0]
    kv = torch.zeros(1, 2, 2, 8, 64)
    tok, i32 = torch.zeros(2, dtype=torch.int32), torch.zeros(6, dtype=torch.int32)
    return {"verify": lambda s: st.tree_verify_stage(kv, 4, 4, hid, 0, par, stream=s),
            "batch": lambda s: st.tree_verify_batch([(kv, 4, 4, 0, 2, par)], hid, stream=s), "mask": lambda s: st.tree_mask(4, 0, 2, par, stream=s),
            "logits": lambda s: st.tree_logits(hid, stream=s), "sample": lambda s: fs.tree_accept_sample(hid, 1.0, tok, tok, 2, 0, 0, i32, tok, stream=s),
            "prune": lambda s: fs.seg_prune(hid, 0, [0], stream=s)}


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("call,n", [("verify", 1), ("batch", 1), ("mask", 2), ("logits", 2), ("sample", 1), ("prune", 2)])
def test_results_and_scratch_of_the_stages_calls(rec, call, n, handle):
    from paper_2507_02620_amd import flowspec as fs
    run = _older_calls(fs)[call]
    rec.start()
    run(77 if handle else rec.given)
    assert len(rec.calls) == 1 and len(rec.made) == n
    assert all(s is rec.given for _, s in rec.made) and all(s is rec.given for s in rec.filled)
    assert all(rec.kept[p] == [rec.current] for p, _ in rec.made)
    rec.start()
    run(None)
    assert all(s is None for _, s in rec.made) and not rec.kept


@pytest.mark.parametrize("handle", [False, True])
def test_the_stages_own_memory(rec, handle):
    """The weights are packed into it on the stream given."""
    from paper_2507_02620_amd import flowspec as fs
    for given in (77 if handle else rec.given, None):
        rec.start()
        st = fs.Stage(n_layers=1, d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, d_ffn=688, vocab=0, dtype=fs.FS_F32, rms_eps=1e-5, rope_theta=1e4,
                      kv_capacity=64, max_tree=16, max_seg=16, layers=[{}], device="cpu", stream=given)
        assert rec.made == [(st.workspace.data_ptr(), None if given is None else rec.given)] and rec.calls == ["fs_stage_workspace_bytes", "fs_stage_create"]
        assert rec.kept == ({} if given is None else {st.workspace.data_ptr(): [rec.current]})
        st._handle = None
