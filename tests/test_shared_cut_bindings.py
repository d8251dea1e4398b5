"""What the bindings of sampling and of attention over a shared prefix refuse and where their own memory comes from.  CPU only: the library is a stand-in."""
import struct

import pytest
import torch

from tests.test_given_stream import _pool, _stage, rec  # noqa: F401  (the fixture)


def _logits(rows=3, vocab=40, dtype=torch.float32):
    return torch.zeros(rows, vocab, dtype=dtype)


def _u(rows=3, dtype=torch.float64):
    return torch.zeros(rows, dtype=dtype)


def _i32(n):
    return torch.zeros(n, dtype=torch.int32)


def _calls(fs, pool):
    kv, q = torch.zeros(1, 2, 2, 8, 64), torch.zeros(4, 4, 64)
    items = fs.paged_items([(0, 64, kv, 64, 0, 2), (1, 64, kv, 64, 0, 2)])
    staged = fs.paged_items([(0, 64, kv, 64, 0, 2, [-1, 0]), (1, 64, kv, 64, 0, 2, [-1, 0])])
    return {"shared": lambda s: fs.shared_attention(pool, 0, q, items, [(2, 64)], stream=s),
            "sample": lambda s: fs.sample_tokens(_logits(), _u(), stream=s)[0],
            "accept": lambda s: fs.tree_accept_filtered(_logits(), 1.0, 5, 0.9, 0.0, _i32(3), _i32(3), 3, 0, 0, _i32(6), _i32(3), stream=s),
            "stage": lambda s: _stage(fs).tree_verify_shared(pool, staged, [(2, 64)], torch.zeros(4, 256), stream=s)}


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("call,made,name", [("shared", 2, "fs_shared_attention"), ("sample", 4, "fs_sample_tokens"), ("accept", 1, "fs_tree_accept_filtered"),
                                            ("stage", 2, "fs_tree_verify_shared")])
def test_results_and_scratch(rec, call, made, name, handle):  # noqa: F811
    from paper_2507_02620_amd import flowspec as fs
    run = _calls(fs, _pool(fs))[call]
    rec.start()
    out = run(77 if handle else rec.given)
    assert rec.calls[-1] == name
    assert len([s for _, s in rec.made if s is rec.given]) == made if call != "stage" else (out.data_ptr(), rec.given) in rec.made
    if call in ("shared", "sample"):
        assert all(s is rec.given for _, s in rec.made if s is not None or call == "shared")
    if out is not None:
        assert rec.kept[out.data_ptr()] == [rec.current]              # the caller reads it there
    rec.start()
    run(None)
    assert all(s is None for _, s in rec.made) and not rec.kept


@pytest.mark.parametrize("kw", [dict(logits=_logits(dtype=torch.float16)), dict(u=_u(dtype=torch.float32)), dict(token=torch.zeros(3, dtype=torch.int64)),
                                dict(logprob=torch.zeros(3, dtype=torch.float64)), dict(kept=torch.zeros(3)), dict(temperature=torch.zeros(3, dtype=torch.float64)),
                                dict(top_k=torch.zeros(3, dtype=torch.int64)), dict(top_p=torch.zeros(3, dtype=torch.int32)), dict(min_p=torch.zeros(3, dtype=torch.bfloat16))])
def test_types_of_sampling(rec, kw):  # noqa: F811
    from paper_2507_02620_amd import flowspec as fs
    with pytest.raises(fs.FlowSpecError) as e:
        fs.sample_tokens(**dict(dict(logits=_logits(), u=_u()), **kw))
    assert e.value.code == fs.FS_EDTYPE and "fs_sample_tokens" not in rec.calls


@pytest.mark.parametrize("kw", [dict(u=_u(2)), dict(u=torch.zeros(6, dtype=torch.float64)[::2]), dict(logits=torch.zeros(40, 3).t()), dict(token=_i32(4)), dict(kept=_i32(6)[::2]),
                                dict(temperature=torch.zeros(1)), dict(top_k=_i32(4)), dict(top_p=torch.zeros(6)[::2]), dict(workspace=torch.zeros(4096)[::2]),
                                dict(top_k=2.5), dict(top_k=1 << 40), dict(top_p="x")])
def test_shapes_and_numbers_of_sampling(rec, kw):  # noqa: F811
    from paper_2507_02620_amd import flowspec as fs
    with pytest.raises((AssertionError, struct.error, OverflowError, TypeError)):
        fs.sample_tokens(**dict(dict(logits=_logits(), u=_u()), **kw))
    assert "fs_sample_tokens" not in rec.calls


def test_arguments_of_acceptance(rec):  # noqa: F811
    from paper_2507_02620_amd import flowspec as fs
    good = dict(logits=_logits(), temperature=1.0, top_k=5, top_p=0.9, min_p=0.0, token=_i32(3), parent=_i32(3), n_ver=3, seed=0, step=0, res=_i32(6), retain=_i32(3))
    for kw in (dict(logits=_logits(dtype=torch.bfloat16)), dict(token=torch.zeros(3, dtype=torch.int64)), dict(res=torch.zeros(6))):
        with pytest.raises(fs.FlowSpecError) as e:
            fs.tree_accept_filtered(**dict(good, **kw))
        assert e.value.code == fs.FS_EDTYPE
    for kw in (dict(n_ver=4), dict(logits=torch.zeros(40, 3).t()), dict(parent=_i32(2)), dict(retain=_i32(2)), dict(res=_i32(5)), dict(token=_i32(6)[::2]), dict(n_ver=1.5),
               dict(top_k=1.5), dict(top_k=1 << 40), dict(temperature="x")):
        with pytest.raises((AssertionError, TypeError, ValueError)):
            fs.tree_accept_filtered(**dict(good, **kw))
    assert "fs_tree_accept_filtered" not in rec.calls
    fs.tree_accept_filtered(**good)
    assert rec.calls[-1] == "fs_tree_accept_filtered"


def test_arguments_of_shared_attention(rec):  # noqa: F811
    from paper_2507_02620_amd import flowspec as fs
    pool, kv, q = _pool(fs), torch.zeros(1, 2, 2, 8, 64), torch.zeros(4, 4, 64)
    items = [(0, 64, kv, 64, 0, 2), (1, 64, kv, 64, 0, 2)]
    for kw in (dict(q=torch.zeros(3, 4, 64)), dict(q=torch.zeros(4, 4, 64, dtype=torch.bfloat16)), dict(q=torch.zeros(4, 4, 128)), dict(out=torch.zeros(4, 4, 128)[..., :64].transpose(0, 1)),
               dict(anc=torch.zeros(4, 16)), dict(groups=[(2, 1 << 40)]), dict(workspace=torch.zeros(512)[::2])):
        with pytest.raises((AssertionError, TypeError, OverflowError)):
            fs.shared_attention(**dict(dict(pool=pool, layer=0, q=q, items=items, groups=[(2, 64)]), **kw))
    with pytest.raises(TypeError):
        fs.prefix_groups([(2, 64.5)])
    assert "fs_shared_attention" not in rec.calls
    made = fs.prefix_groups([(1, 0), (1, 64)])
    fs.shared_attention(pool, 0, q, items, made)
    assert rec.calls[-1] == "fs_shared_attention" and made.n == 2
