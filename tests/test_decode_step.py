"""DecodeCache.step's order of work, with the library's calls replaced by ones that say when they were reached.  CPU only."""
import numpy as np
import pytest
import torch

from paper_2505_24133_amd import decode, rkv


@pytest.fixture
def reached(monkeypatch):
    """The calls made, in order; none of them computes anything."""
    calls = []

    def append(shape, k, v, ring, k_new, v_new, q_new, *args, **kw):
        calls.append("append")
        return q_new.clone()

    def attend(shape, q, *args, **kw):
        calls.append("attend")
        return kw["out"] if kw.get("out") is not None else torch.empty_like(q)

    def compress(shape, *args, **kw):
        calls.append("compress")
        return (rkv.RKV_OK,) * 5

    for name, call in (("rkv_cache_append_rotary", append), ("rkv_attend", attend), ("rkv_attend_shared", attend), ("rkv_compress", compress),
                       ("rkv_compress_inplace", compress)):
        monkeypatch.setattr(rkv, name, call)
    return calls


def make(P=2, H=1, G=2, N=40, budget=30, **kw):
    return decode.DecodeCache(rkv.Shape(num_problems=P, kv_heads=H, q_heads=H * G, n_tokens=N, budget=budget), device="cpu", **kw)


def tokens(n, P=2, H=1, G=2):
    return [torch.zeros((P, n, h, 128), dtype=torch.bfloat16) for h in (H * G, H, H)]


TABLES = rkv.rotary_tables(100, device="cpu")


@pytest.mark.parametrize("error,kw", [
    (ValueError, dict(window=-1)), (ValueError, dict(window=2 ** 31)), (ValueError, dict(sinks=-1)), (ValueError, dict(sinks=2 ** 31)),
    (TypeError, dict(window=1.5)), (TypeError, dict(sinks="2")), (rkv.RkvError, dict(scale=0.0)), (rkv.RkvError, dict(scale=-0.1)),
    (rkv.RkvError, dict(scale=float("nan"))), (rkv.RkvError, dict(scale=float("inf"))), (rkv.RkvError, dict(scale=1e-60)),
    (rkv.RkvError, dict(scale=1e60)), (TypeError, dict(scale="1"))])
@pytest.mark.parametrize("share", [False, True])
def test_what_attention_refuses_is_refused_before_the_append(reached, error, kw, share):
    cache = make()
    if share:
        cache.step(*tokens(4), *TABLES)
        cache.share_prompt([2], [4])
        reached.clear()
    before = cache.length, cache.tokens_seen
    with pytest.raises(error):
        cache.step(*tokens(3), *TABLES, **kw)
    assert reached == [] and (cache.length, cache.tokens_seen) == before
    cache.step(*tokens(3), *TABLES, window=np.int64(5), sinks=2 ** 31 - 1, scale=1)
    assert reached == ["append", "attend"] and cache.length == before[0] + 3


def test_an_output_that_cannot_be_made_is_asked_for_before_the_append(reached, monkeypatch):
    """After the append nothing is allocated: out of memory leaves the caches as they were."""
    cache = make()
    cache.step(*tokens(3), *TABLES)
    reached.clear()

    def none_left(*args, **kw):
        raise torch.OutOfMemoryError("none left")

    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, none_left)
    with pytest.raises(torch.OutOfMemoryError):
        cache.step(*tokens(3), *TABLES)
    assert reached == []


def test_a_step_gives_what_attention_wrote(reached):
    out = make().step(*tokens(3), *TABLES)
    assert out.shape == (2, 3, 2, 128) and reached == ["append", "attend"]


def test_what_is_replaced_is_held_for_the_streams_that_use_it(reached, monkeypatch):
    """A larger workspace, another set of groups, a compression that ends one: what was used until then is let go for every stream of a step."""
    let_go = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: let_go.append((t.data_ptr(), stream)))
    cache = make()
    cache._streams = {0: "one", 7: "other"}

    def replaced(*tensors):
        assert let_go == [(p, s) for p in tensors for s in ("one", "other")]
        let_go.clear()

    room = {1: 1000, 3: 5000, 2: 2000, 30: 9000}
    monkeypatch.setattr(rkv, "rkv_attend_workspace_size", lambda shape, tokens, max_new, groups: room[max_new])
    cache.step(*tokens(1), *TABLES)
    replaced()
    first = cache._attend_ws.data_ptr()
    cache.step(*tokens(3), *TABLES)
    replaced(first)
    cache.step(*tokens(2), *TABLES)
    replaced()                                             # (the larger one does)
    cache.share_prompt([2], [4])
    replaced()
    lists = [t.data_ptr() for t in cache._groups]
    cache.share_prompt([1, 1], [4, 3])
    replaced(*lists)
    lists, first = [t.data_ptr() for t in cache._groups], cache._attend_ws.data_ptr()
    cache.step(*tokens(30), *TABLES)
    replaced(first)
    cache.step(*tokens(3), *TABLES)
    assert reached.count("compress") == 0
    cache.step(*tokens(1), *TABLES)
    assert reached.count("compress") == 1
    replaced(*lists)


def test_tokens_of_other_shapes_are_refused(reached):
    """Keys and values are those of the queries' tokens: as many of each problem, not only as many in all."""
    cache = make(P=2, H=1, G=2)
    q, k, v = tokens(3)
    for bad in ((q, k.view(3, 2, 1, 128), v), (q, k, v.view(3, 2, 1, 128)), (q, k[:, :2], v), (q, k, v[:1]), (q[:, :, :1], k, v), (q.view(2, 6, 1, 128), k, v),
                (q, k.flatten(0, 1), v), (q.flatten(0, 1), k, v), (q, k[..., :64], v)):
        with pytest.raises(ValueError, match="step takes"):
            cache.step(*bad, *TABLES)
    assert reached == [] and cache.length == 0


def test_what_a_captured_step_uses_is_kept(reached, monkeypatch):
    """A graph goes on using the workspace and the groups that its step was captured with: they are not given back when they are replaced."""
    capturing = [False]
    monkeypatch.setattr(decode, "_capturing", lambda device: capturing[0])
    cache = make()
    room = {1: 1000, 3: 5000, 4: 9000}
    monkeypatch.setattr(rkv, "rkv_attend_workspace_size", lambda shape, tokens, max_new, groups: room[max_new])
    cache.step(*tokens(1), *TABLES)
    cache.share_prompt([2], [1])
    cache.step(*tokens(1), *TABLES)
    first = [cache._attend_ws, *cache._groups]
    cache.step(*tokens(3), *TABLES)
    assert cache._kept == [] and cache._attend_ws is not first[0]        # no step was captured: the workspace has gone
    first[0] = cache._attend_ws
    capturing[0] = True
    cache.step(*tokens(1), *TABLES)
    capturing[0] = False
    cache.step(*tokens(4), *TABLES)
    cache.share_prompt([1, 1], [1, 1])
    assert [id(t) for t in cache._kept] == [id(t) for t in first]


def test_a_first_step_is_not_captured(reached, monkeypatch):
    """Lists that are made in a capture hold nothing before the first replay, and the steps behind it would read them."""
    capturing = [True]
    monkeypatch.setattr(decode, "_capturing", lambda device: capturing[0])
    cache = make()
    with pytest.raises(RuntimeError, match="before the capture"):
        cache.step(*tokens(2), *TABLES)
    capturing[0] = False
    cache.step(*tokens(2), *TABLES)
    capturing[0] = True
    cache.step(*tokens(2), *TABLES)
    with pytest.raises(RuntimeError, match="before the capture"):
        cache.step(*tokens(1), *TABLES)
    assert reached == ["append", "attend"] * 2 and cache.length == 4
