"""How the calls around the cache are made: the native host path and the plain one give the same bytes and refuse the same calls."""
import sys

import pytest
import torch

import paper_2505_24133_amd
from attend_reference import Batch, attend64, check, int32
from paper_2505_24133_amd import rkv

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "plain"])
def path(request, monkeypatch):
    print(f"[gpu-case] {request.node.name}", flush=True)
    if request.param == "plain":
        monkeypatch.setitem(sys.modules, "paper_2505_24133_amd._host", None)
        monkeypatch.delattr(paper_2505_24133_amd, "_host", raising=False)
        for name in ("_lib", "_append", "_append_rotary", "_attend_native"):
            monkeypatch.setattr(rkv, name, None)
    return request.param


def test_workspaces_that_do_not_do(path):
    b = Batch(2, 4, [1], [3000], seed=1)
    need = rkv.rkv_attend_workspace_size(b.shape, 1, 1)
    room = torch.empty(need + 1024, dtype=torch.uint8, device="cuda")
    assert need > 0

    def call(ws):
        return rkv.rkv_attend(b.shape, b.q, b.k, b.v, b.starts, b.kv_len, max_new=1, ws=ws, want_lse=True)

    for small in (room[:need - 1], room[1:need + 1], room[1:101], room[:0]):
        with pytest.raises(rkv.RkvError, match="status -4"):
            call(small)
    # neither bytes nor in a row: its size says nothing about what may be written
    for other in (room[:1].expand(need + 1024), room.repeat(2)[::2], torch.empty(need, dtype=torch.float32, device="cuda")):
        with pytest.raises(ValueError, match="ws must be"):
            call(other)
    check(call(room), attend64(b))
    check(call(room[1:]), attend64(b))


def rotary_call(b, interleaved, q_out=None):
    gen = torch.Generator(device="cuda").manual_seed(5)
    wide = torch.randn((b.T, b.H * (b.G + 2), 128), generator=gen, device="cuda").bfloat16()
    q, k, v = wide[:, :b.H * b.G], wide[:, b.H * b.G:b.H * (b.G + 1)], wide[:, b.H * (b.G + 1):]
    cos, sin = rkv.rotary_tables(500, 64)
    ring = torch.zeros((b.P, b.H * b.G, b.shape.alpha, 128), dtype=torch.bfloat16, device="cuda")
    held = b.kv_len - (b.starts[1:] - b.starts[:-1])
    keys, values = b.k.clone(), b.v.clone()
    got = rkv.rkv_cache_append_rotary(b.shape, keys, values, ring, k, v, q, cos, sin, b.starts, held, held + 3, interleaved=interleaved, q_out=q_out)
    return got, ring, keys, values


@pytest.mark.parametrize("how", [dict(), dict(strided=True), dict(page=32)])
def test_both_paths_give_the_same_bytes(how, monkeypatch):
    print(f"[gpu-case] both paths {how}", flush=True)
    rkv.load_library()
    b = Batch(2, 3, [1, 0, 4], [200, 70, 90], seed=2, **how)
    first, lens = int32([1, 3]), int32([32])
    ws = rkv.make_attend_workspace(b.shape, b.T, 4, groups=1)
    b.rows_k[2, :, :32], b.rows_v[2, :, :32] = b.rows_k[1, :, :32], b.rows_v[1, :, :32]
    b.store()

    def everything():
        got = [*rotary_call(b, False), *rotary_call(b, True, torch.empty((b.T, 6, 128), dtype=torch.bfloat16, device="cuda"))]
        for kw in (dict(), dict(window=20, sinks=3), dict(scale=0.2), dict(out=torch.empty((b.T, 9, 128), dtype=torch.bfloat16, device="cuda")[:, 2:8])):
            lists = b.shape, b.q, b.k, b.v, b.starts, b.kv_len
            got += [*rkv.rkv_attend(*lists, max_new=4, want_lse=True, ws=ws, **kw), *rkv.rkv_attend_shared(*lists, first, lens, max_new=4, want_lse=True, ws=ws, **kw)]
            got.append(rkv.rkv_attend(*lists, ws=rkv.make_attend_workspace(b.shape, b.T), **kw))
            kw.pop("out", None)
            got.append(rkv.rkv_attend(*lists, **kw))
        return [t.clone() for t in got]

    native = everything()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        aside = everything()
    other.synchronize()
    monkeypatch.setattr(rkv, "_append_rotary", lambda *args: None)
    monkeypatch.setattr(rkv, "_attend_native", lambda *args: None)
    for got in (aside, everything()):
        assert len(got) == len(native)
        for i, (x, y) in enumerate(zip(native, got)):
            assert torch.equal(x, y), i


def test_what_the_binding_refuses(path):
    b = Batch(2, 3, [1, 2], [50, 60], seed=3)
    half = b.q.half()
    lists = [b.shape, b.q, b.k, b.v, b.starts, b.kv_len]

    def refused(error, i=None, value=None, match=None, **kw):
        args = list(lists)
        if i is not None:
            args[i] = value
        with pytest.raises(error, match=match):
            rkv.rkv_attend(*args, **kw)

    refused(RuntimeError, 1, b.q.cpu())
    refused(ValueError, 1, half, "q must be")
    refused(ValueError, 1, b.q[:, :5], "q must be")
    refused(ValueError, 1, b.q.transpose(1, 2).contiguous().transpose(1, 2), "q must be")
    refused(ValueError, 2, b.k[:1])
    refused(ValueError, 4, b.starts[:2], "starts must be")
    refused(ValueError, 4, b.starts.long(), "starts must be")
    refused(ValueError, 5, torch.zeros((2, 2), dtype=torch.int32, device="cuda")[:, 0], "kv_len must be")
    refused(ValueError, window=-1, match="window, sinks")
    refused(ValueError, sinks=2 ** 31, match="window, sinks")
    refused(ValueError, out=b.q[:2], match="out must be")
    refused(ValueError, lse=torch.empty((3, 5), device="cuda"), match="lse must be")
    refused(rkv.RkvError, max_new=4, match="status -2")
    refused(rkv.RkvError, max_new=0, match="status -2")
    for scale in (0.0, float("inf"), -1.0):
        refused(rkv.RkvError, scale=scale)
    # rows of the outputs that lie in each other
    room = torch.zeros(3 * 6 * 128, dtype=torch.bfloat16, device="cuda")
    for strides in ((6 * 128, 64, 1), (64, 128 * 3, 1)):
        refused(rkv.RkvError, out=room.as_strided((3, 6, 128), strides), match="status -2")
    with pytest.raises(ValueError, match="group_starts must be"):
        rkv.rkv_attend_shared(*lists, int32([0, 1]), int32([1, 2]))
    check(rkv.rkv_attend(*lists, want_lse=True), attend64(b))


@pytest.mark.parametrize("T,H,G", [(5, 1, 1), (5, 2, 3), (1, 2, 3), (1, 1, 6)])
def test_broadcast_token_arrays_are_refused(path, T, H, G):
    """Arrays whose rows are fewer than their places: refused on the host by both paths, whichever array it is."""
    b = Batch(H, G, [T], [40], seed=6)
    one = torch.zeros((1, 1, 128), dtype=torch.bfloat16, device="cuda")
    cos, sin = rkv.rotary_tables(50)
    new = {"k_new": one.repeat(T, H, 1), "v_new": one.repeat(T, H, 1), "q_new": one.repeat(T, H * G, 1), "q_out": one.repeat(T, H * G, 1)}
    before = b.k.clone(), b.v.clone()
    for name, t in new.items():
        if t.shape[0] == t.shape[1] == 1:
            continue
        bad = {**new, name: one.expand(t.shape)}
        with pytest.raises(ValueError, match="broadcast dimension"):
            rkv.rkv_cache_append_rotary(b.shape, b.k, b.v, None, bad["k_new"], bad["v_new"], bad["q_new"], cos, sin, b.starts, int32([3]), int32([3]), q_out=bad["q_out"])
    assert torch.equal(b.k, before[0]) and torch.equal(b.v, before[1])
    if T * H * G > 1:
        room = rkv.make_attend_workspace(b.shape, T)
        for kw in (dict(), dict(ws=room)):
            with pytest.raises(ValueError, match="broadcast dimension"):
                rkv.rkv_attend(b.shape, one.expand(b.q.shape), b.k, b.v, b.starts, b.kv_len, **kw)
            with pytest.raises(ValueError, match="broadcast dimension"):
                rkv.rkv_attend(b.shape, b.q, b.k, b.v, b.starts, b.kv_len, out=one.expand(b.q.shape), **kw)


def test_one_token_or_one_head_in_wider_rows(path):
    """Token arrays with one token or one head, not dense: read and written where they lie."""
    for new, H, G in (([1], 2, 3), ([6], 1, 1)):
        b = Batch(H, G, new, [300], seed=7)
        wide = torch.full((b.T, H * G, 256), 7.0, dtype=torch.bfloat16, device="cuda")
        wide[..., :128] = b.q
        room = torch.full_like(wide, 9.0)
        lse = torch.empty(b.q.shape[:2], device="cuda")
        out, _ = rkv.rkv_attend(b.shape, wide[..., :128], b.k, b.v, b.starts, b.kv_len, max_new=new[0], out=room[..., :128], lse=lse,
                                ws=rkv.make_attend_workspace(b.shape, b.T, new[0]))
        check((out, lse), attend64(b))
        assert (room[..., 128:] == 9).all()


@pytest.mark.parametrize("which", [0, 1, 2])
def test_one_row_as_a_whole_cache_is_refused(path, which):
    """A cache (of keys, values, queries) that is one row broadcast to all places: refused on the host by both paths, in every call that takes one."""
    b = Batch(2, 3, [1, 1], [40, 30], seed=8)
    caches = [b.k, b.v, torch.zeros((2, 6, b.shape.alpha, 128), dtype=torch.bfloat16, device="cuda")]
    caches[which] = torch.zeros(128, dtype=torch.bfloat16, device="cuda").expand(caches[which].shape)
    cos, sin = rkv.rotary_tables(50)
    kv = torch.ones((2, 2, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="one row broadcast"):
        rkv.rkv_cache_append(b.shape, *caches, kv, kv, b.q, 3, 3)
    with pytest.raises(ValueError, match="one row broadcast"):
        rkv.rkv_cache_append_rotary(b.shape, *caches, kv, kv, b.q, cos, sin, b.starts, int32([3, 3]), int32([3, 3]))
    if which < 2:
        with pytest.raises(ValueError, match="one row broadcast"):
            rkv.rkv_attend(b.shape, b.q, caches[0], caches[1], b.starts, b.kv_len, ws=rkv.make_attend_workspace(b.shape, b.T))
