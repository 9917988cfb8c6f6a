"""The decode loop with everything in it: prompts and single tokens rotated, appended, attended and compressed by DecodeCache.step, against
a cache that is kept row by row on the side and attended in float64."""
import pytest
import torch

from attend_reference import Batch, attend64, int32, turned64
from paper_2505_24133_amd import decode, rkv

pytestmark = pytest.mark.gpu


def loop(shape, prompt, steps, inplace=False, window=0, sinks=0, interleaved=False, share=None, rotary=128):
    P, H, Hq, N, d = shape.num_problems, shape.kv_heads, shape.q_heads, shape.n_tokens, shape.head_dim
    cache = decode.DecodeCache(shape, inplace=inplace)
    cos, sin = rkv.rotary_tables(prompt + steps, rotary, 500000.0)
    side = Batch(H, Hq // H, [1] * P, [1] * P, N=N, seed=prompt)            # rows, queries and lengths of the reference
    gen, held, seen, compressions = side.gen, 0, 0, 0
    todo = [prompt] + [1] * steps if prompt else [1] * steps
    for n in todo:
        q, k, v = (torch.randn((P, n, x, d), generator=gen, device="cuda").bfloat16() for x in (Hq, H, H))
        if share and seen == 0:
            q, k, v = (t.view(-1, share, *t.shape[1:])[:, :1].expand(-1, share, -1, -1, -1).reshape(t.shape) for t in (q, k, v))
        # what the rotation gives, by a call of its own into rows of its own, and within its bounds
        flat = [t.flatten(0, 1).contiguous() for t in (q, k, v)]
        rows = torch.zeros((2, P, H, N, d), dtype=torch.bfloat16, device="cuda")
        q_turned = rkv.rkv_cache_append_rotary(shape, rows[0], rows[1], None, flat[1], flat[2], flat[0], cos, sin,
                                               int32([i * n for i in range(P + 1)]), int32([held] * P), int32([seen] * P), interleaved=interleaved)
        c, s = (t[seen:seen + n].repeat(P, 1) for t in (cos, sin))
        new_rows = slice(held, held + n)
        for got, x in ((q_turned, flat[0]), (rows[0][:, :, new_rows].transpose(1, 2).flatten(0, 1), flat[1])):
            want, err = turned64(x, c, s, interleaved)
            assert bool(((got.double() - want).abs() <= err).all())
        side.rows_k[:, :, new_rows], side.rows_v[:, :, new_rows] = rows[0][:, :, new_rows], v.transpose(1, 2)
        held, seen = held + n, seen + n
        side.q, side.new, side.lens, side.T = q_turned, [n] * P, [held] * P, P * n
        full = held >= N
        out = cache.step(q, k, v, cos, sin, interleaved=interleaved, window=window, sinks=sinks)
        assert out.shape == (P, n, Hq, d) and cache.tokens_seen == seen
        ref, _, e_out, _ = attend64(side, window, sinks)
        assert bool(((out.flatten(0, 1).double() - ref).abs() <= e_out).all())
        for j in range(max(0, n - shape.alpha), n):
            assert torch.equal(cache.q_cache[:, :, (seen - n + j) % shape.alpha], q_turned.view(P, n, Hq, d)[:, j])
        if full:
            compressions += 1
            kept = cache.kept_idx.long()[..., None].expand(-1, -1, -1, d)
            held = shape.budget
            side.rows_k[:, :, :held], side.rows_v[:, :, :held] = side.rows_k.gather(2, kept), side.rows_v.gather(2, kept)
        assert cache.length == held and cache.compressions == compressions
        assert torch.equal(cache.k[:, :, :held], side.rows_k[:, :, :held]) and torch.equal(cache.v[:, :, :held], side.rows_v[:, :, :held])
        if share and seen == prompt:
            cache.share_prompt([share] * (P // share), [prompt] * (P // share))


def shape(P, H, G, N, budget):
    return rkv.Shape(num_problems=P, kv_heads=H, q_heads=H * G, n_tokens=N, budget=budget)


@pytest.mark.parametrize("how", [
    pytest.param(dict(shape=shape(2, 2, 4, 48, 32), prompt=20, steps=70), id="a prompt, then three compressions"),
    pytest.param(dict(shape=shape(1, 3, 5, 96, 64), prompt=96, steps=40, inplace=True, interleaved=True), id="a prompt that fills the cache, in place"),
    pytest.param(dict(shape=shape(3, 1, 2, 40, 30), prompt=0, steps=60, window=17, sinks=2, rotary=64), id="tokens only, a window"),
    pytest.param(dict(shape=shape(6, 2, 4, 300, 256), prompt=200, steps=120, share=3), id="samples of two prompts"),
])
def test_loop(how):
    loop(**how)


def test_refusals():
    s = shape(1, 1, 2, 40, 30)
    cache = decode.DecodeCache(s)
    cos, sin = rkv.rotary_tables(20)
    q, k = torch.zeros((1, 41, 2, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 41, 1, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="room for 40"):
        cache.step(q, k, k, cos, sin)
    with pytest.raises(ValueError, match="end at position 20"):
        cache.step(q[:, :21], k[:, :21], k[:, :21], cos, sin)
    cache.step(q[:, :20], k[:, :20], k[:, :20], cos, sin)
    for sizes, rows in (([2], [5]), ([1], [21]), ([1], [5, 6]), ([-1], [3])):
        with pytest.raises(ValueError, match="share_prompt"):
            cache.share_prompt(sizes, rows)


def test_a_refused_step_has_not_taken_place():
    s = shape(2, 1, 2, 40, 30)
    cos, sin = rkv.rotary_tables(200)
    gen = torch.Generator(device="cuda").manual_seed(1)
    tokens = [tuple(torch.randn((2, n, h, 128), generator=gen, device="cuda").bfloat16() for h in (2, 1, 1)) for n in (9, 1, 3)]
    straight, stumbling = decode.DecodeCache(s), decode.DecodeCache(s)
    for t in tokens:
        want = straight.step(*t, cos, sin)
        for error, kw in ((ValueError, dict(window=-1)), (rkv.RkvError, dict(scale=0.0))):
            held = stumbling.length, stumbling.tokens_seen
            with pytest.raises(error):
                stumbling.step(*t, cos, sin, **kw)
            assert (stumbling.length, stumbling.tokens_seen) == held
        assert torch.equal(stumbling.step(*t, cos, sin), want)
    assert torch.equal(stumbling.k, straight.k) and torch.equal(stumbling.v, straight.v) and torch.equal(stumbling.q_cache, straight.q_cache)
    with pytest.raises(ValueError, match="share_prompt"):
        straight.share_prompt([0, 0, 0], [1, 1, 1])


def test_one_workspace_for_all_lengths():
    s = shape(1, 1, 4, 4000, 3000)
    cache = decode.DecodeCache(s)
    cos, sin = rkv.rotary_tables(4000)
    at_most = max(rkv.rkv_attend_workspace_size(s, n, n) for n in range(1, 60)) + 256
    for n in (3, 50, 1, 40, 2, 33):
        t = [torch.zeros((1, n, h, 128), dtype=torch.bfloat16, device="cuda") for h in (4, 1, 1)]
        cache.step(*t, cos, sin)
        assert cache._attend_ws.numel() <= at_most


@pytest.mark.parametrize("inplace", [False, True])
def test_a_refused_step_leaves_the_query_cache(inplace):
    """The tokens of a refused step are never seen again: the next step is another one, shorter, and a compression takes the queries of
    the tokens that were accepted."""
    print(f"[gpu-case] refused step inplace={inplace}", flush=True)
    s = shape(2, 1, 2, 40, 30)
    cos, sin = rkv.rotary_tables(200)
    gen = torch.Generator(device="cuda").manual_seed(2)

    def tokens(n):
        return tuple(torch.randn((2, n, h, 128), generator=gen, device="cuda").bfloat16() for h in (2, 1, 1))

    taken, refused = [tokens(n) for n in (33, 1, 3, 2, 1)], tokens(5)
    straight, stumbling = decode.DecodeCache(s, inplace=inplace), decode.DecodeCache(s, inplace=inplace)
    for t in taken:
        for error, kw in ((ValueError, dict(window=-1)), (ValueError, dict(sinks=2 ** 31)), (rkv.RkvError, dict(scale=0.0)), (TypeError, dict(window=1.5))):
            before = stumbling.q_cache.clone(), stumbling.k.clone(), stumbling.v.clone(), stumbling.length, stumbling.tokens_seen
            n = min(5, s.n_tokens - stumbling.length)
            with pytest.raises(error):
                stumbling.step(*(x[:, :n] for x in refused), cos, sin, **kw)
            assert torch.equal(stumbling.q_cache, before[0]) and torch.equal(stumbling.k, before[1]) and torch.equal(stumbling.v, before[2])
            assert (stumbling.length, stumbling.tokens_seen) == before[3:]
        assert torch.equal(stumbling.step(*t, cos, sin), straight.step(*t, cos, sin))
    assert straight.compressions == stumbling.compressions == 1 and torch.equal(stumbling.kept_idx, straight.kept_idx)
    assert torch.equal(stumbling.q_cache, straight.q_cache) and torch.equal(stumbling.k[:, :, :30], straight.k[:, :, :30])


def test_a_replaced_workspace_is_not_given_out_under_a_step():
    """A step on another stream than the one that the workspace was allocated on, then a longer one: the smaller workspace, and a replaced
    list of groups, stay as they are as long as the other stream has work that reads them."""
    print("[gpu-case] replaced workspace", flush=True)
    s = shape(1, 1, 4, 4000, 3000)
    cache = decode.DecodeCache(s)
    cos, sin = rkv.rotary_tables(4000)
    t = {n: [torch.zeros((1, n, h, 128), dtype=torch.bfloat16, device="cuda") for h in (4, 1, 1)] for n in (1, 60)}
    assert rkv.rkv_attend_workspace_size(s, 60, 60, 1) > rkv.rkv_attend_workspace_size(s, 1, 1, 1)
    decode.DecodeCache(s).step(*t[60], cos, sin)           # (its kernels are loaded now)
    cache.step(*t[1], cos, sin)
    cache.share_prompt([1], [1])
    cache.step(*t[1], cos, sin)
    held = [x for x in (cache._attend_ws, *cache._groups)]
    ptrs, sizes = [x.data_ptr() for x in held], [x.numel() * x.element_size() for x in held]
    del held
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        torch.cuda._sleep(200_000_000)                     # (a time that ends by itself)
        cache.step(*t[1], cos, sin)
        done = torch.cuda.Event()
        done.record()
    # a new list and a larger workspace, with the step on the other stream still to come
    cache.share_prompt([1], [2])
    with torch.cuda.stream(other):
        cache.step(*t[60], cos, sin)
    given = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(20)]
    if done.query():
        pytest.skip("the other stream was through before the memory was asked for")
    assert not {x.data_ptr() for x in given} & set(ptrs)
    torch.cuda.synchronize()


def test_a_captured_step_and_longer_ones_behind_it():
    """A captured step keeps its workspace: replays between and behind longer steps give what they gave, and write over nobody's memory."""
    print("[gpu-case] captured step", flush=True)
    s = shape(2, 2, 4, 3000, 2000)
    cache, same = decode.DecodeCache(s), decode.DecodeCache(s)
    cos, sin = rkv.rotary_tables(3000)
    gen = torch.Generator(device="cuda").manual_seed(3)
    t = {n: [torch.randn((2, n, h, 128), generator=gen, device="cuda").bfloat16() for h in (8, 2, 2)] for n in (700, 1, 90)}
    for c in (cache, same):
        c.step(*t[700], cos, sin)
        c._attend_ws = None                                # (as if the prompt had come another way)
        c.step(*t[1], cos, sin)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cache.step(*t[1], cos, sin)
    want = same.step(*t[1], cos, sin)
    room = cache._attend_ws.numel()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    longer, want_longer = cache.step(*t[90], cos, sin), same.step(*t[90], cos, sin)
    assert torch.equal(longer, want_longer) and cache._attend_ws.numel() > room
    others = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in [room, room, room - 256, 4096, 4096] for _ in range(5)]
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(bool((x == 7).all()) for x in others)
        assert torch.equal(cache.step(*t[1], cos, sin), same.step(*t[1], cos, sin))


def test_a_first_step_is_not_captured():
    print("[gpu-case] first step in a capture", flush=True)
    cache = decode.DecodeCache(shape(1, 1, 2, 40, 30))
    cos, sin = rkv.rotary_tables(40)
    t = [torch.zeros((1, 2, h, 128), dtype=torch.bfloat16, device="cuda") for h in (2, 1, 1)]
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="before the capture"):
        with torch.cuda.graph(graph):
            cache.step(*t, cos, sin)
    assert cache.length == 0 and torch.isfinite(cache.step(*t, cos, sin).float()).all()
