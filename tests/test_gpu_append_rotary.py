"""Ragged batches of new tokens rotated and appended: against float64, byte for byte where nothing is rotated, nothing else written."""
import pytest
import torch

from attend_reference import Batch, int32, turned64
from paper_2505_24133_amd import rkv

pytestmark = pytest.mark.gpu
ALPHA = 8


def append(b, held, seen, rotary=128, interleaved=False, rows=40000, alpha=ALPHA, with_q_cache=True, strided=False, in_place=False):
    """One call on copies; checks everything that it wrote and that the rest is as it was."""
    dev, H, Hq = "cuda", b.H, b.H * b.G
    b.shape.alpha = alpha
    cos, sin = rkv.rotary_tables(rows, rotary, 10000.0)
    heads = Hq + 2 * H
    wide = torch.randn((b.T, heads + 1, 128), generator=b.gen, device=dev).bfloat16()
    if strided:
        q, k_new, v_new = wide[:, :Hq], wide[:, Hq:Hq + H], wide[:, Hq + H:heads]
    else:
        q, k_new, v_new = (wide[:, x:y].contiguous() for x, y in ((0, Hq), (Hq, Hq + H), (Hq + H, heads)))
    ring = torch.randn((b.P, Hq, alpha, 128), generator=b.gen, device=dev).bfloat16() if with_q_cache else None
    k0, v0, ring0, q0 = b.loaded(b.k).clone(), b.loaded(b.v).clone(), None if ring is None else ring.clone(), q.clone()
    out0 = torch.full_like(q, 5.0)
    q_out = rkv.rkv_cache_append_rotary(b.shape, b.k, b.v, ring, k_new, v_new, q, cos, sin, b.starts, int32(held), int32(seen),
                                        interleaved=interleaved, q_out=q if in_place else out0)
    want_k, want_v, want_q = k0.double(), v0.double(), (q0 if in_place else torch.full_like(q0, 5.0)).double()
    err_k, err_q = torch.zeros_like(want_k), torch.zeros_like(want_q)
    want_ring = None if ring is None else ring0.double()
    err_ring = None if ring is None else torch.zeros_like(want_ring)
    at = 0
    for p, n in enumerate(b.new):
        position = (torch.arange(n, device=dev) + seen[p])
        c, s = (t[position.clamp(0, rows - 1)] for t in (cos, sin))
        y, e = turned64(q0[at:at + n], c, s, interleaved)
        want_q[at:at + n], err_q[at:at + n] = y, e
        for j in range(max(0, n - alpha), n):
            if ring is not None:
                want_ring[p, :, (seen[p] + j) % alpha], err_ring[p, :, (seen[p] + j) % alpha] = y[j], e[j]
        y, e = turned64(k_new[at:at + n], c, s, interleaved)
        for j in range(n):
            row = held[p] + j
            if 0 <= row < b.N:
                want_k[p, :, row], err_k[p, :, row] = y[j], e[j]
                want_v[p, :, row] = v_new[at + j].double()
        at += n
    assert bool(((b.loaded(b.k).double() - want_k).abs() <= err_k).all()), "keys"
    assert torch.equal(b.loaded(b.v).double(), want_v), "values"
    assert bool(((q_out.double() - want_q).abs() <= err_q).all()), "queries"
    if ring is not None:
        assert bool(((ring.double() - want_ring).abs() <= err_ring).all()), "query cache"


@pytest.mark.parametrize("rotary,interleaved", [(128, False), (128, True), (64, False), (64, True), (32, False), (16, True), (112, False)])
@pytest.mark.parametrize("page,strided", [(0, False), (0, True), (16, False), (64, True)])
def test_ragged_batch(rotary, interleaved, page, strided):
    print(f"[gpu-case] append rotary={rotary} interleaved={interleaved} page={page} strided={strided}", flush=True)
    new, held = [1, 0, 17, 3, 9, 1], [0, 5, 14, 15, 31, 63]
    b = Batch(2, 3, new, [64] * 6, N=64, page=page, strided=strided, seed=rotary + page, extra_tokens=3)
    append(b, held, [0, 1, 20000, 77, 8, 39990], rotary, interleaved, strided=strided)


@pytest.mark.parametrize("H,G,new,held,page", [
    pytest.param(1, 1, [1], [0], 0, id="one token, one head"),
    pytest.param(8, 4, [1] * 65, [i * 3 for i in range(65)], 16, id="65 problems"),
    pytest.param(2, 4, [1] * 300, [i for i in range(300)], 16, id="300 problems"),
    pytest.param(8, 5, [700, 333], [0, 11], 64, id="prompts"),
    pytest.param(1, 71, [2, 1], [3, 4], 0, id="71 query heads a KV head"),
])
def test_sizes(H, G, new, held, page):
    b = Batch(H, G, new, [h + n for h, n in zip(held, new)], page=page, seed=2)
    append(b, held, [h + 100 for h in held])


def test_query_cache_of_other_sizes_and_none():
    for alpha in (1, 3, 16):
        append(Batch(2, 2, [1, 5, 40], [10, 20, 64], N=64, seed=alpha), [2, 9, 3], [7, 1000, 5], alpha=alpha)
    append(Batch(2, 2, [1, 5], [10, 20], N=64, seed=5), [2, 9], [7, 1000], with_q_cache=False)


def test_in_place():
    append(Batch(2, 2, [1, 5, 40], [10, 20, 64], N=64, seed=6), [2, 9, 3], [7, 1000, 5], in_place=True, strided=True)
    append(Batch(2, 2, [1, 5, 40], [10, 20, 64], N=64, seed=6), [2, 9, 3], [7, 1000, 5], in_place=True, interleaved=True)


def test_rows_outside_the_cache_are_left_out():
    """Rows past the cache or before it, and positions past the table: nothing is written outside, the rest is as it should be."""
    b = Batch(2, 2, [4, 3, 2], [10, 10, 10], N=16, page=16, seed=7)
    append(b, [14, -1, 16], [0, 50, 39999])
    b = Batch(2, 2, [4, 3], [10, 10], N=16, seed=8)
    append(b, [14, -2], [10 ** 9, 5], rows=100)


def test_pages_outside_the_pool_are_left_out():
    b = Batch(1, 2, [2, 2], [32, 32], N=32, page=16, seed=9)
    before = b.k.clone()
    b.table[0, 1], b.table[1, 1] = -1, b.pages
    cos, sin = rkv.rotary_tables(64)
    new = torch.ones((4, 1, 128), dtype=torch.bfloat16, device="cuda")
    q = torch.ones((4, 2, 128), dtype=torch.bfloat16, device="cuda")
    rkv.rkv_cache_append_rotary(b.shape, b.k, b.v, None, new, new, q, cos, sin, b.starts, int32([15, 15]), int32([0, 0]))
    changed = (b.k != before).any(-1)
    assert changed.sum() == 2                                # the one row of either problem that lies in a page of the pool
    for p in range(2):
        assert changed[b.table[p, 0].long(), 0, 15]


def test_graph():
    b = Batch(2, 2, [1, 1], [40, 40], N=64, page=16, seed=10)
    cos, sin = rkv.rotary_tables(100)
    k_new, v_new = (torch.randn((2, 2, 128), generator=b.gen, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((2, 4, 128), generator=b.gen, device="cuda").bfloat16()
    ring = torch.zeros((2, 4, 8, 128), dtype=torch.bfloat16, device="cuda")
    held, seen, out = int32([3, 20]), int32([3, 50]), torch.empty_like(q)

    def call(k, v, ring, out):
        rkv.rkv_cache_append_rotary(b.shape, k, v, ring, k_new, v_new, q, cos, sin, b.starts, held, seen, q_out=out)

    eager = [t.clone() for t in (b.k, b.v, ring, out)]
    call(*[t.clone() for t in eager])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(b.k, b.v, ring, out)
    for _ in range(4):
        graph.replay()
        call(*eager)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((b.k, b.v, ring, out), eager))
        held += 1
        seen += 1
        k_new.normal_(generator=b.gen)


def test_lists_that_begin_before_or_end_behind_the_tokens():
    """starts below 0 and past T are taken as 0 and T, as attention takes them: the same rows, positions and kept queries."""
    print("[gpu-case] append, starts outside the tokens", flush=True)
    for new, outside in (([3, 6], [-2, 3, 12]), ([1, 20], [-(2 ** 31), 1, 2 ** 31 - 1]), ([12], [-5, 40])):
        got = []
        for starts in (outside, None):
            b = Batch(2, 3, new, [64] * len(new), N=64, seed=11)
            q = torch.randn((b.T, 6, 128), generator=b.gen, device="cuda").bfloat16()
            kv = torch.randn((2, b.T, 2, 128), generator=b.gen, device="cuda").bfloat16()
            ring = torch.zeros((b.P, 6, 4, 128), dtype=torch.bfloat16, device="cuda")
            b.shape.alpha = 4
            cos, sin = rkv.rotary_tables(100)
            out = rkv.rkv_cache_append_rotary(b.shape, b.k, b.v, ring, kv[0], kv[1], q, cos, sin, b.starts if starts is None else int32(starts),
                                              int32([5, 7][:b.P]), int32([30, 50][:b.P]))
            got.append((b.k, b.v, ring, out))
        assert all(torch.equal(x, y) for x, y in zip(*got)), new
