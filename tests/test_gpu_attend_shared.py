"""Attention of problems that share prompts: the float64 reference of every problem by itself, and rkv_attend's own answer."""
import pytest
import torch

from attend_reference import Batch, attend64, check, int32, prefix_sum
from paper_2505_24133_amd import rkv

pytestmark = pytest.mark.gpu


def grouped(H, G, sizes, prefixes, new, own, page=0, outside=0, seed=0, **kw):
    """A batch whose problems come in groups (of `sizes`) with common first rows, `own` rows behind the prefix before the new tokens."""
    P = sum(sizes) + outside
    of = [g for g, n in enumerate(sizes) for _ in range(n)]
    lens = [(prefixes[of[p]] if p < len(of) else 0) + own[p % len(own)] + new[p % len(new)] for p in range(P)]
    b = Batch(H, G, [new[p % len(new)] for p in range(P)], lens, page=page, seed=seed, **kw)
    first = prefix_sum(sizes)
    for g, (at, n) in enumerate(zip(first, sizes)):
        for p in range(at + 1, at + n):
            b.rows_k[p, :, :prefixes[g]] = b.rows_k[at, :, :prefixes[g]]
            b.rows_v[p, :, :prefixes[g]] = b.rows_v[at, :, :prefixes[g]]
            if page:
                b.table[p, :prefixes[g] // page] = b.table[at, :prefixes[g] // page]
    b.group_starts, b.prefix_len = int32(first), int32(prefixes)
    b.store()
    return b


def run(b, window=0, sinks=0, **kw):
    kw.setdefault("max_new", max(b.new))
    return rkv.rkv_attend_shared(b.shape, b.q, b.k, b.v, b.starts, b.kv_len, b.group_starts, b.prefix_len, window=window, sinks=sinks,
                                 want_lse=True, **kw)


CASES = [
    pytest.param(dict(H=2, G=4, sizes=[5], prefixes=[333], new=[1], own=[3, 50, 0, 200, 64]), id="one group"),
    pytest.param(dict(H=2, G=4, sizes=[64], prefixes=[1000], new=[1], own=[7, 100], page=16), id="64 samples, paged"),
    pytest.param(dict(H=1, G=5, sizes=[2, 0, 3, 1], prefixes=[37, 20, 128, 65], new=[1, 3], own=[10, 0, 31], page=32), id="groups, one of them empty"),
    pytest.param(dict(H=2, G=7, sizes=[4, 4], prefixes=[0, 500], new=[2], own=[20, 90]), id="one without a prefix"),
    pytest.param(dict(H=2, G=3, sizes=[2, 2], prefixes=[100, 64], new=[1, 2], own=[20, 5], outside=3), id="problems in no group"),
    pytest.param(dict(H=1, G=4, sizes=[3, 2], prefixes=[200, 300], new=[40, 1, 100], own=[0, 77], page=64), id="prompts behind a prompt"),
    pytest.param(dict(H=1, G=1, sizes=[1], prefixes=[1], new=[1], own=[0]), id="one of each"),
    pytest.param(dict(H=1, G=70, sizes=[2], prefixes=[90], new=[1], own=[5]), id="70 query heads a KV head"),
    pytest.param(dict(H=1, G=2, sizes=[3] * 80, prefixes=[20 + i for i in range(80)], new=[1, 0, 2], own=[9, 1], page=16), id="80 groups"),
]


@pytest.mark.parametrize("how", CASES)
def test_against_each_by_itself(how):
    print(f"[gpu-case] attend shared {how}", flush=True)
    b = grouped(seed=3, **how)
    check(run(b), attend64(b))
    for window, sinks in ((16, 0), (100, 4), (40, 150)):
        check(run(b, window, sinks), attend64(b, window, sinks), f"window {window} sinks {sinks}")


def test_the_prefix_is_read_from_the_first_problem():
    """Copies of the prefix in the other problems are not looked at."""
    b = grouped(2, 4, [4], [300], [1], [20, 60], seed=4)
    want = attend64(b)
    b.rows_k[1:, :, :300] = float("nan")
    b.rows_v[1:, :, :300] = float("nan")
    b.store()
    check(run(b), want)


def test_shorter_than_the_prefix():
    """A problem that is not through its prefix yet sees what it holds of it; one with no rows sees nothing."""
    b = grouped(2, 4, [4], [100], [2], [50], seed=5)
    lens = [152, 60, 1, 0]
    b.lens = lens
    b.kv_len.copy_(int32(lens))
    check(run(b), attend64(b))


def test_hidden_values_that_are_not_finite():
    """A prompt's last tokens are hidden from chunks of it that are attended before them."""
    b = grouped(1, 4, [2], [120], [1], [10], seed=6)
    b.lens = [131, 90]
    b.kv_len.copy_(int32(b.lens))
    b.rows_v[0, :, 100, 3] = float("inf")
    b.store()
    out, lse = run(b)
    b.rows_v[1, :, 90:] = 0
    want = attend64(b)
    check((out[1:], lse[1:]), tuple(t[1:] for t in want))
    assert (out[0, :, 3] == float("inf")).all()


def test_groups_in_the_middle_and_padding():
    """Problems before and behind the groups, tokens before the first problem's and behind the last one's."""
    b = grouped(2, 4, [3, 2], [150, 60], [1, 2], [30, 5], outside=2, seed=9, extra_tokens=2000)
    P = b.P
    # the first problem keeps to itself: the groups start behind it
    b2 = grouped(2, 4, [1, 3, 2], [0, 150, 60], [1, 2], [30, 5], outside=1, seed=10, extra_tokens=700)
    b2.group_starts, b2.prefix_len = int32([1, 4, 6]), int32([150, 60])
    for x in (b, b2):
        n = sum(x.new)
        out, lse = torch.full_like(x.q, 3.0), torch.full(x.q.shape[:2], 4.0, device="cuda")
        run(x, out=out, lse=lse)
        check((out[:n], lse[:n]), tuple(t[:n] for t in attend64(x)))
        assert (out[n:] == 3).all() and (lse[n:] == 4).all()
    # tokens that belong to no problem, in front
    shifted = int32([0] * (P + 1)) + b.starts + 5
    q = torch.cat((torch.zeros_like(b.q[:5]), b.q))[:b.T]
    out = torch.full_like(q, 3.0)
    rkv.rkv_attend_shared(b.shape, q, b.k, b.v, shifted, b.kv_len, b.group_starts, b.prefix_len, max_new=2, out=out)
    n = sum(b.new)
    want = attend64(b)
    assert bool(((out[5:5 + n].double() - want[0][:n]).abs() <= want[2][:n]).all()) and (out[:5] == 3).all() and (out[5 + n:] == 3).all()


@pytest.mark.parametrize("G, new", [(70, [1]), (66, [2, 0, 1]), (4, [1, 30])])
def test_problems_in_no_group_beside_many_rows(G, new):
    """What the workspace held before is not taken for a prefix's part."""
    b = grouped(1, G, [2], [90], new, [5, 40], outside=3, seed=11)
    ws = rkv.make_attend_workspace(b.shape, b.T, max(b.new), groups=1)
    for left in (0, 1, 0x3f, 0x7f, 0xff):
        check(run(b, ws=ws.fill_(left)), attend64(b), f"workspace of {left}")


def test_no_groups():
    b = Batch(2, 4, [1, 2], [100, 300], seed=7)
    b.group_starts, b.prefix_len = int32([0]), int32([])
    check(run(b), attend64(b))


def test_graph_and_workspace():
    b = grouped(2, 4, [8, 8], [200, 1000], [1], [20, 60, 300], page=16, seed=8)
    ws = rkv.make_attend_workspace(b.shape, b.T, 1, groups=2).fill_(0xff)
    out, lse = torch.empty_like(b.q), torch.empty(b.q.shape[:2], device="cuda")
    run(b, ws=ws, out=out, lse=lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(b, ws=ws, out=out, lse=lse)
    for _ in range(3):
        b.q.normal_(generator=b.gen)
        graph.replay()
        torch.cuda.synchronize()
        check((out, lse), attend64(b))
        eager = run(b)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 24 + 1, 400, 30])
@pytest.mark.parametrize("G,new", [(4, [5]), (4, [40]), (40, [3, 9])])
def test_tokens_before_the_first_row_under_any_window(window, G, new):
    """Fewer rows than new tokens, in a group too: the first ones see nothing, the others what they see."""
    print(f"[gpu-case] attend shared, tokens before the first row, window={window} G={G} new={new}", flush=True)
    b = grouped(2, G, [4], [100], new, [50], outside=1, seed=12)
    b.lens = [150 + new[0], 60, 2, 1, 3]
    b.kv_len.copy_(int32(b.lens))
    for sinks in (0, 2):
        check(run(b, window, sinks), attend64(b, window, sinks), f"sinks {sinks}")
