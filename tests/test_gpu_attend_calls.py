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
