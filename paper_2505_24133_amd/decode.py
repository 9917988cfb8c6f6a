"""Decode-loop view of the compression step (Sec. 3.1, Alg. 1, App. C.1).

``DecodeCache`` keeps, per (sequence, layer) problem and KV head, a cache of
N = B_budget + B_buffer rows and the query states of the last alpha decode steps.  Every decode
step appends one token; when the buffer behind the budget is full the cache is compressed to
``budget`` rows (the selected candidates in their original order, then the alpha observation
tokens) and decoding continues.  By default two cache allocations are used alternately so that
the compaction is a plain gather from one into the other; with ``inplace=True`` there is one
allocation and the kept rows are moved to its front.  All work runs in the HIP library; this
class only owns the buffers and the counters.

``append`` takes rows that carry their positions already and leaves attention to the caller; ``step`` takes one token or a
whole prompt as the projections give them, rotates and appends them, attends over the cache and compresses it when it is full.
"""
from __future__ import annotations

import torch

from . import rkv


def _capturing(device) -> bool:
    return device.type == "cuda" and torch.cuda.is_current_stream_capturing()


class DecodeCache:
    def __init__(self, shape: rkv.Shape, device="cuda", inplace: bool = False):
        self.shape = shape
        self.inplace = inplace
        P, H, Hq, N, d = shape.num_problems, shape.kv_heads, shape.q_heads, shape.n_tokens, shape.head_dim
        copies = 1 if inplace else 2
        self._k = [torch.zeros((P, H, N, d), dtype=torch.bfloat16, device=device) for _ in range(copies)]
        self._v = [torch.zeros((P, H, N, d), dtype=torch.bfloat16, device=device) for _ in range(copies)]
        self.q_cache = torch.zeros((P, Hq, shape.alpha, d), dtype=torch.bfloat16, device=device)
        self.kept_idx = torch.zeros((P, H, shape.budget), dtype=torch.int32, device=device)
        self._ws = rkv.make_workspace(shape, device)
        self._cur = 0
        self.length = 0            # rows currently held per head
        self.tokens_seen = 0       # decode steps so far
        self.compressions = 0
        self._counts = None        # row n: n for every problem, made at the first step
        self._count_of = {}        # its rows that steps have asked for
        self._starts = {}          # by new tokens a problem: where each problem's begin
        self._attend_room = {}     # and how much workspace their attention needs; one workspace serves them all
        self._attend_ws = None
        self._groups = None
        self._streams = {}         # by handle: the streams that steps were made on
        self._captured = False     # whether one of them was captured into a graph,
        self._kept = []            # and what that graph may use that has been replaced since

    @property
    def k(self) -> torch.Tensor:
        """Current key cache [P, H, N, d]; rows [0, length) are valid."""
        return self._k[self._cur]

    @property
    def v(self) -> torch.Tensor:
        return self._v[self._cur]

    def _count(self, n: int) -> torch.Tensor:
        """n for every problem, as the calls take lengths and positions."""
        row = self._count_of.get(n)
        if row is None:
            row = self._count_of[n] = self._counts[n]
        return row

    def _let_go(self, *tensors) -> None:
        """Tensors that steps have used and that are about to be replaced.  Steps may have been made on other streams than the one they were
        allocated on: their memory is not given out again before what those streams have been given by now is done.  A graph that a step was
        captured into uses them as often as it is replayed: then they stay."""
        if self._captured:
            self._kept += tensors
        for t in tensors:
            for stream in self._streams.values():
                t.record_stream(stream)

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor, q_new: torch.Tensor) -> bool:
        """One decode step: k_new, v_new [P, H, d], q_new [P, Hq, d].  Returns True if the step
        ended with a compression."""
        s = self.shape
        cur = self._cur
        rkv.rkv_cache_append(s, self._k[cur], self._v[cur], self.q_cache, k_new, v_new, q_new,
                             self.length, self.tokens_seen % s.alpha)
        self.length += 1
        self.tokens_seen += 1
        # (what rkv_should_compress answers for a shape that the append has just accepted)
        if self.length >= s.n_tokens > s.budget:
            self.compress()
            return True
        return False

    def share_prompt(self, group_sizes, rows) -> None:
        """Declare that the next group_sizes[0] problems hold the same values in their first rows[0] rows, the next group_sizes[1] in
        rows[1], ... (samples of one prompt): step() reads those rows once for all of them, until the first compression, after
        which every problem has rows of its own."""
        sizes, rows = [int(n) for n in group_sizes], [int(n) for n in rows]
        P = self.shape.num_problems
        if len(sizes) != len(rows) or len(sizes) > P or min(sizes + rows, default=0) < 0 or sum(sizes) > P or max(rows, default=0) > self.length:
            raise ValueError("share_prompt needs as many row counts as groups, groups of the problems there are and rows that are held")
        first = [0]
        for n in sizes:
            first.append(first[-1] + n)
        device = self.q_cache.device
        self._let_go(*self._groups or ())
        self._groups = (torch.tensor(first, dtype=torch.int32, device=device), torch.tensor(rows, dtype=torch.int32, device=device)) if sizes else None
        self._attend_room = {}

    def step(self, q_new: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor,
             interleaved: bool = False, window: int = 0, sinks: int = 0, scale=None) -> torch.Tensor:
        """n new tokens of every problem: q_new [P, n, Hq, d], k_new, v_new [P, n, H, d], not rotated yet.  They are rotated by their
        positions (cos, sin: rotary_tables with a row for every position so far), appended, and attended over everything that is
        held (or, with a window, its last rows and the first `sinks`); then the cache is compressed if it is full.  The counts are the host's:
        a step that is captured into a graph repeats its rows and positions, and needs one of as many tokens before the capture.
        Returns the attention's output [P, n, Hq, d]."""
        s = self.shape
        P, n = s.num_problems, q_new.shape[1]
        of_q, of_kv = (P, n, s.q_heads, s.head_dim), (P, n, s.kv_heads, s.head_dim)
        if q_new.shape != of_q or k_new.shape != of_kv or v_new.shape != of_kv:
            raise ValueError(f"step takes tokens of {P} problems: q_new {of_q}, k_new and v_new {of_kv}, "
                             f"got {tuple(q_new.shape)}, {tuple(k_new.shape)} and {tuple(v_new.shape)}")
        if n < 1 or self.length + n > s.n_tokens:
            raise ValueError(f"step takes tokens of {P} problems, and room for {s.n_tokens - self.length} each is left")
        if cos.shape[0] < self.tokens_seen + n:
            raise ValueError(f"the rotation tables end at position {cos.shape[0]}, before the new tokens do")
        if (self._counts is None or n not in self._starts) and _capturing(self.q_cache.device):
            raise RuntimeError(f"the first step of {n} tokens makes lists that a graph would fill only when it is replayed: make one before the capture")
        if self._counts is None:
            device = self.q_cache.device
            self._counts = torch.arange(s.n_tokens + 1, dtype=torch.int32, device=device)[:, None].expand(-1, P).contiguous()
        if n not in self._starts:
            self._starts[n] = torch.arange(0, P * n + 1, n, dtype=torch.int32, device=self.q_cache.device)
        if n not in self._attend_room:
            self._attend_room[n] = rkv.rkv_attend_workspace_size(s, P * n, n, 0 if self._groups is None else self._groups[1].shape[0])
        if self._attend_ws is None or self._attend_ws.numel() < self._attend_room[n] + 256:
            if self._attend_ws is not None:
                self._let_go(self._attend_ws)
            self._attend_ws = torch.empty(self._attend_room[n] + 256, dtype=torch.uint8, device=self.q_cache.device)
        # what attention may refuse is refused here, and its output made: behind the append the query cache has lost the slots that the new
        # queries take, so nothing may fail there
        rkv._check_sight(window, sinks, n, scale, "DecodeCache.step")
        q = q_new.flatten(0, 1)
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        if self.q_cache.is_cuda and rkv._stream() not in self._streams:
            self._streams[rkv._stream()] = torch.cuda.current_stream()
        self._captured = self._captured or _capturing(self.q_cache.device)
        starts, lens, k, v = self._starts[n], self._count(self.length + n), self.k, self.v
        # positions count from the last multiple of alpha, whose rows of the tables come first: the slots of the query cache go by them
        slot = self.tokens_seen % s.alpha
        at = self.tokens_seen - slot
        q = rkv.rkv_cache_append_rotary(s, k, v, self.q_cache, k_new.flatten(0, 1), v_new.flatten(0, 1), q, cos[at:], sin[at:],
                                        starts, self._count(self.length), self._count(slot), interleaved=interleaved)
        common = dict(window=window, sinks=sinks, scale=scale, max_new=n, ws=self._attend_ws, out=out)
        if self._groups is None:
            rkv.rkv_attend(s, q, k, v, starts, lens, **common)
        else:
            rkv.rkv_attend_shared(s, q, k, v, starts, lens, *self._groups, **common)
        self.length += n                                   # (a step that was refused has not taken place)
        self.tokens_seen += n
        if self.length >= s.n_tokens > s.budget:
            self.compress()
        return out.view(of_q)

    def compress(self) -> None:
        s = self.shape
        if self.length != s.n_tokens:
            raise RuntimeError("compress() runs when the cache holds budget + buffer rows")
        if self._groups is not None:
            self._let_go(*self._groups)
            self._groups, self._attend_room = None, {}
        if self.inplace:
            st, *_ = rkv.rkv_compress_inplace(s, self.q_cache, self.k, self.v, ws=self._ws, kept_idx=self.kept_idx)
            if st != rkv.RKV_OK:
                raise RuntimeError("compression was not triggered")
            self.length = s.budget
            self.compressions += 1
            return
        nxt = 1 - self._cur
        st, *_ = rkv.rkv_compress(s, self.q_cache, self.k, self.v, ws=self._ws,
                                  k_out=self._k[nxt][:, :, :s.budget], v_out=self._v[nxt][:, :, :s.budget],
                                  kept_idx=self.kept_idx)
        if st != rkv.RKV_OK:
            raise RuntimeError("compression was not triggered")
        self._cur = nxt
        self.length = s.budget
        self.compressions += 1
