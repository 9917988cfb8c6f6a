"""The operators around the cache in float64, from their definitions, with the bounds that their arithmetic keeps: inputs for the
tests of attention over (paged) caches, the reference, and the largest error that fp32 sums and bf16 roundings allow."""
import math

import torch

from paper_2505_24133_amd import rkv

D = 128
HALF = 2.0 ** -8            # bf16: half a step, relative


def prefix_sum(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def int32(values, device="cuda"):
    return torch.tensor(values, dtype=torch.int32, device=device)


class Batch:
    """A ragged batch over caches of N rows: `new` tokens a problem, the last of the `lens` rows that its cache holds.  `rows_k`, `rows_v`
    [P, H, N, d] are the caches' rows wherever they lie: contiguous, strided ([P, N, H, d] in memory) or in pages."""

    def __init__(self, H, G, new, lens, N=None, page=0, strided=False, seed=0, device="cuda", extra_tokens=0, fill=None):
        gen = torch.Generator(device=device).manual_seed(seed)
        P, N = len(new), N or max(max(lens), 1)
        self.P, self.H, self.G, self.N, self.new, self.lens, self.page = P, H, G, N, new, lens, page
        T = sum(new) + extra_tokens
        self.T = T
        self.q = torch.randn((T, H * G, D), generator=gen, device=device).bfloat16()
        self.rows_k = (torch.randn((P, H, N, D), generator=gen, device=device) * 1.5).bfloat16()
        self.rows_v = torch.randn((P, H, N, D), generator=gen, device=device).bfloat16()
        if fill is not None:                                   # what lies behind a problem's rows
            for p in range(P):
                self.rows_k[p, :, lens[p]:] = fill
                self.rows_v[p, :, lens[p]:] = fill
        self.starts, self.kv_len = int32(prefix_sum(new), device), int32(lens, device)
        self.shape = rkv.Shape(num_problems=P, kv_heads=H, q_heads=H * G, n_tokens=N, budget=max(N - 1, 9))
        self.strided, self.gen, self.device = strided, gen, device
        if page:
            per = -(-N // page)
            self.per = per
            self.table = torch.randperm(P * per, generator=gen, device=device).int().reshape(P, per)
            self.shape.page_size, self.shape.block_table = page, self.table
            self.pages = P * per
        self.store()

    def store(self):
        """The rows as the call takes them."""
        self.k, self.v = (self._stored(t) for t in (self.rows_k, self.rows_v))

    def _stored(self, rows):
        P, H, N, page = self.P, self.H, self.N, self.page
        if page:
            padded = torch.zeros((P, H, self.per * page, D), dtype=rows.dtype, device=self.device)
            padded[:, :, :N] = rows
            pool = torch.zeros((self.pages, H, page, D), dtype=rows.dtype, device=self.device)
            pool[self.table.reshape(-1).long()] = padded.view(P, H, self.per, page, D).transpose(1, 2).reshape(-1, H, page, D)
            return pool
        if self.strided:
            return rows.transpose(1, 2).contiguous().transpose(1, 2)
        return rows.contiguous()

    def loaded(self, t):
        """The rows [P, H, N, d] of a cache in the stored form."""
        if not self.page:
            return t
        P, H, page = self.P, self.H, self.page
        return t[self.table.reshape(-1).long()].view(P, self.per, H, page, D).transpose(1, 2).reshape(P, H, self.per * page, D)[:, :, :self.N]


def attend64(b, window=0, sinks=0, scale=None):
    """out, lse and the largest errors of both that the kernels' arithmetic allows, all float64 [T, Hq, d] and [T, Hq].

    With weights w (sum 1) and A = sum w |v|: rounding the weights to bf16 moves out by at most HALF A, rounding out itself by HALF |out|.
    Scores: a sum of d = 128 products in fp32 is off by at most d 2^-24 sum |q_i k_i| scale, and their scaling by 2 roundings; with
    E the largest of these over the visible rows a weight is off by 2 E relative, the sum of n of them by E + n 2^-24, and the sums with v by
    another n 2^-24 A.  (2 in front of the fp32 terms: the exponential's own rounding and the rescaling of sums.)"""
    scale = 1 / math.sqrt(D) if scale is None else scale
    T, Hq = b.T, b.H * b.G
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device=b.device)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=b.device)
    e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
    at = 0
    for p, (n, total) in enumerate(zip(b.new, b.lens)):
        for h in range(b.H):
            if n == 0 or total == 0:
                continue
            k, v = (t[p, h, :total].double().nan_to_num(0.0, 0.0, 0.0) for t in (b.rows_k, b.rows_v))
            q = b.q[at:at + n, h * b.G:(h + 1) * b.G].double().reshape(n * b.G, D)
            r = total - n + torch.arange(n, device=b.device).repeat_interleave(b.G)[:, None]
            c = torch.arange(total, device=b.device)
            seen = c <= r
            if window:
                seen = seen & ((c > r - window) | (c < sinks))
            s = torch.where(seen, scale * (q @ k.t()), -math.inf)
            top = s.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, 0.0, top)
            w = torch.exp(s - top)
            total_w = w.sum(-1, keepdim=True)
            w = torch.where(total_w > 0, w / total_w, 0.0)
            o, A = w @ v, w @ v.abs()
            size = scale * (q.abs() @ k.abs().t())
            E = torch.where(seen, (D + 2) * 2.0 ** -24 * size, 0.0).amax(-1, keepdim=True) * 2
            count = seen.sum(-1, keepdim=True)
            part = slice(at, at + n), slice(h * b.G, (h + 1) * b.G)
            out[part] = o.view(n, b.G, D)
            lse[part] = (top + total_w.log()).view(n, b.G)
            e_out[part] = (HALF * (A + o.abs()) + 2 * (3 * E + 2 * count * 2.0 ** -24) * A + 1e-30).view(n, b.G, D)
            e_lse[part] = (2 * (E + count * 2.0 ** -24 + (top + total_w.log()).nan_to_num(0, 0, 0).abs() * 2.0 ** -23 + 2.0 ** -23)).view(n, b.G)
        at += n
    return out, lse, e_out, e_lse


def check(got, want, where=""):
    """(out, lse) within the errors of attend64's answer; what is compared last is printed when it fails."""
    out, lse = got
    ref, ref_lse, e_out, e_lse = want
    empty = ref_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty), f"{where}: rows without a visible row"
    assert (out[empty] == 0).all(), f"{where}: rows without a visible row are zero"
    worst = ((out.double() - ref).abs() / e_out.clamp_min(1e-300))[~empty]
    assert worst.numel() == 0 or bool((worst <= 1).all()), f"{where}: out is off by {worst.max().item():.3g} of what is allowed"
    worst = ((lse.double() - ref_lse).abs() / e_lse.clamp_min(1e-300))[~empty]
    assert worst.numel() == 0 or bool((worst <= 1).all()), f"{where}: lse is off by {worst.max().item():.3g} of what is allowed"


def turned64(x, cos, sin, interleaved):
    """x [T, heads, d] rotated in float64 by cos, sin [T, pairs], and the largest error of the fp32 rotation rounded to bf16."""
    pairs = cos.shape[1]
    x, c, s = x.double(), cos.double()[:, None], sin.double()[:, None]
    i = torch.arange(pairs, device=x.device)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    y, err = x.clone(), torch.zeros_like(x)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    err[..., first] = HALF * y[..., first].abs() + 2 * 2.0 ** -23 * ((a * c).abs() + (b * s).abs())
    err[..., second] = HALF * y[..., second].abs() + 2 * 2.0 ** -23 * ((b * c).abs() + (a * s).abs())
    return y, err
