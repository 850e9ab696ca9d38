"""64-bit restatements of the prompt-side operators and the bounds that their kernels are held to.

Nothing here calls the CUDA library.  Inputs are bf16 tensors; everything is computed in fp64 by elementary torch
operations, request by request, on the device that the inputs are on.

Bounds.  A logit is a sum of D exact bf16 products kept in fp32: its error is at most (D + 2) * 2^-23 times the sum of
the products' magnitudes (``zerr``).  exp2 of an fp32 argument and the weights' sum add 2^-18 relative and 2^-24 per
summed term.  Attention weights enter the product with V as bf16 (2^-8 relative each) and the output is rounded to
bf16 (2^-8 relative)."""
from __future__ import annotations

import dataclasses
import math

import torch

PAGE = 16
HALF_BF16 = torch.finfo(torch.bfloat16).eps / 2


@dataclasses.dataclass
class Batch:
    """A packed batch of new tokens over a paged cache."""
    H_q: int
    H_kv: int
    D: int
    new: list
    total: list
    T: int                     # rows of the token-major arrays, spare ones included
    max_pages: int
    P: int
    qkv: torch.Tensor          # [T, H_q + 2*H_kv, D], the views below share it
    cu: torch.Tensor
    seq_lens: torch.Tensor
    page_table: torch.Tensor
    k_cache: torch.Tensor
    v_cache: torch.Tensor

    @property
    def B(self):
        return len(self.new)

    @property
    def q(self):
        return self.qkv[:, :self.H_q]

    @property
    def k(self):
        return self.qkv[:, self.H_q:self.H_q + self.H_kv]

    @property
    def v(self):
        return self.qkv[:, self.H_q + self.H_kv:]

    def rows(self, r):
        s = sum(self.new[:r])
        return slice(s, s + self.new[r])


def make_batch(seed, new, past, H_q, H_kv, D, device="cuda", spare=0, absent=(), extra_pages=2, wide=0, nan_tail=True):
    """``absent``: (request, logical page) pairs without physical KV.  ``wide``: columns of the page table beyond the
    longest request's.  Slots past a request's length and spare rows hold NaN."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    total = [n + o for n, o in zip(new, past)]
    pages = [(t + PAGE - 1) // PAGE for t in total]
    P = max(1, sum(pages) + extra_pages)
    mp = max(1, max(pages)) + wide
    order = torch.randperm(P, generator=g)
    table = torch.full((len(new), mp), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(pages):
        table[r, :n] = order[at:at + n].to(torch.int32)
        at += n
    T = sum(new) + spare
    qkv = torch.randn(T, H_q + 2 * H_kv, D, generator=g).to(torch.bfloat16)
    k = torch.randn(P, H_kv, PAGE, D, generator=g).to(torch.bfloat16)
    v = torch.randn(P, H_kv, PAGE, D, generator=g).to(torch.bfloat16)
    k[..., :3] *= 4
    if nan_tail:
        qkv[sum(new):] = math.nan
        for r, t in enumerate(total):
            if t % PAGE:
                k[int(table[r, t // PAGE]), :, t % PAGE:] = math.nan
                v[int(table[r, t // PAGE]), :, t % PAGE:] = math.nan
        k[order[at:]] = math.nan
        v[order[at:]] = math.nan
    for r, b in absent:
        table[r, b] = -1
    cu = torch.zeros(len(new) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor(new), 0)
    d = lambda x: x.to(device)  # noqa: E731
    return Batch(H_q, H_kv, D, list(new), total, T, mp, P, d(qkv), d(cu), d(torch.tensor(total, dtype=torch.int32)), d(table), d(k), d(v))


def cached(b: Batch, r, cache):
    """[H_kv, tokens, D] fp64 of request r and the mask of present tokens; absent and unused slots are zero."""
    n = b.total[r]
    row = b.page_table[r, :(n + PAGE - 1) // PAGE].long()
    x = cache[row.clamp(min=0)].double().transpose(0, 1).reshape(b.H_kv, -1, b.D)[:, :n]
    present = (row >= 0).repeat_interleave(PAGE)[:n]
    return torch.where(present[None, :, None], x, 0.0), present


def contiguous(b: Batch, r):
    rows = b.rows(r)
    return b.k[rows].double().transpose(0, 1), b.v[rows].double().transpose(0, 1)


def logits(b: Batch, r, k, present, scale):
    """[H_kv, G, n, tokens] fp64 logits (-inf where not visible) and the per-row bound of their fp32 error."""
    n, past = b.new[r], b.total[r] - b.new[r]
    G = b.H_q // b.H_kv
    q = b.q[b.rows(r)].double().view(n, b.H_kv, G, b.D).permute(1, 2, 0, 3)
    z = q @ k[:, None].transpose(-1, -2) * scale
    zerr = ((q.abs() @ k[:, None].abs().transpose(-1, -2)) * scale).amax(-1, keepdim=True) * (b.D + 2) * 2.0 ** -23
    j = torch.arange(k.shape[1], device=k.device)
    seen = (j[None] <= past + torch.arange(n, device=k.device)[:, None]) & present[None]
    return torch.where(seen, z, -math.inf), zerr, seen


def attend(b: Batch, paged=True, scale=None):
    """out, lse and their bounds for every row; rows without a request are NaN."""
    scale = scale or b.D ** -0.5
    kw = dict(dtype=torch.float64, device=b.qkv.device)
    out, tol = torch.full((b.T, b.H_q, b.D), math.nan, **kw), torch.zeros(b.T, b.H_q, b.D, **kw)
    lse, ltol = torch.full((b.T, b.H_q), math.nan, **kw), torch.zeros(b.T, b.H_q, **kw)
    for r in range(b.B):
        n = b.new[r]
        if n == 0:
            continue
        if paged:
            k, present = cached(b, r, b.k_cache)
            v, _ = cached(b, r, b.v_cache)
        else:
            k, v = contiguous(b, r)
            present = torch.ones(n, dtype=torch.bool, device=k.device)
        z, zerr, seen = logits(b, r, k, present, scale)
        top = z.amax(-1, keepdim=True).clamp(min=-1e300)
        w = torch.where(seen, (z - top).exp(), 0.0)
        tot = w.sum(-1, keepdim=True)
        p = w / tot.clamp(min=1e-300)
        o, mag = p @ v[:, None], p @ v[:, None].abs()
        e = tot.log() + top
        e = torch.where(tot > 0, e, -math.inf)
        rel = HALF_BF16 + 2 * zerr + 2.0 ** -17 + k.shape[1] * 2.0 ** -23
        put = lambda x: x.permute(2, 0, 1, 3).reshape(n, b.H_q, -1)  # noqa: E731
        out[b.rows(r)] = put(o)
        tol[b.rows(r)] = put(1.01 * (HALF_BF16 * o.abs() + rel * mag))
        lse[b.rows(r)] = put(e)[..., 0]
        ltol[b.rows(r)] = put(zerr + 2.0 ** -18 + k.shape[1] * 2.0 ** -24 + 2.0 ** -22 * torch.nan_to_num(e.abs(), posinf=0.0))[..., 0]
    return out, tol, lse, ltol


def accumulate(b: Batch, lse, before, scale=None):
    """score_accum after the call and its bound, for the fp32 ``lse`` that the call is given."""
    scale = scale or b.D ** -0.5
    u, tol = before.double().clone(), before.double().abs() * 2.0 ** -23
    for r in range(b.B):
        n = b.new[r]
        if n == 0:
            continue
        k, present = cached(b, r, b.k_cache)
        z, zerr, seen = logits(b, r, k, present, scale)
        own = lse[b.rows(r)].double().view(n, b.H_kv, -1).permute(1, 2, 0)[..., None]
        w = torch.where(seen, (z - own).exp(), 0.0)
        rel = zerr + 2.0 ** -18 + 2.0 ** -22 * torch.where(seen, z, 0.0).abs().amax(-1, keepdim=True) + n * 2.0 ** -24
        add, bound = w.sum((1, 2)), (w * rel).sum((1, 2)) * 1.01
        for j in range(0, b.total[r], PAGE):
            pid = int(b.page_table[r, j // PAGE])
            if pid >= 0:
                m = min(PAGE, b.total[r] - j)
                u[pid, :, :m] += add[:, j:j + m]
                tol[pid, :, :m] += bound[:, j:j + m] + 2.0 ** -23 * u[pid, :, :m].abs()
    return u, tol


def rotate(x, positions, inv_freq, pair_axis, interleaved):
    """fp64 rotation of x [T, H, D] and its bound against a rotation in fp32 rounded to bf16."""
    n = inv_freq.numel()
    angle = (positions[pair_axis.long()].double() * inv_freq[:, None]).t()[:, None]
    lo, hi = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    x = x.double()
    y, size = x.clone(), torch.zeros_like(x)
    y[..., lo] = x[..., lo] * angle.cos() - x[..., hi] * angle.sin()
    y[..., hi] = x[..., hi] * angle.cos() + x[..., lo] * angle.sin()
    size[..., lo] = size[..., hi] = x[..., lo].abs() + x[..., hi].abs()
    # the angle is off by 2^-20 at most (its fraction of a turn and sincospif in fp32), the products by 2^-23
    return y, torch.where(size > 0, 1.01 * (HALF_BF16 * y.abs() + size * 2.0 ** -19), 0.0)
