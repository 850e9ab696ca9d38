"""64-bit restatements of the operators of the 8-bit cache, and the bounds that their kernels are held to.

Nothing here calls the CUDA library.  A cache is e4m3 codes with a power-of-two scale for each (page, kv-head) of K and of V.
Codes, scales and summaries are exact, so they are compared bit for bit; attention is computed in fp64 from the values that the
codes stand for.

Bounds of the decode kernel (out and lse fp32).  A logit is a sum of D products that are exact in fp32, kept in fp32: its error is
at most (D + 2) * 2^-23 times the sum of the products' magnitudes.  The exponent, logit plus logarithm of V's scale, adds 2^-22 of
its terms' magnitudes, exp2 and the weights' sum 2^-18 relative (as in prompt_ref).  A weight times V's scale enters its product
with V's codes as two halves, 2^-22 relative, not below 2^-25 of the largest such product; the sums over tokens are fp32.

Bounds of the chunk kernel (out bf16, lse fp32): those of prompt_ref, and a query row that is split into two rows of codes.  With
2^e the smallest power of two that brings the row's maximum to 448 or below (so the maximum is above 224 * 2^e), an element of
at least 2^-2 * 2^e has its last bit at 2^-9 * 2^e or above, the smallest step of a code, and is exact; a smaller one is off by
half of that step at most, 2^-10 * 2^e."""
from __future__ import annotations

import math

import prompt_ref
import torch

PAGE = 16
E4M3 = torch.float8_e4m3fn


def scale_of(top):
    """Smallest 2^e, -64 <= e <= 7, with top <= 448 * 2^e (fp64 tensor of magnitudes that are bf16 numbers)."""
    e = torch.full_like(top, -64.0)
    for k in range(-63, 8):
        e = torch.where(top > 448.0 * 2.0 ** (k - 1), torch.full_like(top, float(k)), e)
    return torch.exp2(e)


def nearest_code(x):
    """x (fp64) rounded to the nearest e4m3 value, ties to even, saturated at 448; as fp64."""
    mag = x.abs().clamp(max=448.0)
    e = torch.floor(torch.log2(mag.clamp(min=2.0 ** -6))).clamp(min=-6)
    e = torch.where(torch.exp2(e) > mag.clamp(min=2.0 ** -6), e - 1, e)
    step = torch.exp2(e - 3)
    return torch.sign(x) * torch.round(mag / step) * step          # torch.round: ties to even


def append_rows(codes, scale, rows, held, first, last):
    """Slots first..last-1 of one page get ``rows`` [last - first, H, D] (bf16); codes [H, 16, D] fp64, scale [H] fp64; ``held``:
    the page's earlier slots belong to the request.  Returns new codes and scale."""
    x = rows.double().transpose(0, 1)
    s = scale_of(x.abs().amax((1, 2)))
    codes = codes.clone()
    if held:
        s = torch.maximum(s, scale)
        codes[:, :first] = nearest_code(codes[:, :first] * (scale / s)[:, None, None])
    codes[:, first:last] = nearest_code(x / s[:, None, None])
    return codes, s


def append(k_codes, v_codes, scales, meta, k, v, new, total, page_table):
    """All of se_kv8_append but the rotation: rotated K and V rows [T, H, D] (bf16) into copies of the cache (fp64)."""
    kc, vc, sc = k_codes.double(), v_codes.double(), scales.double()
    mt = None if meta is None else meta.double()
    row = 0
    for r, (n, t) in enumerate(zip(new, total)):
        o = t - n
        for b in range(o // PAGE, (t + PAGE - 1) // PAGE if n else o // PAGE):
            a, z = max(o - b * PAGE, 0), min(t - b * PAGE, PAGE)
            pid = int(page_table[r, b])
            at = slice(row + b * PAGE + a - o, row + b * PAGE + z - o)
            if pid < 0 or pid >= kc.shape[0]:
                continue
            kc[pid], sc[pid, :, 0] = append_rows(kc[pid], sc[pid, :, 0], k[at], a > 0, a, z)
            vc[pid], sc[pid, :, 1] = append_rows(vc[pid], sc[pid, :, 1], v[at], a > 0, a, z)
            if mt is not None:
                x = kc[pid, :, :z] * sc[pid, :, 0][:, None, None]
                mt[pid, :, 0], mt[pid, :, 1] = x.amin(1), x.amax(1)
        row += n
    return kc, vc, sc, mt


def make_cache(g, P, H, D, device, spread=True):
    """Codes of random values and their scales, page by page of different magnitudes; some slots hold NaN codes (0x7f) that
    no call may read into a result, where the caller marks them."""
    x = torch.randn(2, P, H, PAGE, D, generator=g, dtype=torch.float64)
    if spread:
        x *= torch.exp2(torch.randint(-6, 6, (2, P, H, 1, 1), generator=g).double())
    x[0, :, :, :, 3] *= 8.0
    x = x.to(torch.bfloat16).double()
    s = scale_of(x.abs().amax((3, 4)))
    codes = nearest_code(x / s[..., None, None]).float().to(E4M3)
    return codes[0].contiguous().to(device), codes[1].contiguous().to(device), torch.stack([s[0], s[1]], -1).float().contiguous().to(device)


def values(codes, scale):
    """[P, H, 16, D] fp64 values of codes with scales [P, H]."""
    return codes.double() * scale.double()[..., None, None]


def decode(q, k_codes, v_codes, scales, page_table, seq_lens, sel_idx, sel_cnt, sm_scale):
    """out, its tolerance, lse, its tolerance (fp64)."""
    B, H_q, D = q.shape
    H_kv = k_codes.shape[1]
    G = H_q // H_kv
    out = torch.zeros(B, H_q, D, dtype=torch.float64, device=q.device)
    tol, lse = torch.zeros_like(out), torch.full((B, H_q), -math.inf, dtype=torch.float64, device=q.device)
    ltol = torch.zeros_like(lse)
    for r in range(B):
        n = int(seq_lens[r])
        for h in range(H_kv):
            pages = range((n + PAGE - 1) // PAGE) if sel_idx is None else sel_idx[r, h, :int(sel_cnt[r, h])].tolist()
            kk, vv, ss = [], [], []
            for b in pages:
                pid = int(page_table[r, b])
                if pid < 0:
                    continue
                m = min(PAGE, n - b * PAGE)
                kk.append(k_codes[pid, h, :m].double() * scales[pid, h, 0].double())
                vv.append(v_codes[pid, h, :m].double() * scales[pid, h, 1].double())
                ss.append(scales[pid, h, 1].double().expand(m))
            if not kk:
                continue
            kk, vv, ss = torch.cat(kk), torch.cat(vv), torch.cat(ss)
            x = q[r, h * G:(h + 1) * G].double()
            z = sm_scale * x @ kk.t()
            zerr = sm_scale * (D + 2) * 2.0 ** -23 * (x.abs() @ kk.abs().t())
            top = z.amax(1, keepdim=True)
            zerr = zerr + 2.0 ** -22 * (z.abs() + top.abs() + ss.log().abs() + ss.log().abs().max()) + 2.0 ** -18
            p = (z - top).exp()
            s = p.sum(1, keepdim=True)
            w = p / s
            rows = slice(h * G, (h + 1) * G)
            out[r, rows] = w @ vv
            # error of every weight, and of their sum
            werr = w * (zerr + (w * zerr).sum(1, keepdim=True) + 2.0 ** -22) + 2.0 ** -37 * (w * ss).amax(1, keepdim=True) / ss
            tol[r, rows] = 1.01 * (werr @ vv.abs()) + 2.0 ** -18 * (w @ vv.abs())
            lse[r, rows] = (top + s.log())[:, 0]
            ltol[r, rows] = (w * zerr).sum(1) + 2.0 ** -22 * lse[r, rows].abs() + 2.0 ** -22
    return out, tol, lse, ltol


def chunk(b, scale):
    """prompt_ref.attend over the bf16 cache of the codes' values, with the split of the query rows in the bounds.  ``b``: a
    prompt_ref.Batch."""
    out, tol, lse, ltol = prompt_ref.attend(b, True, scale)
    for r in range(b.B):
        n, rows = b.new[r], b.rows(r)
        if n == 0:
            continue
        q = b.q[rows].double().abs().view(n, b.H_kv, -1, b.D).permute(1, 2, 0, 3)
        step = torch.exp2(torch.ceil(torch.log2(q.amax(-1, keepdim=True).clamp(min=1e-300) / 448)))
        k, _ = prompt_ref.cached(b, r, b.k_cache)
        v, _ = prompt_ref.cached(b, r, b.v_cache)
        # the logits' error, and what it does to lse and (twice, for weight and sum) to the output
        z = (((q < 0.25 * step).double() @ k[:, None].abs().transpose(-1, -2)).amax(-1, keepdim=True) * 2.0 ** -10 * step * scale)
        put = lambda x: x.permute(2, 0, 1, 3).reshape(n, b.H_q, -1)  # noqa: E731
        ltol[rows] += put(z)[..., 0]
        tol[rows] += put(2.1 * z * v.abs().amax((1, 2))[:, None, None, None])
    return out, tol, lse, ltol
