"""Codes that are no numbers, in tokens that are seen: appended, and read by both attention calls over the 8-bit cache.

A NaN of V makes its channel NaN in the rows that see the token, one of K the whole row; every other output keeps the bits that it
has with a zero in the NaN's place (which counts as little for a page's scale as a NaN does)."""
import math

import pytest
import torch

from paper_2609_39068_b200 import binding
from test_gpu_kv8 import Chunk, Decode, I32, page_tables

pytestmark = pytest.mark.gpu
NANS = (0x7f, 0xff)


def plant(c, nans):
    """``nans``: (request, token, kv-head, channel) of V.  Returns which elements of out [T, H_q, D] see one."""
    G, row0 = c.H_q // c.H_kv, 0
    hit = torch.zeros(c.out.shape, dtype=torch.bool, device="cuda")
    rows = torch.tensor([0] + c.new).cumsum(0).tolist()
    for i, (r, token, h, ch) in enumerate(nans):
        c.v8.view(torch.uint8)[int(c.table[r, token // 16]), h, token % 16, ch] = NANS[i % 2]
        seen = max(token - (c.total[r] - c.new[r]), 0)               # the first row that sees it
        hit[rows[r] + seen:rows[r + 1], h * G:(h + 1) * G, ch] = True
    return hit


@pytest.mark.parametrize("new,past,H_kv,G,D,absent,nans", [
    ([1], [0], 1, 1, 64, 0.0, [(0, 0, 0, 5)]),
    ([1], [2047], 2, 4, 64, 0.0, [(0, 0, 0, 0), (0, 2047, 1, 63), (0, 1000, 1, 17)]),        # one token, many CTAs
    ([200], [300], 2, 4, 128, 0.0, [(0, 310, 0, 7), (0, 499, 0, 127), (0, 300, 1, 64), (0, 5, 1, 3)]),   # rows of a tile that see it, and not
    ([129, 400], [640, 31], 1, 3, 64, 0.0, [(0, 700, 0, 9), (1, 31, 0, 40), (1, 430, 0, 41)]),
    ([300, 1, 77], [1000, 5000, 0], 4, 7, 128, 0.0, [(0, 999, 3, 1), (0, 1299, 2, 2), (1, 4999, 0, 0), (2, 40, 1, 99), (2, 76, 1, 98)]),
    ([3, 40], [20000, 30001], 2, 5, 128, 0.0, [(0, 100, 0, 11), (0, 20001, 1, 12), (1, 15000, 1, 13), (1, 30040, 0, 14)]),   # parts of many CTAs
    ([64] * 100, [33] * 100, 1, 2, 64, 0.0, [(r, 33 + r % 64, 0, r % 64) for r in range(0, 100, 3)]),
    ([2000], [3001], 2, 4, 128, 0.0, [(0, 3001 + 37 * i, i % 2, 5 * i % 128) for i in range(50)]),
    ([5] * 40, [40 * i for i in range(40)], 2, 8, 128, 0.0, [(r, 40 * r + r % 5, r % 2, 3 * r) for r in range(0, 40, 2)]),  # many short pieces
])
def test_chunk_over_nan_codes_of_v(new, past, H_kv, G, D, absent, nans):
    c = Chunk(51, new, past, H_kv, G, D, absent)
    zeroed = c.v8.view(torch.uint8)
    for r, token, h, ch in nans:
        zeroed[int(c.table[r, token // 16]), h, token % 16, ch] = 0
    c.run()
    want, want_lse = c.out.clone(), c.lse.clone()
    assert bool(want.isfinite().all())
    hit = plant(c, nans)
    for _ in range(2):
        c.out.fill_(7.0)
        c.run()
        assert binding.se_last_device_status(c.ws) == 0
        assert bool(c.out[hit].isnan().all())
        assert torch.equal(c.out[~hit], want[~hit]) and torch.equal(c.lse, want_lse)
    for r, token, h, ch in nans:                                     # and nothing of it stays behind
        zeroed[int(c.table[r, token // 16]), h, token % 16, ch] = 0
    c.run()
    assert torch.equal(c.out, want)


def test_chunk_leaves_nan_codes_of_absent_pages_out():
    c = Chunk(52, [50], [700], 2, 4, 128)
    page = int(c.table[0, 7])
    c.table[0, 7] = -1
    c.run()
    want = c.out.clone()
    c.v8.view(torch.uint8)[page] = 0x7f
    c.run()
    assert torch.equal(c.out, want) and bool(want.isfinite().all())


@pytest.mark.parametrize("D", [64, 128])
def test_chunk_reads_every_code_of_v(D):
    """One token per request and a context of itself: its output is V, whatever the code; scales at both ends and between."""
    n = 256 // D * 8
    c = Chunk(53, [1] * n, [0] * n, 1, 1, D)
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(256 // D, D)
    for r in range(n):
        pid = int(c.table[r, 0])
        c.v8.view(torch.uint8)[pid, 0, 0] = codes[r % (256 // D)]
        c.scales[pid, 0, 1] = 2.0 ** (-64, -60, -20, -3, 0, 1, 6, 7)[r // (256 // D)]
    c.run()
    pages = c.table[:, 0].long()
    want = (c.v8[pages, 0, 0].double() * c.scales[pages, 0, 1].double()[:, None]).to(torch.bfloat16)[:, None]
    assert int(want.isnan().sum()) == 16 and torch.equal(c.out.isnan(), want.isnan())
    assert torch.equal(c.out.nan_to_num(1.0), want.nan_to_num(1.0))


def test_chunk_over_nan_codes_of_k():
    c = Chunk(54, [200], [300], 2, 4, 128)
    at = (int(c.table[0, 350 // 16]), 1, 350 % 16, 20)
    c.k8.view(torch.uint8)[at] = 0
    c.run()
    want, want_lse = c.out.clone(), c.lse.clone()
    c.k8.view(torch.uint8)[at] = 0x7f
    c.run()
    bad = torch.zeros(c.lse.shape, dtype=torch.bool, device="cuda")
    bad[50:, 4:] = True
    assert bool(c.out[bad].isnan().all()) and bool(c.lse[bad].isnan().all())
    assert torch.equal(c.out[~bad], want[~bad]) and torch.equal(c.lse[~bad], want_lse[~bad])


@pytest.mark.parametrize("H_kv,G,D", [(2, 4, 128), (1, 7, 64)])
def test_decode_over_nan_codes(H_kv, G, D):
    d = Decode(55, [5000, 40], H_kv, G, D)
    for r, token, h, ch, cache in ((0, 4321, H_kv - 1, 9, d.v8), (0, 17, 0, D - 1, d.v8), (1, 39, 0, 2, d.k8)):
        cache.view(torch.uint8)[int(d.table[r, token // 16]), h, token % 16, ch] = 0
    d.run()
    want, want_lse = d.out.clone(), d.lse.clone()
    hit, hit_lse = torch.zeros_like(want, dtype=torch.bool), torch.zeros_like(want_lse, dtype=torch.bool)
    for r, token, h, ch, cache in ((0, 4321, H_kv - 1, 9, d.v8), (0, 17, 0, D - 1, d.v8), (1, 39, 0, 2, d.k8)):
        cache.view(torch.uint8)[int(d.table[r, token // 16]), h, token % 16, ch] = 0xff
        heads = slice(h * G, (h + 1) * G)
        if cache is d.v8:
            hit[r, heads, ch] = True
        else:
            hit[r, heads], hit_lse[r, heads] = True, True
    d.run()
    assert bool(d.out[hit].isnan().all()) and torch.equal(d.out[~hit], want[~hit])
    assert bool(d.lse[hit_lse].isnan().all()) and torch.equal(d.lse[~hit_lse], want_lse[~hit_lse])


@pytest.mark.parametrize("H_q,H_kv,D", [(8, 2, 128), (3, 1, 64)])
def test_appended_nans_and_infinities_reach_the_rows_that_see_them(H_q, H_kv, D):
    """K and V with a NaN and infinities, through append: codes as described, summaries of the numbers among them, both attentions."""
    g = torch.Generator().manual_seed(56)
    new, G = [90, 33], H_q // H_kv
    table, P = page_tables(g, new)
    qkv = torch.randn(sum(new), H_q + 2 * H_kv, D, generator=g).to(torch.bfloat16).cuda()
    q, k, v = qkv.split([H_q, H_kv, H_kv], dim=1)
    p = binding.make_params(2, H_q, H_kv, D, table.shape[1], P, 1)
    ws, table = binding.alloc_prompt_workspace(p), table.cuda()
    cu, seq = torch.tensor([0, 90, 123], **I32), torch.tensor(new, **I32)
    freq, axis = torch.zeros(8, dtype=torch.float64, device="cuda"), torch.zeros(8, **I32)
    pos = torch.zeros(1, 123, **I32)

    def run():
        k8, v8 = (torch.zeros(P, H_kv, 16, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
        scales, meta = torch.ones(P, H_kv, 2, device="cuda"), torch.zeros(P, H_kv, 2, D, dtype=torch.bfloat16, device="cuda")
        qr, out = (torch.empty(123, H_q, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lse = torch.empty(123, H_q, device="cuda")
        binding.se_kv8_append(p, q, k, v, cu, seq, table, pos, freq, axis, qr, k8, v8, scales, ws, meta=meta)
        binding.se_kv8_chunk_attend(p, qr, cu, k8, v8, scales, table, seq, out, ws, lse=lse)
        last = qr[torch.tensor([89, 122], device="cuda")].contiguous()
        dout, dlse = torch.empty(2, H_q, D, device="cuda"), torch.empty(2, H_q, device="cuda")
        binding.se_kv8_decode(p, last, k8, v8, scales, table, seq, dout, dlse, ws)
        assert binding.se_last_device_status(ws) == 0
        return k8, v8, scales, meta, out, lse, dout, dlse

    h = H_kv - 1
    v[50, h, 3], k[110, 0, 20] = 0.0, 0.0                             # request 0 token 50, request 1 token 20
    clean = run()
    v[50, h, 3], k[110, 0, 20] = float("nan"), float("nan")
    k8, v8, scales, meta, out, lse, dout, dlse = run()
    at_v, at_k = (int(table[0, 3]), h, 2, 3), (int(table[1, 1]), 0, 4, 20)
    assert bool(v8[at_v].float().isnan()) and bool(k8[at_k].float().isnan()) and torch.equal(scales, clean[2])
    others = k8.view(torch.uint8) != clean[0].view(torch.uint8)
    assert int(others.sum()) == 1 and int((v8.view(torch.uint8) != clean[1].view(torch.uint8)).sum()) == 1
    x = (k8.double() * scales[..., 0].double()[..., None, None])[int(table[1, 1]), 0]
    least, most = meta[int(table[1, 1]), 0, :, 20].double()
    assert least == x[:, 20].nan_to_num(math.inf).amin() and most == x[:, 20].nan_to_num(-math.inf).amax()
    bad, bad_lse = torch.zeros_like(out, dtype=torch.bool), torch.zeros_like(lse, dtype=torch.bool)
    bad[50:90, h * G:(h + 1) * G, 3] = True
    bad[110:, :G], bad_lse[110:, :G] = True, True
    assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], clean[4][~bad])
    assert bool(lse[bad_lse].isnan().all()) and torch.equal(lse[~bad_lse], clean[5][~bad_lse])
    bad, bad_lse = torch.zeros_like(dout, dtype=torch.bool), torch.zeros_like(dlse, dtype=torch.bool)
    bad[0, h * G:(h + 1) * G, 3] = True
    bad[1, :G], bad_lse[1, :G] = True, True
    assert bool(dout[bad].isnan().all()) and torch.equal(dout[~bad], clean[6][~bad])
    assert bool(dlse[bad_lse].isnan().all()) and torch.equal(dlse[~bad_lse], clean[7][~bad_lse])
    # infinities become the largest code of the largest scale
    v[50, h, 3], k[110, 0, 20] = float("inf"), -float("inf")
    k8, v8, scales = run()[:3]
    assert float(v8[at_v]) == 448.0 and float(k8[at_k]) == -448.0
    assert float(scales[at_v[0], h, 1]) == 128.0 and float(scales[at_k[0], 0, 0]) == 128.0
    assert int(v8.float().isnan().sum()) == 0 and int(k8.float().isnan().sum()) == 0
