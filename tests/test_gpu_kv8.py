"""The 8-bit cache on the GPU: append and decode against the restatements of kv8_ref.py."""
import math

import pytest
import torch

import kv8_ref as ref
import prompt_ref
from paper_2609_39068_b200 import binding

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
I32 = dict(dtype=torch.int32, device="cuda")


def page_tables(g, total, extra=2, wide=0):
    """Pages of all requests dealt from one permuted pool."""
    pages = [(t + 15) // 16 for t in total]
    P, width = sum(pages) + extra, max(pages + [1]) + wide
    order, at = torch.randperm(P, generator=g), 0
    table = torch.full((len(total), width), -1, dtype=torch.int32)
    for r, n in enumerate(pages):
        table[r, :n] = order[at:at + n].to(torch.int32)
        at += n
    return table, P


# ---- append ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("H_q,H_kv,D,new,past,rot,interleaved,spare", [
    (8, 2, 64, [1, 1, 1], [0, 5, 31], 64, False, 0),               # single tokens: a fresh page, the middle and the end of one
    (8, 2, 128, [1, 40, 0, 17], [15, 3, 8, 16], 128, False, 3),    # ends inside pages, an idle request, spare rows
    (7, 1, 128, [33, 2], [0, 14], 64, True, 0),                    # heads in groups of seven, part of the head, interleaved
    (4, 4, 64, [100], [60], 32, False, 0),
    (8, 8, 128, [3] * 40, list(range(40)), 128, True, 0),
    (32, 8, 128, [700, 333], [5, 100], 128, False, 0),             # CTAs begin and end inside a page's heads
    (2, 1, 64, [1] * 1500, [i % 40 for i in range(1500)], 64, False, 0),   # more requests than threads
])
def test_append(H_q, H_kv, D, new, past, rot, interleaved, spare):
    g = torch.Generator().manual_seed(7)
    total = [n + o for n, o in zip(new, past)]
    T = sum(new) + spare
    table, P = page_tables(g, total)
    k8, v8, scales = ref.make_cache(g, P, H_kv, D, "cuda")
    qkv = torch.randn(T, H_q + 2 * H_kv, D, generator=g) * torch.exp2(torch.randint(-8, 8, (T, 1, 1), generator=g).float())
    qkv = qkv.to(torch.bfloat16).cuda()
    q, k, v = qkv.split([H_q, H_kv, H_kv], dim=1)
    cu = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), **I32)
    seq = torch.tensor(total, **I32)
    pos = torch.zeros(1, T, **I32)
    pos[0, :sum(new)] = torch.cat([torch.arange(o, o + n) for n, o in zip(new, past)])
    freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device="cuda") * 2 / rot)
    axis = torch.zeros(rot // 2, **I32)
    p = binding.make_params(len(new), H_q, H_kv, D, table.shape[1], P, 1)
    ws = binding.alloc_prompt_workspace(p)
    table = table.cuda()
    meta = torch.zeros(P, H_kv, 2, D, dtype=torch.bfloat16, device="cuda")
    q_out, k_out = torch.zeros(T, H_q, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, H_kv, D, dtype=torch.bfloat16, device="cuda")
    k_new, v_new, s_new, m_new = k8.clone(), v8.clone(), scales.clone(), meta.clone()
    binding.se_kv8_append(p, q, k, v, cu, seq, table, pos, freq, axis, q_out, k_new, v_new, s_new, ws, meta=m_new, k_out=k_out,
                          interleaved=interleaved)
    assert binding.se_last_device_status(ws) == 0
    # the rotation is that of the bf16 cache, bit for bit
    q_ref, k_ref = torch.zeros_like(q_out), torch.zeros_like(k_out)
    kc, vc = (torch.zeros(P, H_kv, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.se_rope_append(p, q, k, v, cu, seq, table, pos, freq, axis, q_ref, kc, vc, ws, k_out=k_ref, interleaved=interleaved)
    assert torch.equal(q_out.view(torch.int16), q_ref.view(torch.int16)) and torch.equal(k_out.view(torch.int16), k_ref.view(torch.int16))
    kk, vv, ss, mm = ref.append(k8, v8, scales, meta, k_out, v, new, total, table.cpu())
    assert torch.equal(s_new.double(), ss)
    assert torch.equal(k_new.double(), kk)
    assert torch.equal(v_new.double(), vv)
    assert torch.equal(m_new.double(), mm)
    # a second time the same, and the same without summaries
    binding.se_kv8_append(p, q, k, v, cu, seq, table, pos, freq, axis, q_out, k_new, v_new, s_new, ws, interleaved=interleaved)
    assert torch.equal(k_new.double(), kk) and torch.equal(v_new.double(), vv) and torch.equal(s_new.double(), ss)


def test_append_rounding_and_range():
    """Every code, ties, subnormals, values that saturate, zeros; pages filled slot by slot with growing magnitudes."""
    H, D, P = 1, 64, 4
    codes = torch.arange(0, 256, dtype=torch.uint8).view(E4M3).float()
    codes = codes[codes.isfinite()]
    mids = (codes.sort()[0][1:] + codes.sort()[0][:-1]) / 2
    pool = torch.cat([codes, mids, mids * 1.0078125]).to(torch.bfloat16).float()
    rows = [pool[torch.randint(pool.numel(), (D,), generator=torch.Generator().manual_seed(i))] * 2.0 ** e
            for i, e in enumerate([-30, -30, -9, -8, -1, 0, 0, 1, 3, 4, 4, 5, 6, 7, 8, 20])]
    rows[0][:] = 0.0
    rows[1][:] = 2.0 ** -100
    rows = torch.stack(rows).to(torch.bfloat16).cuda()             # 16 tokens: one page, one after the other
    p = binding.make_params(1, 1, H, D, 1, P, 1)
    ws = binding.alloc_prompt_workspace(p)
    k8, v8 = (torch.full((P, H, 16, D), 0x7f, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    scales = torch.full((P, H, 2), float("nan"), device="cuda")
    table, freq, axis = torch.tensor([[2]], **I32), torch.zeros(8, dtype=torch.float64, device="cuda"), torch.zeros(8, **I32)
    kc, sc = torch.zeros(H, 16, D, dtype=torch.float64, device="cuda"), torch.zeros(H, dtype=torch.float64, device="cuda")
    q_out = torch.zeros(1, 1, D, dtype=torch.bfloat16, device="cuda")
    for i in range(16):
        x = rows[i:i + 1, None]
        binding.se_kv8_append(p, x.clone(), x, -x, torch.tensor([0, 1], **I32), torch.tensor([i + 1], **I32), table,
                              torch.zeros(1, 1, **I32), freq, axis, q_out, k8, v8, scales, ws)
        kc, sc = ref.append_rows(kc, sc, x, i > 0, i, i + 1)
        assert torch.equal(scales[2].double(), sc[:, None].expand(H, 2))
        assert torch.equal(k8[2].double()[:, :i + 1], kc[:, :i + 1]) and torch.equal(v8[2].double()[:, :i + 1], -kc[:, :i + 1])
    assert float(sc[0]) == 128.0 and float(kc[0, 15].abs().max()) == 448.0
    others = torch.tensor([0, 1, 3], device="cuda")
    assert bool((k8[others].view(torch.uint8) == 0x7f).all()) and bool(scales[others].isnan().all())


# ---- decode ---------------------------------------------------------------------------------------

class Decode:
    def __init__(self, seed, lens, H_kv, G, D, absent=0.0, k_max=1, sm_scale=0.0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.H_kv, self.D, self.lens = len(lens), H_kv, D, lens
        self.H_q = H_kv * G
        table, P = page_tables(g, lens, wide=1)
        self.k8, self.v8, self.scales = ref.make_cache(g, P, H_kv, D, "cuda")
        # what lies behind a request's end is never read into a result
        for r, n in enumerate(lens):
            if n % 16:
                pid = int(table[r, n // 16])
                for c in (self.k8, self.v8):
                    c.view(torch.uint8)[pid, :, n % 16:] = 0x7f
        if absent:
            table[torch.rand(table.shape, generator=g) < absent] = -1
        self.table, self.seq = table.cuda(), torch.tensor(lens, **I32)
        self.q = torch.randn(self.B, self.H_q, D, generator=g).to(torch.bfloat16).cuda()
        self.p = binding.make_params(self.B, self.H_q, H_kv, D, table.shape[1], P, k_max, sm_scale=sm_scale)
        self.scale = sm_scale or D ** -0.5
        self.ws = binding.alloc_prompt_workspace(self.p)
        self.out = torch.full((self.B, self.H_q, D), float("nan"), device="cuda")
        self.lse = torch.full((self.B, self.H_q), float("nan"), device="cuda")
        self.sel = (None, None)

    def select(self, seed, most):
        """For every head a draw of the request's pages, ascending; some heads get none."""
        g = torch.Generator().manual_seed(seed)
        idx = torch.full((self.B, self.H_kv, self.p.k_max), -1, dtype=torch.int32)
        cnt = torch.zeros(self.B, self.H_kv, dtype=torch.int32)
        for r, n in enumerate(self.lens):
            for h in range(self.H_kv):
                m = int(torch.randint(0, min(most, (n + 15) // 16) + 1, (1,), generator=g))
                idx[r, h, :m] = torch.randperm((n + 15) // 16, generator=g)[:m].sort()[0].to(torch.int32)
                cnt[r, h] = m
        self.sel = (idx.cuda(), cnt.cuda())

    def run(self):
        binding.se_kv8_decode(self.p, self.q, self.k8, self.v8, self.scales, self.table, self.seq, self.out, self.lse, self.ws,
                              sel_idx=self.sel[0], sel_cnt=self.sel[1])

    def check(self, status=0):
        self.run()
        assert binding.se_last_device_status(self.ws) == status
        sel = [None if t is None else t.cpu() for t in self.sel]
        out, tol, lse, ltol = ref.decode(self.q.cpu(), self.k8.cpu(), self.v8.cpu(), self.scales.cpu(), self.table.cpu(), self.seq.cpu(),
                                         sel[0], sel[1], self.scale)
        got, gl = self.out.cpu().double(), self.lse.cpu().double()
        assert bool(((got - out).abs() <= tol).all()), float(((got - out).abs() - tol).max())
        same = torch.isinf(lse) & (gl == lse)
        assert bool((same | ((gl - lse).abs() <= ltol)).all())
        first = self.out.clone(), self.lse.clone()
        self.out.fill_(float("nan")), self.lse.fill_(float("nan"))
        self.run()                                                  # equal inputs, equal bits
        assert torch.equal(self.out.view(torch.int32), first[0].view(torch.int32)) and torch.equal(self.lse.view(torch.int32), first[1].view(torch.int32))


@pytest.mark.parametrize("lens,H_kv,G,D,absent", [
    ([1], 1, 1, 64, 0.0),
    ([1], 1, 8, 128, 0.0),
    ([16, 17, 0, 15], 2, 4, 64, 0.0),                              # a page exactly, one token more, nothing, one less
    ([2048], 2, 4, 64, 0.0),                                       # one pair over many CTAs
    ([3000, 1, 700, 2047], 4, 7, 128, 0.1),
    ([9000], 1, 8, 128, 0.5),
    ([40, 33], 8, 5, 128, 1.0),                                    # every page absent
    (list(range(1, 120)), 3, 2, 64, 0.0),                          # more pairs than CTAs
    ([65536], 1, 3, 64, 0.1),                                      # one pair over all runs, merged in groups
    ([3900, 4000, 90, 4090, 0, 12000], 1, 8, 128, 0.0),            # pairs of 30 to 32 runs and more, which begin and end inside groups
    ([20000, 50000], 2, 7, 64, 0.3),
    ([64] * 700, 4, 1, 128, 0.05),                                 # more pairs than prefix sums
    ([i % 50 for i in range(8192)], 1, 1, 64, 0.0),                # the largest batch
])
def test_decode_dense(lens, H_kv, G, D, absent):
    Decode(3, lens, H_kv, G, D, absent).check()


@pytest.mark.parametrize("lens,H_kv,G,D,most,absent", [
    ([5000, 300, 0, 16], 2, 4, 128, 64, 0.0),
    ([5000] * 9, 8, 3, 64, 17, 0.2),
    ([100] * 600, 4, 8, 64, 3, 0.0),                               # more pairs than prefix sums, many of them empty
])
def test_decode_selected(lens, H_kv, G, D, most, absent):
    d = Decode(5, lens, H_kv, G, D, absent, k_max=most)
    d.select(6, most)
    d.check()


def test_decode_magnitudes():
    """Large and tiny logits, a far maximum late in the context, scales at both ends of their range."""
    d = Decode(9, [1500, 800], 2, 4, 128, sm_scale=0.5)
    d.q[0] *= 20
    d.q[1] *= 2.0 ** -100
    d.scales[..., 1] = torch.exp2(torch.randint(-60, 8, d.scales.shape[:2], device="cuda").float())
    d.check()
    d.q.zero_()
    d.check()


@pytest.mark.parametrize("length,gap", [(131000, 18.0), (131000, 22.0), (4000, 13.0)])
def test_decode_of_one_large_weight_and_many_small_ones(length, gap):
    """A first token that takes nearly all the weight and whose V is zero: the output is what the many others add up to."""
    d = Decode(15, [length], 1, 2, 64)
    codes = lambda x: torch.tensor(x).to(E4M3).view(torch.uint8).cuda()  # noqa: E731
    d.q.fill_(1.0), d.scales.fill_(1.0)
    d.k8.view(torch.uint8).fill_(0), d.v8.view(torch.uint8).fill_(codes(1.0))
    first = int(d.table[0, 0])
    d.k8.view(torch.uint8)[first, :, 0] = codes(gap / 8)            # 64 of them, over the square root of 64
    d.v8.view(torch.uint8)[first, :, 0] = 0
    d.check()
    rest = (length - 1) * math.exp(-gap)
    assert float((d.out.double() - rest / (1 + rest)).abs().max()) <= length * 2.0 ** -37 + 2.0 ** -14 * rest


def test_decode_reports():
    d = Decode(11, [500, 90], 2, 4, 128, k_max=8)
    d.select(12, 8)
    d.sel[0][0, 0, :3] = torch.tensor([2, 31, 99999], dtype=torch.int32)      # 31: the last page; beyond the table
    d.sel[1][0, 0] = 3
    d.sel[0][1, 1, :2] = torch.tensor([-5, 6], dtype=torch.int32)             # 6: behind the request's end
    d.sel[1][1, 1] = 2
    d.run()
    assert binding.se_last_device_status(d.ws) == binding.SE_DEV_BAD_SELECTION
    assert bool((d.out[1, 4:] == 0).all()) and bool(torch.isinf(d.lse[1, 4:]).all()) and bool(torch.isfinite(d.out).all())
    e = Decode(13, [500, 90], 2, 4, 128)
    e.table[0, 3] = e.p.num_phys_pages
    e.run()
    assert binding.se_last_device_status(e.ws) == binding.SE_DEV_BAD_PAGE_ID
    e.table[0, 3] = -1
    e.check()
    e.seq[1] = 16 * e.p.max_pages + 1
    e.run()
    assert binding.se_last_device_status(e.ws) == binding.SE_DEV_BAD_LENGTH
    assert bool((e.out[1] == 0).all()) and bool(torch.isfinite(e.out[0]).all())


# ---- chunk ----------------------------------------------------------------------------------------

class Chunk:
    """Packed new tokens over an 8-bit cache."""

    def __init__(self, seed, new, past, H_kv, G, D, absent=0.0, spare=0, sm_scale=0.0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.total = new, [n + o for n, o in zip(new, past)]
        table, P = page_tables(g, self.total, wide=1)
        self.k8, self.v8, self.scales = ref.make_cache(g, P, H_kv, D, "cuda")
        for c, i in ((self.k8, 0), (self.v8, 1)):
            c.view(torch.uint8)[table[0, 0]] = torch.randint(0, 8, c.shape[1:], generator=g, dtype=torch.uint8).cuda()   # subnormal codes, largest scale
            self.scales[table[0, 0], :, i] = 128.0
        self.k16 = ref.values(self.k8, self.scales[..., 0]).to(torch.bfloat16)
        self.v16 = ref.values(self.v8, self.scales[..., 1]).to(torch.bfloat16)
        for r, t in enumerate(self.total):                          # what lies behind a request's end is never read into a result
            if t % 16:
                pid = int(table[r, t // 16])
                for c in (self.k8, self.v8):
                    c.view(torch.uint8)[pid, :, t % 16:] = 0x7f
        if absent:
            for r, o in enumerate(past):
                row = table[r, :o // 16]
                row[torch.rand(row.shape, generator=g) < absent] = -1
        T, H_q = sum(new) + spare, H_kv * G
        qkv = torch.randn(T, H_q + 2, D, generator=g).to(torch.bfloat16).cuda()
        self.qkv, self.q = qkv, qkv[:, :H_q]                        # a view of wider rows
        if spare:
            qkv[sum(new):] = float("nan")
        self.table, self.seq = table.cuda(), torch.tensor(self.total, **I32)
        self.cu = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), **I32)
        self.p = binding.make_params(len(new), H_q, H_kv, D, table.shape[1], P, 1, sm_scale=sm_scale)
        self.ws = binding.alloc_prompt_workspace(self.p)
        self.H_q, self.H_kv, self.D, self.scale = H_q, H_kv, D, sm_scale or D ** -0.5
        self.out = torch.full((T, H_q, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((T, H_q), float("nan"), device="cuda")

    def run(self):
        binding.se_kv8_chunk_attend(self.p, self.q, self.cu, self.k8, self.v8, self.scales, self.table, self.seq, self.out, self.ws,
                                    lse=self.lse)

    def check(self):
        self.run()
        assert binding.se_last_device_status(self.ws) == 0
        b = prompt_ref.Batch(self.H_q, self.H_kv, self.D, self.new, self.total, self.q.shape[0], self.p.max_pages, self.p.num_phys_pages,
                             self.qkv, self.cu, self.seq, self.table, self.k16, self.v16)
        out, tol, lse, ltol = ref.chunk(b, self.scale)
        for got, want, t in ((self.lse.double(), lse, ltol), (self.out.double(), out, tol)):
            live = ~want.isnan()
            assert bool(got[~live].isnan().all())                   # spare rows are left as they were
            bad = live & ~(torch.isinf(want) & (got == want)) & ~((got - want).abs() <= t)
            assert not bool(bad.any()), (int(bad.sum()), float(((got - want).abs() / t)[bad].max()))
        first = self.out.clone(), self.lse.clone()
        self.run()                                                  # equal inputs, equal bits
        assert torch.equal(self.out.view(torch.int16), first[0].view(torch.int16)) and torch.equal(self.lse.view(torch.int32), first[1].view(torch.int32))


@pytest.mark.parametrize("new,past,H_kv,G,D,absent,spare", [
    ([1], [0], 1, 1, 64, 0.0, 0),
    ([1], [15], 2, 4, 128, 0.0, 2),
    ([1], [2047], 2, 4, 64, 0.0, 0),                                # one token, many CTAs
    ([5, 0, 1, 17], [100, 50, 16, 0], 2, 8, 128, 0.0, 5),
    ([300, 1, 77], [1000, 5000, 0], 4, 7, 128, 0.3, 0),
    ([129, 400], [640, 31], 1, 3, 64, 0.5, 1),
    ([2000], [3001], 2, 4, 128, 0.0, 0),                            # neighbouring query tiles share K and V
    ([64] * 100, [33] * 100, 1, 2, 64, 0.1, 0),                     # more requests than prefix sums in shared memory
    ([3, 2], [160, 320], 8, 5, 128, 1.0, 0),                        # nothing but the new tokens is present
])
def test_chunk(new, past, H_kv, G, D, absent, spare):
    Chunk(21, new, past, H_kv, G, D, absent, spare).check()


@pytest.mark.parametrize("D", [64, 128])
def test_chunk_of_rows_with_far_elements(D):
    """Rows whose largest element is 2^0 .. 2^14 times the others, zero rows, tiny rows: the split of a row into codes."""
    c = Chunk(22, [90], [700], 2, 4, D, sm_scale=0.01)
    for i in range(15):
        c.q[6 * i:6 * i + 6, :, 5 + i] *= 2.0 ** i
    c.q[80:82] = 0
    c.q[82:84] *= 2.0 ** -90
    c.check()


def test_chunk_rows_that_are_no_numbers_stay_alone():
    c = Chunk(24, [200], [300], 2, 4, 128)
    c.run()
    want = c.out.clone()
    c.q[7, 3, 11] = float("nan")
    c.q[150, 6, 0] = float("inf")
    c.run()
    bad = torch.zeros(c.out.shape[:2], dtype=torch.bool, device="cuda")
    bad[7, 3] = bad[150, 6] = True
    assert bool(c.out[bad].isnan().all()) and bool(c.lse[bad].isnan().all())
    assert torch.equal(c.out[~bad], want[~bad]) and bool(c.lse[~bad].isfinite().all())


def test_chunk_reports():
    c = Chunk(23, [4, 9], [100, 40], 2, 4, 128)
    c.table[0, 2] = c.p.num_phys_pages
    c.run()
    assert binding.se_last_device_status(c.ws) == binding.SE_DEV_BAD_PAGE_ID
    c.table[0, 2] = -1
    c.check()
    c.seq[1] = 3
    c.run()
    assert binding.se_last_device_status(c.ws) == binding.SE_DEV_BAD_LENGTH
