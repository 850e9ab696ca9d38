"""The 8-bit cache and the page pool together, as a serving loop uses them: a prompt enters in chunks, is forked into beams, the
beams go on with tokens of their own over shared pages, one ends, the pool is compacted, decoding goes on."""
import os
import subprocess
import sys

import pytest
import torch

import kv8_ref as ref
import pages_ref
import prompt_ref
from paper_2609_39068_b200 import binding

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


class Engine:
    """B slots over one pool of an 8-bit cache."""

    def __init__(self, B, H_q, H_kv, D, P, max_pages, seed):
        self.B, self.H_q, self.H_kv, self.D = B, H_q, H_kv, D
        self.p = binding.make_params(B, H_q, H_kv, D, max_pages, P, max_pages)
        self.ws, self.sws, self.pws = binding.alloc_prompt_workspace(self.p), binding.alloc_workspace(self.p), binding.alloc_pages_workspace(self.p)
        # a pool that others have used: NaN codes and scales everywhere
        self.k8, self.v8 = (torch.full((P, H_kv, 16, D), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
        self.scales = torch.full((P, H_kv, 2), float("nan"), device="cuda")
        self.meta = torch.full((P, H_kv, 2, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.buffers = binding.page_buffers([self.k8, self.v8, self.scales, self.meta])
        self.table, self.lens, self.refs = torch.full((B, max_pages), -1, **I32), torch.zeros(B, **I32), torch.zeros(P, **I32)
        self.free = torch.zeros(1, **I32)
        self.g = torch.Generator().manual_seed(seed)
        self.freq = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device="cuda") * 2 / D)
        self.axis = torch.zeros(D // 2, **I32)

    def update(self, new_lens, parent=None):
        want = pages_ref.update(self.table.tolist(), self.lens.tolist(), self.refs.tolist(), new_lens, parent)
        outs = [torch.empty_like(t) for t in (self.table, self.lens, self.refs)]
        binding.se_pages_update(self.p, self.table, self.lens, self.refs, torch.tensor(new_lens, **I32), *outs, self.free, self.pws,
                                parent=None if parent is None else torch.tensor(parent, **I32), buffers=self.buffers)
        self.table, self.lens, self.refs = outs
        assert self.table.tolist() == want[0] and self.refs.tolist() == want[2] and self.free.tolist() == [want[3]]
        return len(want[4])

    def append(self, new):
        """``new`` tokens of each slot; the pages and lengths are in place.  Returns the rotated q and their offsets."""
        T = sum(new)
        qkv = torch.randn(T, self.H_q + 2 * self.H_kv, self.D, generator=self.g).to(torch.bfloat16).cuda()
        cu = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), **I32)
        total = self.lens.tolist()
        pos = torch.cat([torch.arange(t - n, t) for n, t in zip(new, total)]).to(torch.int32).cuda()[None].contiguous()
        q, k = (torch.empty(T, h, self.D, dtype=torch.bfloat16, device="cuda") for h in (self.H_q, self.H_kv))
        before = [t.clone() for t in (self.k8, self.v8, self.scales, self.meta)]
        binding.se_kv8_append(self.p, *qkv.split([self.H_q, self.H_kv, self.H_kv], dim=1), cu, self.lens, self.table, pos, self.freq, self.axis,
                              q, self.k8, self.v8, self.scales, self.ws, meta=self.meta, k_out=k)
        want = ref.append(*before, k, qkv[:, self.H_q + self.H_kv:], new, total, self.table.cpu())
        for got, x in zip((self.k8, self.v8, self.scales, self.meta), want):
            assert torch.equal(got.double().nan_to_num(7e7), x.nan_to_num(7e7))
        return q, cu

    def chunk(self, q, cu, new):
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        binding.se_kv8_chunk_attend(self.p, q, cu, self.k8, self.v8, self.scales, self.table, self.lens, out, self.ws, lse=lse)
        k16, v16 = (ref.values(c, self.scales[..., i]).nan_to_num(0.0).to(torch.bfloat16) for c, i in ((self.k8, 0), (self.v8, 1)))
        b = prompt_ref.Batch(self.H_q, self.H_kv, self.D, new, self.lens.tolist(), q.shape[0], self.p.max_pages, self.p.num_phys_pages, q, cu,
                             self.lens, self.table, k16, v16)
        want, tol, want_lse, ltol = ref.chunk(b, self.D ** -0.5)
        assert bool(((out.double() - want).abs() <= tol).all()) and bool(((lse.double() - want_lse).abs() <= ltol).all())

    def decode(self, q, budget=None):
        """One token per slot; budget: over the pages that se_page_select finds in the summaries."""
        out, lse = torch.empty(self.B, self.H_q, self.D, device="cuda"), torch.empty(self.B, self.H_q, device="cuda")
        sel = cnt = None
        if budget:
            sel, cnt = torch.empty(self.B, self.H_kv, self.p.k_max, **I32), torch.empty(self.B, self.H_kv, **I32)
            binding.se_page_select(self.p, q, self.meta, self.table, self.lens, budget, sel, cnt, self.sws)
            assert int(cnt.max()) == budget // 16
        binding.se_kv8_decode(self.p, q, self.k8, self.v8, self.scales, self.table, self.lens, out, lse, self.ws, sel_idx=sel, sel_cnt=cnt)
        want, tol, want_lse, ltol = ref.decode(q, self.k8, self.v8, self.scales, self.table, self.lens, sel, cnt, self.D ** -0.5)
        assert bool(((out.double() - want).abs() <= tol).all())
        assert bool(((lse.double() == want_lse) | ((lse.double() - want_lse).abs() <= ltol)).all())
        return out, lse

    def clean(self):
        assert [binding.se_last_device_status(w) for w in (self.ws, self.sws, self.pws)] == [0, 0, 0]


@pytest.mark.parametrize("H_q,H_kv,D", [(8, 2, 128), (7, 1, 64)])
def test_prompt_beams_and_a_compacted_pool(H_q, H_kv, D):
    e = Engine(4, H_q, H_kv, D, 80, 24, 31)
    for length, new in ((181, [181, 0, 0, 0]), (300, [119, 0, 0, 90])):      # two chunks of one prompt, another prompt beside the second
        e.update([length, 0, 0, new[3]])
        q, cu = e.append(new)
        e.chunk(q, cu, new)
    assert e.update([301, 301, 301, 91], [0, 0, 0, 3]) == 2                  # three beams: 18 shared pages, two copies of the last
    q, _ = e.append([1, 1, 1, 1])
    assert bool((e.meta[e.table[0, 18]] != e.meta[e.table[1, 18]]).any())    # their last pages have parted
    e.decode(q)
    e.decode(q, budget=64)
    e.update([302, 302, 0, 92], [1, 2, -1, 3])                              # two beams go on from the last two, the third slot is free
    q, _ = e.append([1, 1, 0, 1])
    q = torch.cat([q[:2], torch.zeros_like(q[:1]), q[2:]])
    before = e.decode(q)
    assert bool((before[0][2] == 0).all()) and bool(torch.isinf(before[1][2]).all())
    where, live, table, refs = torch.empty_like(e.refs), torch.zeros(1, **I32), torch.empty_like(e.table), torch.empty_like(e.refs)
    binding.se_pages_compact(e.p, e.table, e.lens, e.refs, table, refs, where, live, e.pws, buffers=e.buffers)
    assert int(live) == int((e.refs > 0).sum()) and bool((refs[:int(live)] > 0).all()) and int(table.max()) < int(live)
    e.table, e.refs = table, refs
    after = e.decode(q)
    assert all(torch.equal(x, y) for x, y in zip(before, after))             # the same pages elsewhere
    e.decode(q, budget=48)
    e.clean()


def test_two_streams_and_a_replayed_step():
    """Two engines on two streams at once, a step captured and replayed on each."""
    engines, want, graphs = [], [], []
    for i in range(2):
        e = Engine(3, 8, 2, 128, 400, 120, 41 + i)
        e.update([1500, 700, 1])
        q, _ = e.append([1500, 700, 1])
        e.q = q[torch.tensor([1499, 2199, 2200], device="cuda")].contiguous()
        engines.append(e)
        want.append(e.decode(e.q))
    torch.cuda.synchronize()
    for e in engines:
        e.stream = torch.cuda.Stream()
        e.out, e.lse, e.new = torch.empty_like(want[0][0]), torch.empty_like(want[0][1]), e.lens.clone()
        e.outs = [torch.empty_like(t) for t in (e.table, e.lens, e.refs)]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=e.stream):
            binding.se_pages_update(e.p, e.table, e.lens, e.refs, e.new, *e.outs, e.free, e.pws, buffers=e.buffers)
            binding.se_kv8_decode(e.p, e.q, e.k8, e.v8, e.scales, e.outs[0], e.outs[1], e.out, e.lse, e.ws)
        graphs.append(g)
    for _ in range(20):
        for e, g in zip(engines, graphs):
            with torch.cuda.stream(e.stream):
                g.replay()
    torch.cuda.synchronize()
    for e, (out, lse) in zip(engines, want):
        assert torch.equal(e.out, out) and torch.equal(e.lse, lse) and torch.equal(e.outs[0], e.table)
        e.clean()


FIRST_CALLS = """
import torch
from paper_2609_39068_b200 import binding
i32 = dict(dtype=torch.int32, device="cuda")
B, H_q, H_kv, D, P, mp = 2, 8, 2, 128, 20, 6
p = binding.make_params(B, H_q, H_kv, D, mp, P, 1)
ws, pws = binding.alloc_prompt_workspace(p), binding.alloc_pages_workspace(p)
k8, v8 = (torch.zeros(P, H_kv, 16, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
scales, table, lens, refs, free = torch.zeros(P, H_kv, 2, device="cuda"), torch.full((B, mp), -1, **i32), torch.zeros(B, **i32), torch.zeros(P, **i32), torch.zeros(1, **i32)
new, qkv = torch.tensor([40, 7], **i32), torch.ones(47, H_q + 2 * H_kv, D, device="cuda").to(torch.bfloat16)
q, k, v = qkv.split([H_q, H_kv, H_kv], dim=1)
cu, pos = torch.tensor([0, 40, 47], **i32), torch.zeros(1, 47, **i32)
freq, axis = torch.ones(64, dtype=torch.float64, device="cuda"), torch.zeros(64, **i32)
qr, out = (torch.zeros(47, H_q, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
dout, lse = torch.zeros(B, H_q, D, device="cuda"), torch.zeros(B, H_q, device="cuda")
q1 = torch.ones(B, H_q, D, device="cuda").to(torch.bfloat16)
buffers, where = binding.page_buffers([k8, v8, scales]), torch.zeros(P, **i32)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    binding.se_pages_update(p, table, lens, refs, new, table, lens, refs, free, pws, buffers=buffers)
    binding.se_kv8_append(p, q, k, v, cu, lens, table, pos, freq, axis, qr, k8, v8, scales, ws)
    binding.se_kv8_chunk_attend(p, qr, cu, k8, v8, scales, table, lens, out, ws)
    binding.se_kv8_decode(p, q1, k8, v8, scales, table, lens, dout, lse, ws)
    binding.se_pages_compact(p, table, lens, refs, table, refs, where, free, pws, buffers=buffers)
g.replay()
torch.cuda.synchronize()
assert bool((out == 1).all()) and bool((dout == 1).all()) and lens.tolist() == [40, 7] and free.tolist() == [4]
assert binding.se_last_device_status(ws) == 0 and binding.se_last_device_status(pws) == 0
"""


def test_the_first_calls_of_a_process_may_be_captured():
    here = os.path.dirname(os.path.abspath(__file__))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([here, os.path.dirname(here)]))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
