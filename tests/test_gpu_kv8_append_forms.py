"""Forms of se_kv8_append that the bf16 call's tests cover there: several position axes, new tokens whose page is absent, q and k rotated in
place.  The rotation is compared with the bf16 call's, bit for bit, codes and scales with kv8_ref."""
import pytest
import torch

import kv8_ref as ref
from paper_2609_39068_b200 import binding
from test_gpu_kv8 import I32, page_tables

pytestmark = pytest.mark.gpu


class Append:
    def __init__(self, seed, new, past, H_q, H_kv, D, axes=1, rot=None, interleaved=False):
        g = torch.Generator().manual_seed(seed)
        self.new, self.total, self.interleaved = new, [n + o for n, o in zip(new, past)], interleaved
        T, rot = sum(new), rot or D
        table, self.P = page_tables(g, self.total)
        self.table, self.H_q, self.H_kv, self.D = table.cuda(), H_q, H_kv, D
        self.cache = ref.make_cache(g, self.P, H_kv, D, "cuda")
        self.q, self.k, self.v = (torch.randn(T, h, D, generator=g).to(torch.bfloat16).cuda() for h in (H_q, H_kv, H_kv))
        self.cu = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), **I32)
        self.seq = torch.tensor(self.total, **I32)
        self.pos = torch.randint(0, 100000, (axes, T), generator=g, dtype=torch.int32).cuda()
        self.freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device="cuda") * 2 / rot)
        self.axis = (torch.arange(rot // 2, device="cuda") % axes).to(torch.int32)
        self.p = binding.make_params(len(new), H_q, H_kv, D, table.shape[1], self.P, 1)
        self.ws = binding.alloc_prompt_workspace(self.p)

    def run(self, q=None, k=None, q_out=None, k_out=None, status=0):
        """Codes, scales, summaries, rotated q and k."""
        q, k = self.q if q is None else q, self.k if k is None else k
        q_out, k_out = torch.zeros_like(q) if q_out is None else q_out, torch.zeros_like(k) if k_out is None else k_out
        cache = [t.clone() for t in self.cache]
        meta = torch.zeros(self.P, self.H_kv, 2, self.D, dtype=torch.bfloat16, device="cuda")
        binding.se_kv8_append(self.p, q, k, self.v, self.cu, self.seq, self.table, self.pos, self.freq, self.axis, q_out, *cache, self.ws,
                              meta=meta, k_out=k_out, interleaved=self.interleaved)
        assert binding.se_last_device_status(self.ws) == status
        return (*cache, meta, q_out, k_out)

    def check(self, got):
        k8, v8, scales, meta, q_out, k_out = got
        q_ref, k_ref = torch.zeros_like(q_out), torch.zeros_like(k_out)
        k16, v16 = (torch.zeros(self.P, self.H_kv, 16, self.D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        binding.se_rope_append(self.p, self.q, self.k, self.v, self.cu, self.seq, self.table, self.pos, self.freq, self.axis, q_ref, k16, v16,
                               self.ws, k_out=k_ref, interleaved=self.interleaved)
        binding.se_last_device_status(self.ws)
        assert torch.equal(q_out, q_ref) and torch.equal(k_out, k_ref)
        want = ref.append(*self.cache, torch.zeros_like(meta), k_out, self.v, self.new, self.total, self.table.cpu())
        for x, y in zip((k8, v8, scales, meta), want):
            assert torch.equal(x.double(), y)


@pytest.mark.parametrize("axes,rot,interleaved", [(3, 128, False), (2, 64, True), (4, 96, False)])
def test_several_axes(axes, rot, interleaved):
    a = Append(91, [70, 1, 33], [5, 16, 0], 8, 2, 128, axes, rot, interleaved)
    a.check(a.run())


def test_new_tokens_without_a_page():
    a = Append(92, [70, 20], [5, 40], 8, 2, 64)
    a.table[0, 2], a.table[1, 3] = -1, a.P                            # a whole page; one that is no page of the pool
    a.check(a.run(status=binding.SE_DEV_BAD_PAGE_ID))


@pytest.mark.parametrize("D,new", [(128, [50, 1, 7]), (64, [1] * 40), (128, [3] * 500), (128, [60] * 100)])
def test_rotated_in_place(D, new):
    a = Append(93, new, [i % 20 for i in range(len(new))], 4, 2, D)
    want = a.run()
    q, k = a.q.clone(), a.k.clone()
    got = a.run(q=q, k=k, q_out=q, k_out=k)
    for x, y in zip(got, want):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    a.check(want)
