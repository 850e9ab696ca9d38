"""Decode over an 8-bit cache where every warp has far more pages than the 32 that it looks up at a time: contexts of up to 131072
tokens for many requests at once (which share their pages, as requests with one prefix do).

Bounds: those of kv8_ref.decode.  With equal logits all that is left of them are the weights' and the sums' 2^-18 each."""
import math

import pytest
import torch

import kv8_ref as ref
from paper_2609_39068_b200 import binding

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


class Shared:
    """``lens`` tokens of the requests, all in the same pages; ``absent``: (first, count) logical pages that are not there."""

    def __init__(self, seed, lens, H_kv, G, D, absent=()):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.H_kv, self.G, self.D = lens, H_kv, G, D
        pages = (max(lens) + 15) // 16
        self.k8, self.v8, self.scales = ref.make_cache(g, pages, H_kv, D, "cuda")
        order = torch.randperm(pages, generator=g).to(torch.int32)
        for first, count in absent:
            order[first:first + count] = -1
        self.order = order.cuda()
        self.table = self.order.repeat(len(lens), 1).contiguous()
        self.seq = torch.tensor(lens, **I32)
        self.q = torch.randn(len(lens), H_kv * G, D, generator=g).to(torch.bfloat16).cuda()
        self.p = binding.make_params(len(lens), H_kv * G, H_kv, D, pages, pages, 1)
        self.ws = binding.alloc_prompt_workspace(self.p)
        self.out = torch.full((len(lens), H_kv * G, D), float("nan"), device="cuda")
        self.lse = torch.full((len(lens), H_kv * G), float("nan"), device="cuda")

    def run(self):
        binding.se_kv8_decode(self.p, self.q, self.k8, self.v8, self.scales, self.table, self.seq, self.out, self.lse, self.ws)
        assert binding.se_last_device_status(self.ws) == 0

    def want(self, r, h):
        """kv8_ref.decode's values and bounds of one pair, the pages gathered at once."""
        n, sm = self.lens[r], self.D ** -0.5
        at = self.order[:(n + 15) // 16].long()
        here = ((at >= 0)[:, None] & (torch.arange(len(at) * 16, device="cuda").view(-1, 16) < n)).view(-1)
        at = at.clamp(min=0)
        kk, vv = ((c[at, h].double() * self.scales[at, h, i].double()[:, None, None]).view(-1, self.D)[here]
                  for i, c in enumerate((self.k8, self.v8)))
        ss = self.scales[at, h, 1].double().repeat_interleave(16)[here]
        x = self.q[r, h * self.G:(h + 1) * self.G].double()
        z = sm * x @ kk.t()
        top = z.amax(1, keepdim=True)
        zerr = sm * (self.D + 2) * 2.0 ** -23 * (x.abs() @ kk.abs().t())
        zerr = zerr + 2.0 ** -22 * (z.abs() + top.abs() + ss.log().abs() + ss.log().abs().max()) + 2.0 ** -18
        p = (z - top).exp()
        s = p.sum(1, keepdim=True)
        w = p / s
        werr = w * (zerr + (w * zerr).sum(1, keepdim=True) + 2.0 ** -22) + 2.0 ** -37 * (w * ss).amax(1, keepdim=True) / ss
        lse = (top + s.log())[:, 0]
        return (w @ vv, 1.01 * (werr @ vv.abs()) + 2.0 ** -18 * (w @ vv.abs()), lse,
                (w * zerr).sum(1) + 2.0 ** -22 * lse.abs() + 2.0 ** -22)

    def check(self, pairs):
        self.run()
        worst = 0.0
        for r, h in pairs:
            out, tol, lse, ltol = self.want(r, h)
            rows = slice(h * self.G, (h + 1) * self.G)
            err, lerr = (self.out[r, rows].double() - out).abs(), (self.lse[r, rows].double() - lse).abs()
            worst = max(worst, float((err / tol).max()), float((lerr / ltol).max()))
        assert worst <= 1.0, worst
        first = self.out.clone(), self.lse.clone()
        self.out.fill_(float("nan")), self.lse.fill_(float("nan"))
        self.run()                                                  # equal inputs, equal bits
        assert torch.equal(self.out, first[0]) and torch.equal(self.lse, first[1])


MANY = [131072, 131067, 100001, 65536] * 16                         # 1500 pages for each warp
SOME = [20000 + 701 * i for i in range(16)]                         # 86


@pytest.mark.parametrize("lens,H_kv,G,D", [(SOME, 8, 4, 128), (SOME, 8, 7, 64), (MANY, 8, 1, 128), (MANY, 8, 8, 64)])
@pytest.mark.parametrize("absent", [(), ((0, 33), (100, 200), (700, 1), (1000, 140))])
def test_long_contexts(lens, H_kv, G, D, absent):
    d = Shared(61, lens, H_kv, G, D, absent)
    n = len(lens)
    d.check([(0, 0), (1, H_kv - 1), (n // 2, 3), (n - 2, 1), (n - 1, H_kv - 1)])


@pytest.mark.parametrize("lens,H_kv,G,D", [(SOME, 8, 4, 128), (MANY, 8, 1, 128), (MANY, 8, 8, 64), ([131072] * 64, 8, 2, 128), ([131072], 1, 2, 128)])
@pytest.mark.parametrize("kind", ["near", "two"])
def test_sums_of_nearly_equal_weights(lens, H_kv, G, D, kind):
    """Logits near one another, or of two kinds, and positive V: every rounding of a sum goes the same way, if the sums let it."""
    d = Shared(62, lens, H_kv, G, D)
    d.scales.fill_(1.0)
    d.v8.view(torch.uint8).bitwise_and_(0x07).bitwise_or_(0x38)     # 1 .. 1.875
    if kind == "near":
        d.scales[..., 0] = 2.0 ** -9
    else:
        d.q.fill_(1.0)
        d.k8.view(torch.uint8).fill_(0)
        d.k8.view(torch.uint8)[:, :, 0, 0] = 0x51                   # 9 / sqrt(D) for the first token of every page, 0 for the others
    n = len(lens)
    d.check([(0, 0), (n - 1, H_kv - 1)] if n > 1 else [(0, 0)])
    d.q.zero_()
    d.v8.view(torch.uint8).fill_(0x38)
    d.run()
    assert float((d.out.double() - 1).abs().max()) <= 3.03 * 2.0 ** -18 + 2.0 ** -22
    want = torch.tensor(lens, device="cuda").double().log()[:, None]
    assert float((d.lse.double() - want).abs().max()) <= 2.0 ** -18 + 2.0 ** -22 * (1 + math.log(131072))
