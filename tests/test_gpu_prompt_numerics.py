"""Attention of new tokens where its sums are long: the log-sum-exp against closed forms."""
import pytest
import torch

import prompt_ref as ref
from paper_2609_39068_b200 import binding
from test_gpu_prompt import Calls

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def flat_bound(delta, lse, tiles_merged):
    """Bound of the error of ln(a + b exp(-delta)) where the kernel's maximum is exactly 0.  A weight: the argument of the
    exponential is one product with two rounded factors (3 U relative, so 3 U delta absolute in the exponent), the exponential
    is good to 2^-22 = 4 U.  The sum: a chain of 63 additions per lane and KV tile, one to join the two lanes, compensated
    sums of tiles (2 U), and 4 U for each partial result that is merged (two exponentials' products and an addition, and the
    exponential of an argument that is 0).  The logarithm and its two products: 4 U of the result."""
    return (3 * delta + 4 + 64 + 2 + 4 * tiles_merged + 4 * lse.abs()) * U


@pytest.mark.parametrize("tokens", [32768, 65536])
def test_lse_of_long_flat_rows_of_single_tokens(tokens):
    # 160 pairs of (request, kv-head), so a CTA has half a context to itself and more; the requests share their pages.  Every
    # page begins with a dominant token, the others have one weight
    B, H_kv, G, D = 20, 8, 4, 64
    P = tokens // 16
    delta = torch.linspace(1, 9, H_kv * G, device="cuda").bfloat16()
    q = torch.zeros(B, H_kv * G, D, dtype=torch.bfloat16, device="cuda")
    q[:, :, 5] = delta
    k = torch.zeros(P, H_kv, 16, D, dtype=torch.bfloat16, device="cuda")
    k[:, :, 1:, 5] = -1
    v = torch.ones_like(k)
    table = torch.randperm(P, device="cuda").to(torch.int32)[None].repeat(B, 1)
    cu = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    lens = torch.full((B,), tokens, dtype=torch.int32, device="cuda")
    p = binding.make_params(B, H_kv * G, H_kv, D, P, P, 1, sm_scale=1.0)
    ws = binding.alloc_prompt_workspace(p)
    out, lse = torch.empty_like(q), torch.empty(B, H_kv * G, device="cuda")
    binding.se_chunk_attend(p, q, cu, k, v, table, lens, out, ws, lse=lse)
    assert binding.se_last_device_status(ws) == 0
    d = delta.double()
    want = torch.log(P + (tokens - P) * torch.exp(-d))[None].expand(B, -1)
    # of 148 large pieces, each about as long as an item, an item meets three at most, of the small ones ten; two results each
    off = (lse.double() - want).abs()
    assert bool((off <= flat_bound(d, want, 26)).all()), float(off.max())
    # the weights' sum is rounded to bf16 only in the result, the weights are rounded before (to nearest, 2^-9 relative or less)
    assert bool(((out.double() - 1).abs() <= 2 * ref.HALF_BF16).all())


@pytest.mark.parametrize("D", [64, 128])
def test_lse_of_a_long_flat_prompt(D):
    # the first token dominates, all others have one weight; every row has a closed form
    n, G = 32768, 8
    b = ref.Batch(G, 1, D, [n], [n], n, n // 16, 1, torch.zeros(n, G + 2, D, dtype=torch.bfloat16, device="cuda"),
                  torch.tensor([0, n], dtype=torch.int32, device="cuda"), None, None, None, None)
    delta = torch.linspace(1, 9, G, device="cuda").bfloat16()
    b.qkv[:, :G, 7] = delta
    b.qkv[1:, G, 7] = -1
    c = Calls(b, scale=1.0)
    c.prompt()
    assert c.status() == 0
    d = delta.double()[None]
    want = torch.log(1 + torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * torch.exp(-d))
    # pieces are longer than items: an item meets two large ones or 20 small ones at most (its cost is 1/500 of the batch)
    off = (c.lse.double() - want).abs()
    assert bool((off <= flat_bound(d, want, 22)).all()), float(off.max())
