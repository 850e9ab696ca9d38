"""Attention of new tokens where its sums are long: the log-sum-exp against closed forms.  And values that are not finite: rows
that they enter are NaN, however the batch was cut, and other rows are what they were."""
import math

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


# whole items in a CTA, one KV tile (alternating streams of a single tile, pairs of query tiles) and several; items in many parts
CUTS = {
    "one_tile": ([20], [40], 8, 2, 64),
    "pair_of_tiles": ([300], [0], 8, 2, 128),
    "a_few_tiles": ([20], [300], 8, 2, 128),
    "whole_items_of_several_tiles": ([20] * 40, [300] * 40, 32, 8, 64),
    "many_parts": ([20], [9000], 8, 2, 128),
    "pairs_in_many_parts": ([150], [9000], 8, 2, 64),
}


def expect(c, paged, bad, blind=()):
    """`bad` [T, H_q]: rows that have to be NaN, but for those in `blind` (token, head), all of whose logits are -infinity: they
    see nothing.  The others are held to the reference of the batch without the bad values."""
    c.out.fill_(7.0)
    c.lse.fill_(7.0)
    c.chunk() if paged else c.prompt()
    torch.cuda.synchronize()
    assert c.status() == 0
    lost = bad.clone()
    for at, head in blind:
        assert bool((c.out[at, head] == 0).all()) and float(c.lse[at, head]) == -math.inf
        lost[at, head] = False
    assert bool(c.out[lost].isnan().all()) and bool(c.lse[lost].isnan().all())
    want, tol, lse, ltol = ref.attend(c.b_clean, paged)
    assert bool(((c.out.double() - want).abs() <= tol)[~bad].all())
    assert bool(((c.lse.double() - lse).abs() <= ltol)[~bad].all())


def copies(name, paged):
    """The batch twice: one to spoil, one for the reference."""
    new, past, H_q, H_kv, D = CUTS[name]
    batches = [ref.make_batch(17, new, past if paged else [0] * len(new), H_q, H_kv, D) for _ in range(2)]
    c = Calls(batches[0])
    c.b_clean = batches[1]
    return c


@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("name", sorted(CUTS))
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_bad_query_head_makes_its_own_row_nan(name, paged, value):
    # (an infinite channel gives infinite logits of both signs, and the difference of two infinities)
    c = copies(name, paged)
    bad = torch.zeros(c.b.T, c.b.H_q, dtype=torch.bool, device="cuda")
    for at, head in ((0, 0), (7, 1), (c.b.T - 1, c.b.H_q - 1)):
        c.b.qkv[at, head, 3] = value
        bad[at, head] = True
    if not paged:                        # the first token sees itself alone: one infinite logit, of either sign
        c.b.qkv[0, 0, 3] = math.nan
    blind = []
    if paged and math.isinf(value) and c.b.total[0] == c.b.new[0]:             # the same
        own = c.b.k_cache[int(c.b.page_table[0, 0]), 0, 0, 3]
        blind = [(0, 0)] if float(own) < 0 else []
    expect(c, paged, bad, blind)


@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("name", sorted(CUTS))
def test_a_nan_key_reaches_the_rows_that_see_it(name, paged):
    c = copies(name, paged)
    b = c.b
    i, H_kv = 5, b.H_kv                  # a new token of the first request, last kv-head
    if paged:
        j = b.total[0] - b.new[0] + i
        b.k_cache[int(b.page_table[0, j // 16]), H_kv - 1, j % 16, 9] = math.nan
    else:
        b.k[i, H_kv - 1, 9] = math.nan
    bad = torch.zeros(b.T, b.H_q, dtype=torch.bool, device="cuda")
    bad[i:b.new[0], (H_kv - 1) * b.H_q // H_kv:] = True
    expect(c, paged, bad)


@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_bad_values_of_a_request_stay_in_it(paged, value):
    # three requests side by side, the rows and keys of the one in the middle all bad
    new, past = [40, 33, 140], [200, 5000, 0] if paged else [0, 0, 0]
    batches = [ref.make_batch(18, new, past, 8, 2, 128) for _ in range(2)]
    c = Calls(batches[0])
    c.b_clean = batches[1]
    b = c.b
    b.qkv[b.rows(1)] = value
    if paged:
        pages = b.page_table[1, :(b.total[1] + 15) // 16].long()
        b.k_cache[pages] = value
        b.v_cache[pages] = value
    bad = torch.zeros(b.T, b.H_q, dtype=torch.bool, device="cuda")
    bad[b.rows(1)] = True
    expect(c, paged, bad)


def test_rows_that_see_nothing_are_zero_in_every_cut():
    # no visible position, and no NaN from the division by the sum of no weights
    for new, past in (([20], [40]), ([20], [9000]), ([150], [9000]), ([20], [300])):
        pages = (new[0] + past[0] + 15) // 16
        b = ref.make_batch(19, new, past, 8, 2, 64, absent=[(0, i) for i in range(pages)])
        c = Calls(b)
        c.chunk()
        torch.cuda.synchronize()
        assert c.status() == 0
        assert bool((c.out == 0).all()) and bool((c.lse == -math.inf).all())
