"""Large batches of attention, which are cut into pieces of two sizes: CTAs begin with a large one and take small ones as they
become free.  Both head widths, paged and contiguous, groups that fill a query tile and one that does not, absent pages."""
import pytest
import torch

import prompt_ref as ref
from test_gpu_prompt import Calls, check_attention

pytestmark = pytest.mark.gpu

CTAS, SHARE_COST, START, ROWS = 148, 2560, 128, 128


def cost(new, past, H_q, H_kv):
    """What the batch costs in the kernel's units (tokens seen by a query tile, and the start of a tile), and its longest item."""
    tpt = ROWS // (H_q // H_kv)
    total, longest = 0, 0
    for n, o in zip(new, past):
        for at in range(0, n, 2 * tpt):
            rows = min(2 * tpt, n - at)
            c = (2 if rows > tpt else 1) * (o + at + rows + START)
            total, longest = total + c * H_kv, max(longest, c)
    return total, longest


BATCHES = {
    "paged_128": ([600, 1, 333] * 18, [1400, 4000, 2000] * 18, 32, 8, 128, 0),
    "paged_128_seven_heads_absent": ([600, 1, 40, 555] * 22, [1400, 3000, 700, 1111] * 22, 28, 4, 128, 9),
    "paged_64_three_heads": ([700, 5] * 26, [1800, 2600] * 26, 24, 8, 64, 0),
    "contiguous_128": ([3000, 2500, 1, 2900, 3100, 129, 2777, 3000, 2800], None, 32, 8, 128, 0),
    "contiguous_64_five_heads": ([3000, 2500, 1, 2900, 3100, 129, 2777, 2000], None, 40, 8, 64, 0),
}


@pytest.mark.parametrize("name", sorted(BATCHES))
def test_pieces_of_two_sizes(name):
    new, past, H_q, H_kv, D, every = BATCHES[name]
    paged = past is not None
    past = past or [0] * len(new)
    total, longest = cost(new, past, H_q, H_kv)
    assert total / 10 > 2 * CTAS * SHARE_COST and total / 10 > 2 * longest        # well above where two sizes begin
    absent = [(r, b) for r in range(len(new)) for b in range(past[r] // 16) if every and (7 * r + b) % every == 0]
    c = Calls(ref.make_batch(61, new, past, H_q, H_kv, D, spare=2, absent=absent))
    # the second half of the workspace belongs to the small pieces
    half = c.ws[c.ws.numel() // 2 + 8192:]
    half.fill_(0xa5)
    check_attention(c, paged)
    assert bool((half != 0xa5).any()), "no small piece has left a partial result"
    first, lse = c.out.clone(), c.lse.clone()
    for _ in range(2):                   # the counters were left as they were found
        c.out.fill_(7.0)
        c.chunk() if paged else c.prompt()
        torch.cuda.synchronize()
        assert c.status() == 0
        n = sum(new)
        assert torch.equal(c.out[:n], first[:n]) and torch.equal(c.lse[:n], lse[:n])


def test_small_batches_have_pieces_of_one_size():
    new, past = [600, 1] * 7, [1400, 4000] * 7
    total, _ = cost(new, past, 32, 8)
    assert total / 10 < CTAS * SHARE_COST / 1.5
    c = Calls(ref.make_batch(62, new, past, 32, 8, 128))
    half = c.ws[c.ws.numel() // 2 + 8192:]
    half.fill_(0xa5)
    check_attention(c)
    assert bool((half == 0xa5).all())


@pytest.mark.parametrize("B", [87, 88, 89, 96, 97])
def test_batches_around_the_size_that_fits_shared_memory(B):
    b = ref.make_batch(63, [(5 * i) % 23 for i in range(B)], [(31 * i) % 200 for i in range(B)], 4, 2, 64, spare=1)
    c = Calls(b)
    check_attention(c)
    lse = ref.attend(b)[2].float()
    u = torch.rand(b.P, 2, 16, device="cuda")
    want, tol = ref.accumulate(b, lse, u)
    c.mass(lse, u)
    torch.cuda.synchronize()
    assert c.status() == 0
    assert bool(((u.double() - want).abs() <= tol).all())
