"""Decode over an 8-bit cache with logits so far from zero that fp32's steps are wider than a power of two: one token's logit is above
the others by more than half of itself, so it takes all of the weight, whatever the magnitude."""
import pytest
import torch

from test_gpu_kv8 import Decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("D", [64, 128])
def test_one_token_far_above_the_others(D, sign):
    for exponent in range(16, 60):
        d = Decode(81, [700, 30], 1, 4, D)
        step = 2.0 ** 7 if exponent > 20 else 1.0
        d.scales.fill_(1.0)
        d.scales[..., 0] = step
        d.k8.view(torch.uint8).fill_(0x40 if sign > 0 else 0xc0)      # 2, and 4 for the token that stands out
        pages = [int(d.table[0, 20]), int(d.table[1, 1])]
        for pid in pages:
            d.k8.view(torch.uint8)[pid, 0, 3] = 0x48 if sign > 0 else 0xb8
        d.q.fill_(1.37 * 2.0 ** exponent / (2 * D ** 0.5 * step))
        d.run()
        q = d.q[:, 0, 0].double()
        for r, pid in enumerate(pages):
            want = d.v8[pid, 0, 3].double()
            top = float(q[r]) * D ** 0.5 * step * (4 if sign > 0 else -1)
            assert float((d.out[r].double() - want).abs().max()) <= 2.0 ** -18 * float(want.abs().max()), exponent
            assert float((d.lse[r].double() - top).abs().max()) <= 2.0 ** -20 * abs(top), exponent
