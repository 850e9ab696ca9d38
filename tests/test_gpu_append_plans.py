"""The append's ways to share out its pages: whatever the batch, every token's rows, codes, scales and summaries are those that its
request gets in a call of its own, bit for bit, over a 16-bit and an 8-bit cache."""
import pytest
import torch

import kv8_ref as ref
from paper_2609_39068_b200 import binding
from test_gpu_kv8 import I32, page_tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H_q,H_kv,D", [(32, 8, 128), (28, 4, 128), (7, 1, 64), (8, 2, 64)])
@pytest.mark.parametrize("new,past", [
    ([1] * 130, list(range(130))),                                   # the heads of a page over two or more CTAs
    ([1] * 250, [3 * i % 70 for i in range(250)]),                   # a CTA per page
    ([2] * 250, [15] * 250),                                         # twice as many pages as the batch's sizes tell
    ([1] * 520, [i % 33 for i in range(520)]),                       # two rounds
    ([3] * 700, [5 * i % 61 for i in range(700)]),                   # many short pages
    ([40] * 200, [7 * i % 90 for i in range(200)]),                  # many full ones
    ([3000, 1, 0, 2500], [37, 15, 20, 0]),
    ([0, 0, 5] * 300, [i % 50 for i in range(900)]),                 # idle requests
])
def test_every_plan(H_q, H_kv, D, new, past):
    g = torch.Generator().manual_seed(71)
    total, T = [n + o for n, o in zip(new, past)], sum(new)
    table, P = page_tables(g, total)
    qkv = (torch.randn(T, H_q + 2 * H_kv, D, generator=g) * 3).to(torch.bfloat16).cuda()
    q, k, v = qkv.split([H_q, H_kv, H_kv], dim=1)
    cu = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), **I32)
    seq, table = torch.tensor(total, **I32), table.cuda()
    pos = torch.cat([torch.arange(o, o + n) for n, o in zip(new, past)]).to(torch.int32).cuda()[None].contiguous()
    freq = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device="cuda") * 2 / D)
    axis = torch.zeros(D // 2, **I32)
    whole = binding.make_params(len(new), H_q, H_kv, D, table.shape[1], P, 1)
    one = binding.make_params(1, H_q, H_kv, D, table.shape[1], P, 1)
    ws = binding.alloc_prompt_workspace(whole)
    k8, v8, scales = ref.make_cache(g, P, H_kv, D, "cuda")
    k16, v16 = (torch.randn(P, H_kv, 16, D, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    for call, cache in ((binding.se_rope_append, (k16, v16)), (binding.se_kv8_append, (k8, v8, scales))):
        got, want = [t.clone() for t in cache], [t.clone() for t in cache]
        outs = [[torch.zeros(T, H_q, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, H_kv, D, dtype=torch.bfloat16, device="cuda"),
                 torch.zeros(P, H_kv, 2, D, dtype=torch.bfloat16, device="cuda")] for _ in range(2)]
        call(whole, q, k, v, cu, seq, table, pos, freq, axis, outs[0][0], *got, ws, meta=outs[0][2], k_out=outs[0][1])
        row = 0
        for r, n in enumerate(new):
            if n:
                at = slice(row, row + n)
                call(one, q[at], k[at], v[at], torch.tensor([0, n], **I32), seq[r:r + 1].clone(), table[r:r + 1].clone(), pos[:, at].clone(), freq,
                     axis, outs[1][0][at], *want, ws, meta=outs[1][2], k_out=outs[1][1][at])
            row += n
        assert binding.se_last_device_status(ws) == 0
        for x, y in zip(got + outs[0], want + outs[1]):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
