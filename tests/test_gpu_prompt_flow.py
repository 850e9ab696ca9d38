"""The prompt-side operators together, as a serving step uses them: a prompt enters in chunks (rotation and append,
attention, accumulated weights), is evicted down to its budget, and decoding goes on over what is left."""
import os
import subprocess
import sys

import pytest
import torch

import prompt_ref as ref
from paper_2609_39068_b200 import binding

pytestmark = pytest.mark.gpu


def test_prompt_in_chunks_then_eviction_then_decode():
    H_q, H_kv, D, budget, recent = 8, 2, 128, 256, 32
    lens = [700, 333]                                           # prompt tokens of two requests
    chunks = [[300, 333], [400, 0]]                             # the second request's prompt fits one chunk
    b = ref.make_batch(7, lens, [0, 0], H_q, H_kv, D, nan_tail=False, wide=2)
    b.k_cache.fill_(float("nan"))
    b.v_cache.fill_(float("nan"))
    table = b.page_table
    for r, t in enumerate(lens):                                # room for the decoded token behind the prompt
        if t % 16 == 0:
            table[r, t // 16] = b.P - 1 - r
    p = binding.make_params(2, H_q, H_kv, D, b.max_pages, b.P, b.max_pages)
    ws, dws = binding.alloc_prompt_workspace(p), binding.alloc_workspace(p)
    n = D // 2
    inv_freq = 10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)
    axis = (torch.arange(n, device="cuda") * 3 // n).to(torch.int32)
    meta = torch.zeros(b.P, H_kv, 2, D, dtype=torch.bfloat16, device="cuda")
    u = torch.zeros(b.P, H_kv, 16, device="cuda")
    outs, lses, qs = [[], []], [[], []], [[], []]
    done = [0, 0]
    for sizes in chunks:
        rows = torch.cat([torch.arange(sum(lens[:r]) + done[r], sum(lens[:r]) + done[r] + m) for r, m in enumerate(sizes)]).cuda()
        qkv = b.qkv[rows]
        pos = torch.cat([torch.arange(done[r], done[r] + m) for r, m in enumerate(sizes)]).to(torch.int32).cuda()[None].repeat(3, 1).contiguous()
        pos[2] += 5                                             # another position on the third axis
        done = [d + m for d, m in zip(done, sizes)]
        cu = torch.tensor([0, sizes[0], sum(sizes)], dtype=torch.int32, device="cuda")
        sl = torch.tensor(done, dtype=torch.int32, device="cuda")
        q, k, v = qkv[:, :H_q], qkv[:, H_q:H_q + H_kv], qkv[:, H_q + H_kv:]
        T = sum(sizes)
        q_rot = torch.empty(T, H_q, D, dtype=torch.bfloat16, device="cuda")
        out, lse = torch.empty_like(q_rot), torch.empty(T, H_q, device="cuda")
        binding.se_rope_append(p, q, k, v, cu, sl, table, pos, inv_freq, axis, q_rot, b.k_cache, b.v_cache, ws, meta=meta)
        binding.se_chunk_attend(p, q_rot, cu, b.k_cache, b.v_cache, table, sl, out, ws, lse=lse)
        binding.se_h2o_accumulate(p, q_rot, cu, b.k_cache, table, sl, lse, u, ws)
        for r in range(2):
            s = slice(int(cu[r]), int(cu[r + 1]))
            outs[r].append(out[s]), lses[r].append(lse[s]), qs[r].append(q_rot[s])
    assert binding.se_last_device_status(ws) == 0
    # the same as one pass over the whole prompts
    b.qkv[:, :H_q] = torch.cat([torch.cat(x) for x in qs])
    want, tol, want_lse, ltol = ref.attend(b)
    got, got_lse = torch.cat([torch.cat(x) for x in outs]), torch.cat([torch.cat(x) for x in lses])
    assert bool(((got.double() - want).abs() <= tol).all()) and bool(((got_lse.double() - want_lse).abs() <= ltol).all())
    want_u, u_tol = ref.accumulate(b, got_lse, torch.zeros_like(u))
    assert bool(((u.double() - want_u).abs() <= u_tol + 1e-6 * want_u).all())
    rebuilt = torch.zeros_like(meta)
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    binding.se_meta_update(p, b.k_cache, table, sl, rebuilt, first_tok=torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert torch.equal(meta, rebuilt)

    # eviction down to the budget, by the prompt's own statistic
    kept_k = [ref.cached(b, r, b.k_cache)[0] for r in range(2)]
    kept_v = [ref.cached(b, r, b.v_cache)[0] for r in range(2)]
    weights = [torch.stack([u[table[r, j // 16].long(), :, j % 16] for j in range(lens[r])], 1) for r in range(2)]
    keep = torch.zeros(2, H_kv, budget, dtype=torch.int32, device="cuda")
    cnt = torch.zeros(2, H_kv, dtype=torch.int32, device="cuda")
    binding.se_h2o_retain(p, u, table, sl, budget, recent, keep, cnt, dws)
    binding.se_h2o_compact(p, b.k_cache, b.v_cache, u, table, keep, cnt, sl, dws)
    assert sl.tolist() == [budget, budget]
    for r in range(2):
        for h in range(H_kv):
            w = weights[r][h].clone()
            w[-recent:] = float("inf")
            assert keep[r, h].tolist() == sorted(w.argsort(descending=True, stable=True)[:budget].tolist())

    # one decoded token per request: appended, then attended densely by both the prompt call and the decode step
    sl += 1
    cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    qkv = torch.randn(2, H_q + 2 * H_kv, D, device="cuda").to(torch.bfloat16)
    pos = torch.tensor([lens] * 3, dtype=torch.int32, device="cuda")
    q_rot = torch.empty(2, H_q, D, dtype=torch.bfloat16, device="cuda")
    k_rot = torch.empty(2, H_kv, D, dtype=torch.bfloat16, device="cuda")
    binding.se_rope_append(p, qkv[:, :H_q], qkv[:, H_q:H_q + H_kv], qkv[:, H_q + H_kv:], cu, sl, table, pos, inv_freq, axis, q_rot,
                           b.k_cache, b.v_cache, ws, k_out=k_rot)
    out, lse = torch.empty_like(q_rot), torch.empty(2, H_q, device="cuda")
    binding.se_chunk_attend(p, q_rot, cu, b.k_cache, b.v_cache, table, sl, out, ws, lse=lse)
    sel = torch.zeros(2, H_kv, b.max_pages, dtype=torch.int32, device="cuda")
    sel_cnt = torch.zeros(2, H_kv, dtype=torch.int32, device="cuda")
    dout, dlse = torch.empty(2, H_q, D, device="cuda"), torch.empty(2, H_q, device="cuda")
    binding.se_meta_update(p, b.k_cache, table, sl, meta, first_tok=torch.zeros(2, dtype=torch.int32, device="cuda"))
    binding.se_decode_step(p, q_rot, b.k_cache, b.v_cache, meta, table, sl, 16 * b.max_pages, sel, sel_cnt, dout, dlse, dws)
    assert binding.se_last_device_status(ws) == 0 and binding.se_last_device_status(dws) == 0
    for r in range(2):
        for h in range(H_kv):
            at = keep[r, h].long()
            k = torch.cat([kept_k[r][h, at], k_rot[r, h].double()[None]])
            v = torch.cat([kept_v[r][h, at], qkv[r, H_q + H_kv + h].double()[None]])
            for a in range(h * 4, h * 4 + 4):
                z = k @ q_rot[r, a].double() / D ** 0.5
                w = z.softmax(0)
                assert abs(float(lse[r, a]) - float(z.logsumexp(0))) < 1e-4
                assert abs(float(dlse[r, a]) - float(z.logsumexp(0))) < 1e-3
                bound = 1.01 * (ref.HALF_BF16 * (w @ v).abs() + (ref.HALF_BF16 + 1e-3) * (w @ v.abs()))
                assert bool(((out[r, a].double() - w @ v).abs() <= bound).all())
                assert float((dout[r, a].double() - w @ v).abs().max()) < 1e-2


def test_contiguous_and_paged_attention_of_a_prompt_agree():
    b = ref.make_batch(8, [500, 90], [0, 0], 6, 2, 128, nan_tail=False)
    p = binding.make_params(2, 6, 2, 128, b.max_pages, b.P, 1)
    ws = binding.alloc_prompt_workspace(p)
    inv_freq = 10000.0 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    axis = torch.zeros(64, dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(500), torch.arange(90)]).to(torch.int32).cuda()[None].contiguous()
    q = torch.empty(b.T, 6, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.empty(b.T, 2, 128, dtype=torch.bfloat16, device="cuda")
    binding.se_rope_append(p, b.q, b.k, b.v, b.cu, b.seq_lens, b.page_table, pos, inv_freq, axis, q, b.k_cache, b.v_cache, ws, k_out=k)
    out = [torch.empty_like(q) for _ in range(2)]
    lse = [torch.empty(b.T, 6, device="cuda") for _ in range(2)]
    binding.se_chunk_attend(p, q, b.cu, b.k_cache, b.v_cache, b.page_table, b.seq_lens, out[0], ws, lse=lse[0])
    binding.se_prompt_attend(p, q, k, b.v, b.cu, out[1], ws, lse=lse[1])
    assert binding.se_last_device_status(ws) == 0
    assert torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1])      # the same tiles in the same order


FIRST_CALLS = """
import torch, prompt_ref as ref
from paper_2609_39068_b200 import binding
b = ref.make_batch(5, [7, 40], [100, 3], 8, 2, 128)
p = binding.make_params(b.B, b.H_q, b.H_kv, b.D, b.max_pages, b.P, 1)
ws = binding.alloc_prompt_workspace(p)
out, first = (torch.zeros(b.T, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
lse, u = torch.zeros(b.T, 8, device="cuda"), torch.zeros(b.P, 2, 16, device="cuda")
pos = torch.zeros(1, b.T, dtype=torch.int32, device="cuda")
freq, axis = torch.ones(64, dtype=torch.float64, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
q, k, v = torch.empty_like(out), b.k_cache.clone(), b.v_cache.clone()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    binding.se_rope_append(p, b.q, b.k, b.v, b.cu, b.seq_lens, b.page_table, pos, freq, axis, q, k, v, ws)
    binding.se_prompt_attend(p, b.q, b.k, b.v, b.cu, first, ws)
    binding.se_chunk_attend(p, b.q, b.cu, b.k_cache, b.v_cache, b.page_table, b.seq_lens, out, ws, lse=lse)
    binding.se_h2o_accumulate(p, b.q, b.cu, b.k_cache, b.page_table, b.seq_lens, lse, u, ws)
g.replay()
torch.cuda.synchronize()
want, tol, _, _ = ref.attend(b)
assert bool(((out.double() - want).abs() <= tol).all()) and binding.se_last_device_status(ws) == 0
assert torch.equal(q, b.q) and abs(float(u.double().sum()) - 47 * 8) < 0.04
b.total = list(b.new)                  # whole prompts: nothing lies before the rows
want, tol, _, _ = ref.attend(b, paged=False)
assert bool(((first.double() - want).abs() <= tol).all())
"""


def test_the_first_calls_of_a_process_may_be_captured():
    here = os.path.dirname(os.path.abspath(__file__))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([here, os.path.dirname(here)]))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
