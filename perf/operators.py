"""The prompt-side operators of the engine: cases to measure, plain forms and 64-bit values.

Four operators carry a prompt (or a chunk of it) up to the point where decoding starts:

  append     rotary positions with several axes applied to the new tokens' q and k, K and V written into the
             paged cache, summaries of the touched pages brought up to date        (binding.se_rope_append)
  chunk      causal attention of the new tokens over the paged cache               (binding.se_chunk_attend)
  prompt     causal attention of packed whole prompts over contiguous K and V      (binding.se_prompt_attend)
  mass       accumulated attention weight of the cached tokens over the queries of
             a chunk, the statistic that the eviction reads                        (binding.se_h2o_accumulate)

A case says the operator, the head layout and how the lengths of its requests are drawn ("mix" seeds
that draw: the lengths belong to the case, the values to the seed given to ``prepare``).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE = 16


# ---- cases ----------------------------------------------------------------------------------------

def _case(op, B, H_kv, G, D, new, past, mix, name=None, **more):
    """``new`` = (lo, hi) new tokens of a request, ``past`` = (lo, hi) tokens cached before them."""
    c = {"op": op, "B": B, "H_kv": H_kv, "G": G, "D": D, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0],
         "past_hi": past[1], "mix": mix, "axes": 1, "rot": D, "interleaved": False, "summaries": False,
         "absent_percent": 0, "spare_rows": 0}
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of a continuous batch: one token of each of 64 requests goes into the cache
        _case("append", 64, 8, 4, 128, (1, 1), (0, 2047), 1, "append_decode_b64"),
        # a chunk of an image prompt: three position axes, heads in groups of seven, ragged lengths
        _case("append", 5, 4, 7, 128, (150, 900), (0, 1000), 2, "append_image_chunks", axes=3, summaries=True),
        # prefill of a packed batch of prompts
        _case("append", 8, 8, 4, 128, (1500, 4500), (0, 0), 3, "append_prompts_24k", summaries=True),
        # one new token of one request of the tiny layer: the latency of a call
        _case("chunk", 1, 2, 4, 64, (1, 1), (2047, 2047), 4, "chunk_one_token_tiny"),
        # a few drafted tokens verified at once over long contexts
        _case("chunk", 8, 8, 4, 128, (5, 5), (32000, 32768), 5, "chunk_drafts_b8_32k"),
        # continuous batching: decode tokens and prompt chunks of all sizes in one call, a tenth of the pages pruned
        _case("chunk", 24, 4, 7, 128, (1, 700), (100, 16000), 6, "chunk_mixed_b24", absent_percent=10),
        # one chunk of a long prompt over what is cached of it
        _case("chunk", 1, 8, 4, 128, (2048, 2048), (63488, 63488), 7, "chunk_2k_at_64k"),
        # short prompts of the tiny layer, packed, with unused rows behind the last one
        _case("prompt", 6, 2, 4, 64, (1, 301), (0, 0), 8, "prompt_short_tiny", spare_rows=13),
        # a packed batch of prompts of different lengths
        _case("prompt", 8, 8, 4, 128, (500, 4000), (0, 0), 9, "prompt_packed_b8"),
        # one long prompt
        _case("prompt", 1, 8, 4, 128, (32768, 32768), (0, 0), 10, "prompt_32k"),
        # a short chunk's share of the accumulated weights over long contexts
        _case("mass", 4, 8, 4, 128, (100, 500), (30000, 32000), 11, "mass_chunks_b4_32k"),
        # accumulated weights of a whole prompt, before the first eviction
        _case("mass", 1, 8, 4, 128, (16384, 16384), (0, 0), 12, "mass_prompt_16k"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    while True:
        op = rng.choice(["append", "chunk", "chunk", "prompt", "prompt", "mass"])
        H_kv, G, D = rng.choice([1, 2, 4, 8]), rng.randint(1, 8), rng.choice([64, 128, 128])
        B = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 16384)
        lo = rng.choice([1, max(1, hi // 4), hi])
        past = 0 if op == "prompt" else rng.choice([0, _log_int(rng, 1, 65536)])
        past_lo = rng.choice([0, past // 2, past])
        c = _case(op, B, H_kv, G, D, (lo, hi), (past_lo, past), rng.randint(100, 1 << 30))
        if op == "append":
            c.update(axes=rng.choice([1, 1, 2, 3]), rot=rng.choice([D, D, D // 2]), interleaved=rng.random() < 0.4,
                     summaries=rng.random() < 0.6)
        if op in ("chunk", "mass"):
            c["absent_percent"] = rng.choice([0, 0, 10, 50])
        if op == "prompt":
            c["spare_rows"] = rng.choice([0, 0, rng.randint(1, 40)])
        new, old = lengths(c)
        tokens = sum(new) + sum(old)
        if sum(new) > 32768 or tokens * H_kv * D > (1 << 28) or sum(new) * G * H_kv * D > (1 << 28):
            continue
        if op != "append" and not 1e6 < work(c)["flops"] < 5e12:
            continue
        return c


def lengths(case):
    """(new tokens, tokens cached before) of each request of the case."""
    r = random.Random(case["mix"])
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["B"])]
    old = [r.randint(case["past_lo"], case["past_hi"]) for _ in range(case["B"])]
    return new, old


def _absent(case, new, old):
    """Logical pages without physical KV, request by request: never a page that receives new tokens."""
    r = random.Random(case["mix"] + 1)
    return [[b for b in range(o // PAGE) if r.random() * 100 < case["absent_percent"]] for o in old]


def work(case):
    new, old = lengths(case)
    H_kv, G, D = case["H_kv"], case["G"], case["D"]
    H_q, T = H_kv * G, sum(new)
    gone = [PAGE * len(a) for a in _absent(case, new, old)]
    seen = [n + o - g for n, o, g in zip(new, old, gone)]             # cached tokens that are present, the new ones included
    pairs = sum(n * (o - g) + n * (n + 1) // 2 for n, o, g in zip(new, old, gone))
    if case["op"] == "append":
        rows = 2 * T * (H_q + 2 * H_kv) * D * 2
        pages = sum((n + o + PAGE - 1) // PAGE - o // PAGE for n, o in zip(new, old))
        extra = pages * H_kv * 2 * D * 2 + sum(o % PAGE for o in old) * H_kv * D * 2 if case["summaries"] else 0
        return {"bytes": rows + extra + case["axes"] * T * 4, "flops": 3.0 * T * (H_q + H_kv) * case["rot"]}
    table = 0 if case["op"] == "prompt" else sum((n + o + PAGE - 1) // PAGE for n, o in zip(new, old)) * 4
    if case["op"] == "mass":
        return {"bytes": T * H_q * (2 * D + 4) + sum(seen) * H_kv * (2 * D + 8) + table, "flops": 2.0 * pairs * H_q * D}
    return {"bytes": T * H_q * (4 * D + 4) + sum(seen) * H_kv * 4 * D + table, "flops": 4.0 * pairs * H_q * D}


# ---- inputs ---------------------------------------------------------------------------------------

def _normal(g, *shape):
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = x.view(-1)
    for s in range(0, flat.numel(), 1 << 27):
        e = min(flat.numel(), s + (1 << 27))
        flat[s:e] = torch.randn(e - s, generator=g, device="cuda", dtype=torch.float32)
    return x


def prepare(case, seed):
    new, old = lengths(case)
    B, H_kv, G, D, op = case["B"], case["H_kv"], case["G"], case["D"], case["op"]
    H_q, T = H_kv * G, sum(new) + case["spare_rows"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    host = random.Random(seed)
    dev = dict(device="cuda")
    # what the projection of a layer leaves: the heads of q, k and v side by side in one row; a few channels of k are large
    qkv = _normal(g, T, H_q + 2 * H_kv, D)
    large = torch.tensor([[host.randrange(D) for _ in range(4)] for _ in range(H_kv)], **dev)
    factor = torch.ones(H_kv, D, **dev).scatter_(1, large, 8.0).to(torch.bfloat16)
    qkv[:, H_q:H_q + H_kv] *= factor
    s = {"case": dict(case), "new": new, "old": old, "T": T,
         "q": qkv[:, :H_q], "k": qkv[:, H_q:H_q + H_kv], "v": qkv[:, H_q + H_kv:],
         "cu": torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, **dev)}
    total = [n + o for n, o in zip(new, old)]
    s["total"] = total
    pages = [(t + PAGE - 1) // PAGE for t in total]
    s["seq_lens"] = torch.tensor(total, dtype=torch.int32, **dev)
    if op != "prompt":
        # pages of all requests dealt from one permuted pool
        P, widest = max(1, sum(pages)), max(pages)
        order = torch.randperm(P, generator=g, **dev).to(torch.int32)
        table = np.full((B, widest), -1, dtype=np.int64)
        at = 0
        for r, n in enumerate(pages):
            table[r, :n] = np.arange(at, at + n)
            at += n
        for r, gone in enumerate(_absent(case, new, old)):
            table[r, gone] = -1
        dealt = torch.tensor(table, **dev)
        s["page_table"] = torch.where(dealt >= 0, order[dealt.clamp(min=0)], torch.full_like(dealt, -1).int()).contiguous()
        s["k_cache"] = _normal(g, P, H_kv, PAGE, D)
        s["v_cache"] = _normal(g, P, H_kv, PAGE, D)
        s["k_cache"] *= factor[None, :, None]
    else:
        P, widest = 1, 1
    s["P"] = P
    if op == "append":
        # text counts on along every axis; a part of every prompt is an image of 16 columns
        spot = torch.cat([torch.arange(o, o + n, **dev) for n, o in zip(new, old)])
        pos = spot[None].repeat(case["axes"], 1)
        image = (spot % 1024) >= 512
        for a in range(1, case["axes"]):
            step = (spot % 16) if a == case["axes"] - 1 else (spot // 16) % 16
            pos[a] = torch.where(image, spot - spot % 256 + step, pos[a])
        s["positions"] = pos.to(torch.int32).contiguous()
        n = case["rot"] // 2
        s["inv_freq"] = 500000.0 ** (-torch.arange(n, dtype=torch.float64, **dev) / n)
        s["pair_axis"] = (torch.arange(n, **dev) * case["axes"] // n).to(torch.int32)
        s["meta"] = torch.zeros(P, H_kv, 2, D, dtype=torch.bfloat16, **dev) if case["summaries"] else None
        s["q_out"] = torch.zeros(T, H_q, D, dtype=torch.bfloat16, **dev)
    else:
        # rotation has left q in a buffer of its own
        s["q"] = s["q"].contiguous()
        s["out"] = torch.zeros(T, H_q, D, dtype=torch.bfloat16, **dev)
        s["lse"] = torch.zeros(T, H_q, dtype=torch.float32, **dev)
    if op == "mass":
        _plain_attention(s, lse_only=True)
        s["before"] = torch.rand(P, H_kv, PAGE, generator=g, **dev)
    if own:
        from paper_2609_39068_b200 import binding
        s["p"] = binding.make_params(B, H_q, H_kv, D, widest, P, 1)
        s["workspace"] = binding.alloc_prompt_workspace(s["p"])
    return s


# ---- plain forms ----------------------------------------------------------------------------------

def _blocks(s, width):
    """Requests cut into blocks of query rows whose scores fit about 2 GB at ``width`` bytes each."""
    H_q, at = s["q"].shape[1], 0
    for r, (n, o) in enumerate(zip(s["new"], s["old"])):
        rows = max(16, int((2 << 30) / (width * H_q * (n + o))))
        for i in range(0, n, rows):
            j = min(n, i + rows)
            yield r, slice(at + i, at + j), o + i, o + j
        at += n


def _keys(s, r, end, name, dtype):
    """K or V of the first ``end`` tokens of request r, [H_kv, end, D], and which of them are present."""
    if s["case"]["op"] == "prompt":
        at = sum(s["new"][:r])
        return s[name][at:at + end].to(dtype).transpose(0, 1), torch.ones(end, dtype=torch.bool, device="cuda")
    row = s["page_table"][r, :(end + PAGE - 1) // PAGE]
    x = s[name + "_cache"][row.clamp(min=0)].to(dtype).transpose(0, 1)
    return x.reshape(x.shape[0], -1, x.shape[-1])[:, :end], (row >= 0).repeat_interleave(PAGE)[:end]


def _scores(s, r, rows, first, last, dtype):
    """Logits [H_kv, G, rows, tokens] of a block of query rows, -inf where the row does not see the token."""
    H_kv, G, D = s["case"]["H_kv"], s["case"]["G"], s["case"]["D"]
    k, present = _keys(s, r, last, "k", dtype)
    q = s["q"][rows].to(dtype).view(-1, H_kv, G, D).permute(1, 2, 0, 3)
    z = torch.matmul(q.reshape(H_kv, -1, D), k.transpose(1, 2)).view(H_kv, G, -1, last) * (D ** -0.5)
    at = torch.arange(last, device="cuda")
    hidden = (at[None, :] > torch.arange(first, last, device="cuda")[:, None]) | ~present[None, :]
    return z.masked_fill_(hidden, -math.inf)


def _plain_attention(s, lse_only=False):
    for r, rows, first, last in _blocks(s, 4):
        z = _scores(s, r, rows, first, last, torch.float32)
        top = z.amax(-1, keepdim=True)
        weight = (z - top.clamp(min=-1e30)).exp_()
        total = weight.sum(-1, keepdim=True)
        s["lse"][rows] = (top + total.log())[..., 0].permute(2, 0, 1).flatten(1)
        if not lse_only:
            v = _keys(s, r, last, "v", torch.float32)[0]
            H_kv, G = z.shape[:2]
            o = torch.matmul(weight.view(H_kv, -1, last), v).view(H_kv, G, -1, v.shape[-1]) / total.clamp(min=1e-30)
            s["out"][rows] = o.permute(2, 0, 1, 3).flatten(1, 2).to(torch.bfloat16)
    return s["out"], s["lse"]


def _plain_mass(s):
    u = s["before"].clone()
    for r, rows, first, last in _blocks(s, 4):
        H_kv, G = s["case"]["H_kv"], s["case"]["G"]
        lse = s["lse"][rows].view(-1, H_kv, G).permute(1, 2, 0)[..., None]
        share = (_scores(s, r, rows, first, last, torch.float32) - lse).exp_().sum((1, 2))
        row = s["page_table"][r, :(last + PAGE - 1) // PAGE]
        share = torch.nn.functional.pad(share, (0, row.numel() * PAGE - last)).view(H_kv, -1, PAGE).transpose(0, 1)
        u.index_add_(0, row[row >= 0], share[row >= 0])
    return u


def _slots(s):
    """Physical page and slot of every new token, in row order."""
    r = torch.repeat_interleave(torch.arange(len(s["new"]), device="cuda"), s["cu"][1:] - s["cu"][:-1], output_size=sum(s["new"]))
    at = torch.arange(sum(s["new"]), device="cuda") - s["cu"][r + 1] + s["seq_lens"][r]
    return r, s["page_table"][r, at // PAGE].long(), at


def _rotated(x, s, cos, sin):
    """``x`` [T, H, D] in 32 bits, its first ``rot`` channels turned."""
    n = s["case"]["rot"] // 2
    lo, hi = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if s["case"]["interleaved"] else (slice(0, n), slice(n, 2 * n))
    x = x.float()
    y = x.clone()
    y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
    y[..., hi] = x[..., hi] * cos + x[..., lo] * sin
    return y.to(torch.bfloat16)


def _plain_append(s):
    angle = s["positions"][s["pair_axis"].long()].double().t() * s["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    s["q_out"][:] = _rotated(s["q"], s, cos, sin)
    r, page, at = _slots(s)
    s["k_cache"][page, :, at % PAGE] = _rotated(s["k"], s, cos, sin)
    s["v_cache"][page, :, at % PAGE] = s["v"]
    if s["meta"] is not None:
        _summaries(s, r, page, at, s["k_cache"], s["meta"])
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"], "meta": s["meta"]}


def _summaries(s, r, page, at, k_cache, meta):
    """Channel-wise smallest and largest key of every page that received a token."""
    filled = (s["seq_lens"][r] - at // PAGE * PAGE).clamp(max=PAGE)
    spare = (torch.arange(PAGE, device="cuda") >= filled[:, None])[:, None, :, None]
    first = (at % PAGE == 0) | (torch.arange(at.numel(), device="cuda") == s["cu"][r])
    page, spare, k = page[first], spare[first], k_cache[page[first]]
    meta[page, :, 0] = k.masked_fill(spare, math.inf).amin(2)
    meta[page, :, 1] = k.masked_fill(spare, -math.inf).amax(2)


# ---- one pass -------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if not own:
        return {"append": _plain_append, "chunk": _plain_attention, "prompt": _plain_attention, "mass": _plain_mass}[op](s)
    from paper_2609_39068_b200 import binding
    p, ws = s["p"], s["workspace"]
    if op == "append":
        binding.se_rope_append(p, s["q"], s["k"], s["v"], s["cu"], s["seq_lens"], s["page_table"], s["positions"],
                               s["inv_freq"], s["pair_axis"], s["q_out"], s["k_cache"], s["v_cache"], ws,
                               meta=s["meta"], interleaved=s["case"]["interleaved"])
        return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"], "meta": s["meta"]}
    if op == "mass":
        u = s["before"].clone()
        binding.se_h2o_accumulate(p, s["q"], s["cu"], s["k_cache"], s["page_table"], s["seq_lens"], s["lse"], u, ws)
        return u
    if op == "chunk":
        binding.se_chunk_attend(p, s["q"], s["cu"], s["k_cache"], s["v_cache"], s["page_table"], s["seq_lens"],
                                s["out"], ws, lse=s["lse"])
    else:
        binding.se_prompt_attend(p, s["q"], s["k"], s["v"], s["cu"], s["out"], ws, lse=s["lse"])
    return s["out"], s["lse"]


# ---- 64-bit values --------------------------------------------------------------------------------

def _exact_append(s):
    n, T = s["case"]["rot"] // 2, sum(s["new"])
    turn = torch.polar(torch.ones(T, n, dtype=torch.float64, device="cuda"),
                       s["positions"][s["pair_axis"].long()].t() * s["inv_freq"])[:, None]

    def turned(x):
        x = x.double()
        if s["case"]["interleaved"]:
            z = torch.view_as_complex(x[..., :2 * n].unflatten(-1, (n, 2)).contiguous()) * turn
            return torch.cat([torch.view_as_real(z).flatten(-2), x[..., 2 * n:]], -1)
        z = torch.complex(x[..., :n].contiguous(), x[..., n:2 * n].contiguous()) * turn
        return torch.cat([z.real, z.imag, x[..., 2 * n:]], -1)

    out = {"q": turned(s["q"]), "k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double(), "meta": None}
    where = [(int(s["page_table"][r, j // PAGE]), j % PAGE) for r, (m, o) in enumerate(zip(s["new"], s["old"])) for j in range(o, o + m)] \
        if T < 2000 else None
    page, slot = (torch.tensor(x, device="cuda") for x in zip(*where)) if where else (_slots(s)[1], _slots(s)[2] % PAGE)
    out["k_cache"][page, :, slot] = turned(s["k"])
    out["v_cache"][page, :, slot] = s["v"].double()
    if s["meta"] is not None:
        out["meta"] = torch.zeros(s["meta"].shape, dtype=torch.float64, device="cuda")
        table = s["page_table"].cpu()
        for r, (m, o) in enumerate(zip(s["new"], s["old"])):
            for b in range(o // PAGE, (m + o + PAGE - 1) // PAGE):
                k = out["k_cache"][int(table[r, b]), :, :min(PAGE, m + o - b * PAGE)]
                out["meta"][int(table[r, b])] = torch.stack([k.min(1).values, k.max(1).values], 1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s)
    H_kv, G, D = case["H_kv"], case["G"], case["D"]
    out = torch.zeros(s["T"], H_kv * G, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["T"], H_kv * G, dtype=torch.float64, device="cuda")
    u = s["before"].double() if case["op"] == "mass" else None
    for r, rows, first, last in _blocks(s, 24):
        k, present = _keys(s, r, last, "k", torch.float64)
        v = None if u is not None else _keys(s, r, last, "v", torch.float64)[0]
        seen = torch.ones(last - first, last, dtype=torch.bool, device="cuda").tril(first) & present
        for h in range(H_kv):
            q = s["q"][rows, h * G:(h + 1) * G].double().transpose(0, 1)
            z = torch.where(seen, q @ k[h].t() / math.sqrt(D), -math.inf)
            if u is None:
                total = z.logsumexp(-1)
                lse[rows, h * G:(h + 1) * G] = total.t()
                share = torch.where(seen, (z - total[..., None]).exp(), 0.0)
                out[rows, h * G:(h + 1) * G] = (share @ v[h]).transpose(0, 1)
            else:
                own_lse = s["lse"][rows, h * G:(h + 1) * G].double().t()
                share = torch.where(seen, (z - own_lse[..., None]).exp(), 0.0).sum((0, 1))
                page = s["page_table"][r, torch.arange(last, device="cuda") // PAGE].long()
                slot = torch.arange(last, device="cuda") % PAGE
                u[page[present], h, slot[present]] += share[present]
    return u if u is not None else (out, lse)
