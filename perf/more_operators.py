"""The operators of the 8-bit cache and of the page pool: cases to measure, plain forms and 64-bit values.

Three operators work on a paged cache whose keys and values are held as e4m3 codes with a power-of-two scale for each
(page of 16 tokens, kv-head); two keep the pool's pages in order for any kind of cache:

  append    rotary positions for the new tokens' q and k, K and V quantised into their pages, older codes of a page
            brought to its new scale, page summaries                                    (binding.se_kv8_append)
  decode    attention of one token per request over the selected (or all) pages         (binding.se_kv8_decode)
  chunk     causal attention of packed new tokens over the cache                        (binding.se_kv8_chunk_attend)
  update    requests fork, end, shrink and grow: new page tables and reference counts,
            shared pages that will be written copied                                    (binding.se_pages_update)
  compact   live pages moved to the front of the pool                                   (binding.se_pages_compact)

A case says the operator, the head layout and how lengths are drawn ("mix" seeds that draw: the structure belongs to
the case, the values to the seed given to ``prepare``).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE = 16
E4M3 = torch.float8_e4m3fn
TOP, LEAST, MOST = 448.0, -64, 7          # largest code; range of the scales' exponents


# ---- cases ----------------------------------------------------------------------------------------

def _attention(op, B, H_kv, G, D, new, past, mix, name=None, **more):
    """``new`` = (lo, hi) new tokens of a request, ``past`` = (lo, hi) tokens cached before them."""
    c = {"op": op, "B": B, "H_kv": H_kv, "G": G, "D": D, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0],
         "past_hi": past[1], "mix": mix, "rot": D, "interleaved": False, "summaries": False, "absent_percent": 0, "selected": 0}
    return _named(c, name, more)


def _pool(op, kind, B, beams, P, layers, H_kv, D, tokens, mix, name=None, **more):
    """``tokens`` = (lo, hi) tokens of a request; ``beams`` requests in a row share a prompt."""
    c = {"op": op, "kind": kind, "B": B, "beams": beams, "P": P, "layers": layers, "H_kv": H_kv, "D": D, "lo": tokens[0],
         "hi": tokens[1], "mix": mix, "codes": False}
    return _named(c, name, more)


def _named(c, name, more):
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of a continuous batch: one token of each of 64 requests goes into the cache
        _attention("append", 64, 8, 4, 128, (1, 1), (0, 2047), 1, "append_decode_b64", summaries=True),
        # prefill of a packed batch of prompts
        _attention("append", 8, 8, 4, 128, (1500, 4500), (0, 0), 2, "append_prompts_24k", summaries=True),
        # one token of one request of the tiny layer over all of its pages: the latency of a call
        _attention("decode", 1, 2, 4, 64, (1, 1), (2047, 2047), 3, "decode_one_tiny"),
        # a sparse layer: 64 requests of very different lengths, 2048 selected tokens per head
        _attention("decode", 64, 8, 4, 128, (1, 1), (4095, 65535), 4, "decode_sparse_b64", selected=128),
        # a dense layer of a continuous batch, heads in groups of seven, a tenth of the pages pruned
        _attention("decode", 16, 4, 7, 128, (1, 1), (100, 32767), 5, "decode_dense_b16", absent_percent=10),
        # a few drafted tokens verified at once over long contexts
        _attention("chunk", 8, 8, 4, 128, (5, 5), (32000, 32768), 6, "chunk_drafts_b8_32k"),
        # continuous batching: decode tokens and prompt chunks of all sizes in one call
        _attention("chunk", 24, 4, 7, 128, (1, 700), (100, 16000), 7, "chunk_mixed_b24", absent_percent=10),
        # one chunk of a long prompt over what is cached of it
        _attention("chunk", 1, 8, 4, 128, (2048, 2048), (63488, 63488), 8, "chunk_2k_at_64k"),
        # the step between two decode steps: every request has room for one more token
        _pool("update", "grow", 64, 1, 65536, 1, 2, 64, (100, 8000), 9, "update_grow_b64"),
        # beam search, 16 prompts with 8 beams each: beams go on from other beams, eight layers follow
        _pool("update", "beams", 128, 8, 16384, 8, 8, 128, (500, 3000), 10, "update_beams_b128"),
        # a small pool of the tiny layer
        _pool("compact", "serve", 8, 1, 1024, 1, 2, 64, (50, 1000), 11, "compact_small"),
        # a pool that has served for a while, half of it live, four layers of an 8-bit cache
        _pool("compact", "serve", 64, 1, 40000, 4, 8, 128, (200, 9500), 12, "compact_40k", codes=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    while True:
        op = rng.choice(["append", "decode", "decode", "chunk", "chunk", "update", "update", "compact"])
        H_kv, G, D = rng.choice([1, 2, 4, 8]), rng.randint(1, 8), rng.choice([64, 128, 128])
        B, mix = _log_int(rng, 1, 64), rng.randint(100, 1 << 30)
        if op in ("update", "compact"):
            beams = rng.choice([1, 1, 2, 4, 5])
            hi = _log_int(rng, 16, 8192)
            lo = rng.choice([1, hi // 4 + 1, hi])
            need = B * (hi // PAGE + 3)
            c = _pool(op, rng.choice(["serve", "beams"]) if op == "update" else "serve", B, beams, _log_int(rng, need, 4 * need + 64),
                      rng.randint(1, 6), H_kv, D, (lo, hi), mix, codes=rng.random() < 0.5)
            if c["P"] > 65536 or c["P"] * c["layers"] * H_kv * D > 1 << 28:
                continue
            return c
        hi = 1 if op == "decode" else _log_int(rng, 1, 8192)
        lo = rng.choice([1, max(1, hi // 4), hi])
        past = rng.choice([0, _log_int(rng, 1, 65536)])
        c = _attention(op, B, H_kv, G, D, (lo, hi), (rng.choice([0, past // 2, past]), past), mix)
        if op == "append":
            c.update(rot=rng.choice([D, D, D // 2]), interleaved=rng.random() < 0.4, summaries=rng.random() < 0.6)
        if op != "append":
            c["absent_percent"] = rng.choice([0, 0, 10, 50])
        if op == "decode":
            c["selected"] = rng.choice([0, 0, _log_int(rng, 1, 512)])
        new, old = lengths(c)
        widest = max(n + o for n, o in zip(new, old))
        if sum(new) > 24576 or B * widest * H_kv * D > (1 << 29) or sum(new) * G * H_kv * D > (1 << 27):
            continue
        if op == "chunk" and not 1e6 < work(c)["flops"] < 2e12:
            continue
        return c


def lengths(case):
    """(new tokens, tokens cached before) of each request of an attention case."""
    r = random.Random(case["mix"])
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["B"])]
    old = [r.randint(case["past_lo"], case["past_hi"]) for _ in range(case["B"])]
    return new, old


def _absent(case, new, old):
    """Logical pages without physical KV, request by request: never a page that receives new tokens."""
    r = random.Random(case["mix"] + 1)
    return [[b for b in range(o // PAGE) if r.random() * 100 < case["absent_percent"]] for o in old]


def _pages(tokens):
    return (tokens + PAGE - 1) // PAGE


def _page_bytes(case):
    """Bytes of one page in all of a pool case's buffers."""
    rows = case["H_kv"] * PAGE * case["D"]
    return case["layers"] * (2 * rows + 8 * case["H_kv"] if case["codes"] else 4 * rows)


def work(case):
    if case["op"] in ("update", "compact"):
        s = _structure(case)
        entries = int(_pages(s["lens"]).sum())
        if case["op"] == "compact":
            moved = int((s["live"] >= len(s["live"])).sum())       # live pages behind the place where the live ones will end
            return {"bytes": 8.0 * entries + 12.0 * case["P"] + 2.0 * moved * _page_bytes(case), "flops": 0.0}
        copies = int(((s["new_lens"] > 0) & (s["parent"] != np.arange(case["B"]))).sum())
        return {"bytes": 8.0 * entries + 8.0 * case["P"] + 2.0 * copies * _page_bytes(case), "flops": 0.0}
    new, old = lengths(case)
    H_kv, G, D = case["H_kv"], case["G"], case["D"]
    H_q, T = H_kv * G, sum(new)
    if case["op"] == "append":
        rows = 2 * T * (2 * H_q + 2 * H_kv) * D + 2 * T * H_kv * D
        pages = sum(_pages(n + o) - o // PAGE for n, o in zip(new, old))
        extra = pages * H_kv * 4 * D if case["summaries"] else 0
        return {"bytes": float(rows + extra + pages * H_kv * 8 + sum(o % PAGE for o in old) * H_kv * 2 * D + 4 * T),
                "flops": 3.0 * T * (H_q + H_kv) * case["rot"] + 2.0 * T * 2 * H_kv * D}
    gone = [PAGE * len(a) for a in _absent(case, new, old)]
    seen = [n + o - g for n, o, g in zip(new, old, gone)]
    if case["selected"]:
        seen = [min(s, case["selected"] * PAGE) for s in seen]
        pairs = sum(seen)
    else:
        pairs = sum(n * (o - g) + n * (n + 1) // 2 for n, o, g in zip(new, old, gone))
    per_token = 2 * D + 8 / PAGE
    out = 2 if case["op"] == "chunk" else 4
    return {"bytes": T * H_q * ((2 + out) * D + 4) + sum(seen) * H_kv * per_token + sum(_pages(s) for s in seen) * 4.0,
            "flops": 4.0 * pairs * H_q * D}


# ---- inputs ---------------------------------------------------------------------------------------

def _structure(case):
    """Lengths, page tables and reference counts of a pool case, with page numbers before they are permuted."""
    r = np.random.RandomState(case["mix"] % (1 << 32))
    B, beams, P = case["B"], case["beams"], case["P"]
    prompt = np.repeat(r.randint(case["lo"], case["hi"] + 1, -(-B // beams)), beams)[:B]
    lens = prompt + (r.randint(0, 40, B) if beams > 1 else 0)
    if case["kind"] == "serve":
        lens[r.rand(B) < 0.15] = 0                                  # idle slots
    shared = np.where(np.arange(B) % beams > 0, prompt // PAGE, 0)  # full pages of the prompt that the first of the group owns
    shared[(lens == 0) | (lens[np.arange(B) // beams * beams] == 0)] = 0
    width = int(_pages(case["hi"] + 200)) + 8
    table = np.full((B, width), -1, dtype=np.int64)
    at = np.arange(width)
    held = at[None] < _pages(lens)[:, None]
    fresh = held & (at[None] >= shared[:, None])
    table[fresh] = np.arange(int(fresh.sum()))
    alias = held & ~fresh
    table[alias] = table[np.arange(B) // beams * beams][alias]
    # the pool's numbering: live pages are spread over all of it
    order = r.permutation(P)
    table = np.where(table >= 0, order[np.maximum(table, 0)], -1)
    refs = np.bincount(table[table >= 0], minlength=P)
    refs[r.choice(P, min(P // 50, int((refs == 0).sum())), replace=False)] += 1     # pages that a prefix cache holds too
    # what becomes of the slots
    parent = np.arange(B)
    first = np.arange(B) // beams * beams
    if case["kind"] == "beams":
        parent = np.minimum(first + r.randint(0, beams, B), B - 1)
        new_lens = lens[parent] + 1
    elif case["kind"] == "grow":
        new_lens = lens + 1
    else:
        what = r.rand(B)
        fork = (what < 0.2) & (lens == 0)
        parent[fork] = r.randint(0, B, int(fork.sum()))
        new_lens = lens[parent] + np.where(what > 0.4, 1, r.randint(0, 100, B))
        cut = (what >= 0.2) & (what < 0.3)
        new_lens[cut] = new_lens[cut] // 2
        gone = (what >= 0.3) & (what < 0.35)
        parent[gone], new_lens[gone] = -1, 0
        new_lens[(lens[np.maximum(parent, 0)] == 0) & (what > 0.8)] = 0
    return {"lens": lens, "table": table, "refs": refs, "parent": parent, "new_lens": new_lens, "live": np.nonzero(refs)[0]}


def _normal(g, *shape):
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = x.view(-1)
    for s in range(0, flat.numel(), 1 << 27):
        e = min(flat.numel(), s + (1 << 27))
        flat[s:e] = torch.randn(e - s, generator=g, device="cuda", dtype=torch.float32)
    return x


def _coded(g, P, H_kv, D, factor):
    """Codes and scales of P pages of normal values whose channels are multiplied by ``factor`` [H_kv, D]."""
    codes = torch.empty(P, H_kv, PAGE, D, dtype=E4M3, device="cuda")
    scale = torch.empty(P, H_kv, device="cuda")
    step = max(1, (1 << 26) // (H_kv * PAGE * D))
    for s in range(0, P, step):
        x = torch.randn(min(step, P - s), H_kv, PAGE, D, generator=g, device="cuda") * factor[:, None]
        scale[s:s + step] = _scale_of(x.to(torch.bfloat16).abs().float().amax((2, 3)))
        codes[s:s + step] = (x.to(torch.bfloat16).float() / scale[s:s + step, :, None, None]).clamp(-TOP, TOP).to(E4M3)
    return codes, scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (_prepare_pool if case["op"] in ("update", "compact") else _prepare_attention)(case, g, random.Random(seed))


def _prepare_attention(case, g, host):
    new, old = lengths(case)
    B, H_kv, G, D, op = case["B"], case["H_kv"], case["G"], case["D"], case["op"]
    H_q, T = H_kv * G, sum(new)
    dev = dict(device="cuda")
    qkv = _normal(g, T, H_q + 2 * H_kv, D)
    large = torch.tensor([[host.randrange(D) for _ in range(4)] for _ in range(H_kv)], **dev)
    factor = torch.ones(H_kv, D, **dev).scatter_(1, large, 8.0)     # a few channels of k are large
    qkv[:, H_q:H_q + H_kv] *= factor.to(torch.bfloat16)
    total = [n + o for n, o in zip(new, old)]
    pages = [_pages(t) for t in total]
    P, widest = sum(pages), max(pages)
    table = np.full((B, widest), -1, dtype=np.int64)
    at = 0
    for r, n in enumerate(pages):
        table[r, :n] = np.arange(at, at + n)
        at += n
    if op != "append":
        for r, gone in enumerate(_absent(case, new, old)):
            table[r, gone] = -1
    order = torch.randperm(P, generator=g, **dev).to(torch.int32)
    dealt = torch.tensor(table, **dev)
    s = {"case": dict(case), "new": new, "old": old, "T": T, "P": P,
         "q": qkv[:, :H_q], "k": qkv[:, H_q:H_q + H_kv], "v": qkv[:, H_q + H_kv:],
         "cu": torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, **dev),
         "seq_lens": torch.tensor(total, dtype=torch.int32, **dev),
         "page_table": torch.where(dealt >= 0, order[dealt.clamp(min=0)], torch.full_like(dealt, -1).int()).contiguous()}
    k8, ks = _coded(g, P, H_kv, D, factor)
    v8, vs = _coded(g, P, H_kv, D, torch.ones_like(factor))
    s["k8"], s["v8"], s["scales"] = k8, v8, torch.stack([ks, vs], -1).contiguous()
    if op == "append":
        spot = torch.cat([torch.arange(o, o + n, **dev) for n, o in zip(new, old)])
        s["positions"] = spot[None].to(torch.int32).contiguous()
        n = case["rot"] // 2
        s["inv_freq"] = 500000.0 ** (-torch.arange(n, dtype=torch.float64, **dev) / n)
        s["pair_axis"] = torch.zeros(n, dtype=torch.int32, **dev)
        s["meta"] = torch.zeros(P, H_kv, 2, D, dtype=torch.bfloat16, **dev) if case["summaries"] else None
        s["q_out"] = torch.zeros(T, H_q, D, dtype=torch.bfloat16, **dev)
    else:
        s["q"] = s["q"].contiguous()                                # rotation has left q in a buffer of its own
        s["out"] = torch.zeros(T, H_q, D, dtype=torch.float32 if op == "decode" else torch.bfloat16, **dev)
        s["lse"] = torch.zeros(T, H_q, **dev)
    if case["selected"]:
        # for every head its own pages: the newest one and a draw of the present ones
        n = min(case["selected"], widest)
        luck = torch.rand(B, H_kv, widest, generator=g, **dev).masked_fill_((s["page_table"] < 0)[:, None], -1.0)
        luck.scatter_(2, ((s["seq_lens"].long() - 1) // PAGE)[:, None, None].expand(B, H_kv, 1), 2.0)
        took, which = luck.topk(n, -1)
        which = torch.where(took >= 0, which, widest).sort(-1)[0]
        s["sel_idx"] = torch.where(which < widest, which, -1).to(torch.int32).contiguous()
        s["sel_cnt"] = (took >= 0).sum(-1).to(torch.int32)
    if own:
        from paper_2609_39068_b200 import binding
        s["p"] = binding.make_params(B, H_q, H_kv, D, widest, P, s["sel_idx"].shape[-1] if case["selected"] else 1)
        s["workspace"] = binding.alloc_prompt_workspace(s["p"])
    return s


def _prepare_pool(case, g, host):
    t = _structure(case)
    B, P, H_kv, D = case["B"], case["P"], case["H_kv"], case["D"]
    dev = dict(device="cuda")
    i32 = dict(dtype=torch.int32, **dev)
    order = torch.randperm(P, generator=g, **dev)                   # another seed: other page numbers
    table = torch.tensor(t["table"], **dev)
    s = {"case": dict(case), "page_table": torch.where(table >= 0, order[table.clamp(min=0)], -1).to(torch.int32).contiguous(),
         "seq_lens": torch.tensor(t["lens"], **i32), "new_lens": torch.tensor(t["new_lens"], **i32),
         "ref_count": torch.zeros(P, **i32).scatter_(0, order, torch.tensor(t["refs"], **i32)),
         "parent": None if case["kind"] == "grow" else torch.tensor(t["parent"], **i32)}
    s["buffers"] = []
    for _ in range(case["layers"]):
        for _ in range(2):
            if case["codes"]:
                bits = torch.randint(0, 127, (P, H_kv, PAGE, D), dtype=torch.uint8, generator=g, **dev)
                s["buffers"].append(bits.view(E4M3))
            else:
                s["buffers"].append(_normal(g, P, H_kv, PAGE, D))
        if case["codes"]:
            s["buffers"].append(torch.exp2(torch.randint(-9, 0, (P, H_kv, 2), generator=g, **dev).float()))
    s["table_out"], s["lens_out"] = torch.empty_like(s["page_table"]), torch.empty_like(s["seq_lens"])
    s["refs_out"], s["count"] = torch.empty_like(s["ref_count"]), torch.zeros(1, **i32)
    s["page_map"] = torch.empty(P, **i32)
    if own:
        from paper_2609_39068_b200 import binding
        s["p"] = binding.make_params(B, H_kv, H_kv, D, table.shape[1], P, 1)
        s["workspace"] = binding.alloc_pages_workspace(s["p"])
        s["handle"] = binding.page_buffers(s["buffers"])
    return s


# ---- plain forms: the 8-bit cache -----------------------------------------------------------------

def _scale_of(top):
    """The smallest power of two that brings ``top`` to 448 or below, its exponent between -64 and 7."""
    part, e = torch.frexp(top)                                      # top = part * 2^e, part in [0.5, 1)
    e = e - 9 + (part > 0.875).int()                                # 448 = 0.875 * 2^9
    return torch.ldexp(torch.ones_like(top), torch.where(top > 0, e, LEAST).clamp(LEAST, MOST))


def _rotated(x, s, cos, sin):
    """``x`` [T, H, D] in 32 bits, its first ``rot`` channels turned, rounded to bf16."""
    n = s["case"]["rot"] // 2
    lo, hi = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if s["case"]["interleaved"] else (slice(0, n), slice(n, 2 * n))
    x = x.float()
    y = x.clone()
    y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
    y[..., hi] = x[..., hi] * cos + x[..., lo] * sin
    return y.to(torch.bfloat16)


def _slots(s):
    """Request, logical position, physical page and touched-page number of every new token."""
    n = s["cu"][1:] - s["cu"][:-1]
    r = torch.repeat_interleave(torch.arange(n.numel(), device="cuda"), n, output_size=s["T"])
    at = torch.arange(s["T"], device="cuda") - s["cu"][r + 1] + s["seq_lens"][r]
    first = (at % PAGE == 0) | (torch.arange(s["T"], device="cuda") == s["cu"][r])
    return r, at, s["page_table"][r, at // PAGE].long(), first


def _quantise(s, new, codes, scale, r, at, page, first):
    """New rows [T, H_kv, D] (bf16) into the codes of their pages; the scale of a page never shrinks while it holds tokens."""
    item = torch.cumsum(first, 0) - 1
    touched, start = page[first], at[first]
    older = start % PAGE                                            # tokens that the page held before
    slot = torch.arange(PAGE, device="cuda")[None, :, None, None]
    top = torch.zeros(touched.numel(), new.shape[1], device="cuda")
    top.scatter_reduce_(0, item[:, None].expand(-1, new.shape[1]), new.float().abs().amax(-1), "amax")
    before = scale[touched]
    after = torch.where(older[:, None] > 0, torch.maximum(before, _scale_of(top)), _scale_of(top))
    held = codes[touched].float().transpose(1, 2)                   # [pages, slot, head, channel]
    again = (held * (before / after)[:, None, :, None]).to(E4M3).float()
    held = torch.where(slot < older[:, None, None, None], again, held)
    held[item, at % PAGE] = (new.float() / after[item][..., None]).clamp(-TOP, TOP)
    held = held.to(E4M3).transpose(1, 2).contiguous()
    codes.view(torch.uint8)[touched] = held.view(torch.uint8)
    scale[touched] = after
    return touched, held, after


def _plain_append(s):
    angle = s["positions"][s["pair_axis"].long()].double().t() * s["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    s["q_out"][:] = _rotated(s["q"], s, cos, sin)
    r, at, page, first = _slots(s)
    touched, held, after = _quantise(s, _rotated(s["k"], s, cos, sin), s["k8"], s["scales"][..., 0], r, at, page, first)
    _quantise(s, s["v"], s["v8"], s["scales"][..., 1], r, at, page, first)
    if s["meta"] is not None:
        filled = (s["seq_lens"][r] - at // PAGE * PAGE).clamp(max=PAGE)[first]
        spare = (torch.arange(PAGE, device="cuda") >= filled[:, None])[:, None, :, None]
        k = held.float() * after[..., None, None]
        s["meta"][touched, :, 0] = k.masked_fill(spare, math.inf).amin(2).to(torch.bfloat16)
        s["meta"][touched, :, 1] = k.masked_fill(spare, -math.inf).amax(2).to(torch.bfloat16)
    return {"q": s["q_out"], "k": s["k8"], "v": s["v8"], "scales": s["scales"], "meta": s["meta"]} if s["meta"] is not None else \
        {"q": s["q_out"], "k": s["k8"], "v": s["v8"], "scales": s["scales"]}


def _plain_decode(s):
    c = s["case"]
    B, H_kv, G, D = c["B"], c["H_kv"], c["G"], c["D"]
    if c["selected"]:
        logical = s["sel_idx"].long()
    else:
        logical = torch.arange(s["page_table"].shape[1], device="cuda").expand(B, H_kv, -1)
    page = s["page_table"].long()[:, None].expand(B, H_kv, -1).gather(2, logical.clamp(min=0))
    at = logical[..., None] * PAGE + torch.arange(PAGE, device="cuda")
    seen = ((logical >= 0) & (page >= 0))[..., None] & (at < s["seq_lens"][:, None, None, None])
    page, head = page.clamp(min=0), torch.arange(H_kv, device="cuda")[None, :, None]
    scale = s["scales"][page, head][..., None, None, :]
    z = torch.matmul(s["q"].float().view(B, H_kv, G, D) * (D ** -0.5), (s["k8"][page, head].float() * scale[..., 0]).flatten(2, 3).transpose(2, 3))
    z = z.masked_fill_(~seen.flatten(2)[:, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    weight = (z - top.clamp(min=-1e30)).exp_()
    total = weight.sum(-1, keepdim=True)
    s["lse"][:] = (top + total.log()).view(B, H_kv * G)
    s["out"][:] = (torch.matmul(weight, (s["v8"][page, head].float() * scale[..., 1]).flatten(2, 3)) / total.clamp(min=1e-30)).view(B, H_kv * G, D)
    return s["out"], s["lse"]


def _blocks(s, width):
    """Requests cut into blocks of query rows whose scores fit about 2 GB at ``width`` bytes each."""
    H_q, at = s["q"].shape[1], 0
    for r, (n, o) in enumerate(zip(s["new"], s["old"])):
        rows = max(16, int((2 << 30) / (width * H_q * (n + o))))
        for i in range(0, n, rows):
            j = min(n, i + rows)
            yield r, slice(at + i, at + j), o + i, o + j
        at += n


def _values(s, r, end, which, dtype):
    """K (0) or V (1) of the first ``end`` tokens of request r, [H_kv, end, D], and which of them are present."""
    row = s["page_table"][r, :_pages(end)].long()
    x = s["v8" if which else "k8"][row.clamp(min=0)].to(dtype) * s["scales"][row.clamp(min=0), :, which].to(dtype)[..., None, None]
    x = x.transpose(0, 1)
    return x.reshape(x.shape[0], -1, x.shape[-1])[:, :end], (row >= 0).repeat_interleave(PAGE)[:end]


def _plain_chunk(s):
    H_kv, G, D = s["case"]["H_kv"], s["case"]["G"], s["case"]["D"]
    for r, rows, first, last in _blocks(s, 4):
        k, present = _values(s, r, last, 0, torch.float32)
        q = s["q"][rows].float().view(-1, H_kv, G, D).permute(1, 2, 0, 3)
        z = torch.matmul(q.reshape(H_kv, -1, D), k.transpose(1, 2)).view(H_kv, G, -1, last) * (D ** -0.5)
        at = torch.arange(last, device="cuda")
        z.masked_fill_((at[None, :] > torch.arange(first, last, device="cuda")[:, None]) | ~present[None, :], -math.inf)
        top = z.amax(-1, keepdim=True)
        weight = (z - top.clamp(min=-1e30)).exp_()
        total = weight.sum(-1, keepdim=True)
        s["lse"][rows] = (top + total.log())[..., 0].permute(2, 0, 1).flatten(1)
        v = _values(s, r, last, 1, torch.float32)[0]
        o = torch.matmul(weight.view(H_kv, -1, last), v).view(H_kv, G, -1, D) / total.clamp(min=1e-30)
        s["out"][rows] = o.permute(2, 0, 1, 3).flatten(1, 2).to(torch.bfloat16)
    return s["out"], s["lse"]


# ---- plain forms: the pool ------------------------------------------------------------------------

def _plain_update(s):
    table, lens, refs, new = s["page_table"].long(), s["seq_lens"].long(), s["ref_count"].long(), s["new_lens"].long()
    (B, width), P = table.shape, refs.numel()
    slot, at = torch.arange(B, device="cuda"), torch.arange(table.shape[1], device="cuda")
    parent = slot if s["parent"] is None else s["parent"].long()
    keep = torch.minimum(torch.where(parent >= 0, lens[parent.clamp(min=0)], 0), new)
    rows = table[parent.clamp(min=0)]
    n_kept, n_new = _pages(keep), _pages(new)
    kept = (at < n_kept[:, None]) & (rows >= 0)
    held = (at < _pages(lens)[:, None]) & (table >= 0)
    refs = refs - torch.bincount(table[held], minlength=P) + torch.bincount(rows[kept], minlength=P)
    # a page that will be written (a row ends inside it) and that others refer to is copied; of rows that only share it with
    # rows that end inside it too, the first goes on with it
    last = (keep // PAGE).clamp(max=width - 1)
    page = rows.gather(1, last[:, None])[:, 0]
    opened = (keep % PAGE > 0) & (page >= 0)
    where = torch.where(opened, page, P)
    opens = torch.bincount(where, minlength=P + 1)
    owner = torch.full((P + 1,), B, device="cuda").scatter_reduce_(0, where, slot, "amin")
    copy = opened & ((refs[page.clamp(min=0)] > opens[where]) | (owner[where] != slot))
    ask = (copy[:, None] & (at == last[:, None])) | ((at >= n_kept[:, None]) & (at < n_new[:, None]))
    free = (refs == 0).nonzero()[:, 0]
    asked = int(ask.sum())
    s["count"].fill_(free.numel() - asked)
    if asked > free.numel():
        s["table_out"].copy_(s["page_table"]), s["lens_out"].copy_(s["seq_lens"]), s["refs_out"].copy_(s["ref_count"])
    else:
        got = torch.where(kept, rows, -1)
        got[ask] = free[:asked]
        refs[free[:asked]] = 1
        refs -= torch.bincount(page[copy], minlength=P)
        to = got.gather(1, last[:, None])[copy, 0]
        for buffer in s["buffers"]:
            bits = buffer.view(torch.uint8)
            bits[to] = bits[page[copy]]
        s["table_out"].copy_(got), s["lens_out"].copy_(new), s["refs_out"].copy_(refs)
    return {"table": s["table_out"], "lens": s["lens_out"], "refs": s["refs_out"], "free": s["count"], "buffers": s["buffers"]}


def _plain_compact(s):
    refs = s["ref_count"]
    live = refs > 0
    n = int(live.sum())
    holes, movers = (~live[:n]).nonzero()[:, 0], live[n:].nonzero()[:, 0] + n
    moved = torch.arange(refs.numel(), device="cuda")
    moved[movers] = holes
    s["page_map"].copy_(torch.where(live, moved, -1))
    table = s["page_table"].long()
    held = (torch.arange(table.shape[1], device="cuda") < _pages(s["seq_lens"].long())[:, None]) & (table >= 0)
    s["table_out"].copy_(torch.where(held, moved[table.clamp(min=0)], table))
    s["refs_out"].zero_()
    s["refs_out"][moved[live]] = refs[live]
    for buffer in s["buffers"]:
        bits = buffer.view(torch.uint8)
        bits[holes] = bits[movers]
    s["count"].fill_(n)
    return {"table": s["table_out"], "map": s["page_map"], "refs": s["refs_out"], "live": s["count"], "buffers": s["buffers"]}


# ---- one pass -------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if not own:
        return {"append": _plain_append, "decode": _plain_decode, "chunk": _plain_chunk, "update": _plain_update,
                "compact": _plain_compact}[op](s)
    from paper_2609_39068_b200 import binding
    p, ws = s["p"], s["workspace"]
    if op == "append":
        binding.se_kv8_append(p, s["q"], s["k"], s["v"], s["cu"], s["seq_lens"], s["page_table"], s["positions"], s["inv_freq"],
                              s["pair_axis"], s["q_out"], s["k8"], s["v8"], s["scales"], ws, meta=s["meta"],
                              interleaved=s["case"]["interleaved"])
        got = {"q": s["q_out"], "k": s["k8"], "v": s["v8"], "scales": s["scales"]}
        return got if s["meta"] is None else {**got, "meta": s["meta"]}
    if op == "decode":
        binding.se_kv8_decode(p, s["q"], s["k8"], s["v8"], s["scales"], s["page_table"], s["seq_lens"], s["out"], s["lse"], ws,
                              sel_idx=s.get("sel_idx"), sel_cnt=s.get("sel_cnt"))
        return s["out"], s["lse"]
    if op == "chunk":
        binding.se_kv8_chunk_attend(p, s["q"], s["cu"], s["k8"], s["v8"], s["scales"], s["page_table"], s["seq_lens"], s["out"],
                                    ws, lse=s["lse"])
        return s["out"], s["lse"]
    if op == "update":
        binding.se_pages_update(p, s["page_table"], s["seq_lens"], s["ref_count"], s["new_lens"], s["table_out"], s["lens_out"],
                                s["refs_out"], s["count"], ws, parent=s["parent"], buffers=s["handle"])
        return {"table": s["table_out"], "lens": s["lens_out"], "refs": s["refs_out"], "free": s["count"], "buffers": s["buffers"]}
    binding.se_pages_compact(p, s["page_table"], s["seq_lens"], s["ref_count"], s["table_out"], s["refs_out"], s["page_map"],
                             s["count"], ws, buffers=s["handle"])
    return {"table": s["table_out"], "map": s["page_map"], "refs": s["refs_out"], "live": s["count"], "buffers": s["buffers"]}


# ---- 64-bit values --------------------------------------------------------------------------------

def _exact_append(s):
    """What the codes stand for before they are rounded: value / scale; the scales from the values rounded to bf16."""
    n, T, D = s["case"]["rot"] // 2, s["T"], s["case"]["D"]
    turn = torch.polar(torch.ones(T, n, dtype=torch.float64, device="cuda"), s["positions"][0].double()[:, None] * s["inv_freq"])[:, None]

    def turned(x):
        x = x.double()
        if s["case"]["interleaved"]:
            z = torch.view_as_complex(x[..., :2 * n].unflatten(-1, (n, 2)).contiguous()) * turn
            return torch.cat([torch.view_as_real(z).flatten(-2), x[..., 2 * n:]], -1)
        z = torch.complex(x[..., :n].contiguous(), x[..., n:2 * n].contiguous()) * turn
        return torch.cat([z.real, z.imag, x[..., 2 * n:]], -1)

    out = {"q": turned(s["q"]), "k": s["k8"].double(), "v": s["v8"].double(), "scales": s["scales"].double()}
    if s["meta"] is not None:
        out["meta"] = None                                          # extremes of rounded codes
    rows = {"k": turned(s["k"]), "v": s["v"].double()}
    table, row = s["page_table"].cpu().tolist(), 0
    for r, (m, o) in enumerate(zip(s["new"], s["old"])):
        for b in range(o // PAGE, _pages(o + m)):
            a, z, pid = max(o - b * PAGE, 0), min(o + m - b * PAGE, PAGE), table[r][b]
            for i, name in enumerate("kv"):
                x = rows[name][row + b * PAGE + a - o:row + b * PAGE + z - o].transpose(0, 1)        # [H_kv, tokens, D]
                top = x.to(torch.bfloat16).double().abs().amax((1, 2))
                scale = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)).clamp(-64, 7))
                if a:
                    scale = torch.maximum(scale, out["scales"][pid, :, i])
                    out[name][pid, :, :a] *= (out["scales"][pid, :, i] / scale)[:, None, None]
                out[name][pid, :, a:z] = (x / scale[:, None, None]).clamp(-448, 448)
                out["scales"][pid, :, i] = scale
        row += m
    return out


def _exact_attention(s):
    H_kv, G, D = s["case"]["H_kv"], s["case"]["G"], s["case"]["D"]
    out = torch.zeros(s["T"], H_kv * G, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["T"], H_kv * G, dtype=torch.float64, device="cuda")
    for r, rows, first, last in _blocks(s, 24):
        k, present = _values(s, r, last, 0, torch.float64)
        v = _values(s, r, last, 1, torch.float64)[0]
        seen = torch.ones(last - first, last, dtype=torch.bool, device="cuda").tril(first) & present
        for h in range(H_kv):
            sees = seen
            if s["case"]["selected"]:
                took = s["sel_idx"][r, h, :int(s["sel_cnt"][r, h])].long()
                chosen = torch.zeros(s["page_table"].shape[1], dtype=torch.bool, device="cuda")
                chosen[took] = True
                sees = seen & chosen.repeat_interleave(PAGE)[:last]
            q = s["q"][rows, h * G:(h + 1) * G].double().transpose(0, 1)
            z = torch.where(sees, q @ k[h].t() / math.sqrt(D), -math.inf)
            total = z.logsumexp(-1)
            lse[rows, h * G:(h + 1) * G] = total.t()
            share = torch.where(sees, (z - total[..., None]).exp(), 0.0)
            out[rows, h * G:(h + 1) * G] = (share @ v[h]).transpose(0, 1)
    return out, lse


def exact(case, seed):
    if case["op"] in ("update", "compact"):                         # numbers of pages, and copies
        return None
    s = prepare(case, seed)
    return _exact_append(s) if case["op"] == "append" else _exact_attention(s)
