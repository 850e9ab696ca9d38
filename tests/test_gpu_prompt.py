"""Prompt-side operators on the GPU against the 64-bit restatements of prompt_ref.py."""
import math

import pytest
import torch

import prompt_ref as ref
from paper_2609_39068_b200 import binding

pytestmark = pytest.mark.gpu
NAN = float("nan")


class Calls:
    """The calls on one batch, with output buffers that show untouched rows."""

    def __init__(self, b, scale=0.0):
        self.b, self.scale = b, scale or None
        self.p = binding.make_params(b.B, b.H_q, b.H_kv, b.D, b.max_pages, b.P, 1, sm_scale=scale)
        self.ws = binding.alloc_prompt_workspace(self.p)
        self.out = torch.full((b.T, b.H_q, b.D), NAN, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((b.T, b.H_q), NAN, device="cuda")

    def chunk(self, lse=True):
        b = self.b
        binding.se_chunk_attend(self.p, b.q, b.cu, b.k_cache, b.v_cache, b.page_table, b.seq_lens, self.out, self.ws,
                                lse=self.lse if lse else None)

    def prompt(self):
        b = self.b
        binding.se_prompt_attend(self.p, b.q, b.k, b.v, b.cu, self.out, self.ws, lse=self.lse)

    def mass(self, lse, u):
        b = self.b
        binding.se_h2o_accumulate(self.p, b.q, b.cu, b.k_cache, b.page_table, b.seq_lens, lse, u, self.ws)

    def status(self):
        return binding.se_last_device_status(self.ws)


def held(got, want, tol, what):
    got = got.double()
    live = ~want.isnan()
    assert bool(got[~live].isnan().all()), what + ": spare rows were written"
    same = torch.isinf(want) & (got == want)
    bad = live & ~same & ~((got - want).abs() <= tol)
    if bool(bad.any()):
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError("%s: %d values off, first at %s: %r, want %r +- %r" % (
            what, int(bad.sum()), i, float(got[i]), float(want[i]), float(tol[i])))


def check_attention(c, paged=True):
    c.chunk() if paged else c.prompt()
    torch.cuda.synchronize()
    assert c.status() == 0
    out, tol, lse, ltol = ref.attend(c.b, paged, c.scale)
    held(c.lse, lse, ltol, "lse")
    held(c.out, out, tol, "out")


# (new, past): single tokens, lengths of zero and one, page and tile edges, ragged mixes, long axes with few rows
SHAPES = {
    "one_token_alone": ([1], [0]),
    "one_token_17": ([1], [16]),
    "one_token_each": ([1, 1, 1, 1, 1], [0, 15, 16, 127, 500]),
    "empty_requests": ([0, 3, 0, 1, 0], [5, 0, 0, 40, 0]),
    "tile_edges": ([127, 128, 129], [1, 0, 127]),
    "page_edges": ([16, 15, 17, 32], [16, 1, 15, 0]),
    "prompts": ([300, 1, 77], [0, 0, 0]),
    "long_context_few_rows": ([3, 1], [9000, 4097]),
    "chunk": ([260, 31], [517, 1000]),
}


@pytest.mark.parametrize("name", sorted(SHAPES))
@pytest.mark.parametrize("H_q,H_kv,D", [(8, 2, 128), (8, 2, 64)])
def test_chunk_attention_shapes(name, H_q, H_kv, D):
    new, past = SHAPES[name]
    check_attention(Calls(ref.make_batch(11, new, past, H_q, H_kv, D, spare=3)))


@pytest.mark.parametrize("G", range(1, 9))
@pytest.mark.parametrize("D", [64, 128])
def test_chunk_attention_every_group_size(G, D):
    check_attention(Calls(ref.make_batch(20 + G, [45, 1, 150, 2], [33, 300, 0, 1000], 2 * G, 2, D)))


@pytest.mark.parametrize("name", ["one_token_alone", "prompts", "tile_edges", "empty_requests", "page_edges"])
@pytest.mark.parametrize("H_q,H_kv,D", [(8, 2, 128), (3, 1, 64), (14, 2, 128), (5, 5, 64)])
def test_prompt_attention(name, H_q, H_kv, D):
    new, _ = SHAPES[name]
    check_attention(Calls(ref.make_batch(31, new, [0] * len(new), H_q, H_kv, D, spare=5)), paged=False)


def test_long_prompt_and_large_batch():
    check_attention(Calls(ref.make_batch(41, [2500], [0], 8, 2, 128)), paged=False)
    new = [(7 * i) % 40 for i in range(300)]
    past = [(13 * i) % 90 for i in range(300)]
    check_attention(Calls(ref.make_batch(42, new, past, 4, 1, 64, spare=2)))


@pytest.mark.parametrize("new,past", [
    ([600, 1] * 12 + [1, 2] * 4 + [37], [1400, 4000] * 12 + [4100, 900] * 4 + [0]),   # long and short items side by side
    ([64] * 100 + [1] * 20, [1950] * 110 + [2500] * 10),
], ids=["chunks_and_tokens", "many_requests"])
def test_batches_large_enough_for_pieces_of_two_sizes(new, past):
    check_attention(Calls(ref.make_batch(44, new, past, 32, 8, 64, spare=1)))


def test_buffers_that_begin_on_16_bytes():
    b = ref.make_batch(45, [40, 1, 200], [900, 5000, 0], 8, 2, 128)
    c = Calls(b)
    room = torch.zeros(c.ws.numel() + 16, dtype=torch.uint8, device="cuda")
    c.ws = room[16:]
    binding.se_prompt_workspace_init(c.p, c.ws)
    c.out = torch.full((c.out.numel() + 8,), NAN, dtype=torch.bfloat16, device="cuda")[8:].view(c.out.shape)
    assert c.ws.data_ptr() % 32 == 16 and c.out.data_ptr() % 32 == 16
    check_attention(c)
    lse = ref.attend(b)[2].float()
    u = torch.zeros(b.P, 2, 16, device="cuda")
    want, tol = ref.accumulate(b, lse, u)
    c.mass(lse, u)
    held(u, want, tol, "score_accum")


def test_absent_pages_and_rows_that_see_nothing():
    # request 0 has lost its first page and its query page, so its first rows see nothing; request 1 has nothing at all
    b = ref.make_batch(51, [20, 5, 40], [0, 30, 400], 8, 2, 128, absent=[(0, 0), (1, 0), (1, 1), (1, 2), (2, 3), (2, 9), (2, 10)])
    c = Calls(b)
    check_attention(c)
    assert bool((c.lse[:16] == -math.inf).all()) and bool((c.out[:16] == 0).all())
    assert bool((c.lse[20:25] == -math.inf).all()) and bool((c.out[20:25] == 0).all())


def test_every_page_absent_but_the_last_of_a_long_request():
    b = ref.make_batch(52, [3], [5000], 8, 2, 64, absent=[(0, i) for i in range(312)])
    check_attention(Calls(b))


def test_scale_large_logits_and_missing_lse():
    b = ref.make_batch(53, [70, 9], [200, 64], 8, 4, 64)
    b.qkv.mul_(8)                                    # logits of hundreds: rows dominated by one token
    c = Calls(b, scale=0.3)
    check_attention(c)
    first = c.out.clone()
    c.out.fill_(NAN)
    c.lse.fill_(NAN)
    c.chunk(lse=False)
    torch.cuda.synchronize()
    assert torch.equal(first, c.out) and bool(c.lse.isnan().all())


def test_rising_logits_move_the_maximum_in_every_tile():
    # keys grow along the context, so every tile of the online softmax raises the maximum by a lot
    b = ref.make_batch(54, [40], [1500], 4, 1, 128, nan_tail=False)
    ramp = (torch.arange(b.max_pages, device="cuda").float() / 8)[:, None, None, None]
    rows = b.page_table[0].long()
    b.k_cache[rows] = (b.q[0, 0].float() * ramp / 16 + torch.randn(b.k_cache[rows].shape, device="cuda") * 0.1).to(torch.bfloat16)
    check_attention(Calls(b))


def test_bad_lengths_and_pages_are_left_out_and_reported():
    b = ref.make_batch(61, [5, 6, 7], [20, 30, 40], 8, 2, 128)
    c = Calls(b)
    want, tol, _, _ = ref.attend(b)
    b.seq_lens[1] = 5                                # fewer tokens than new ones
    c.chunk()
    assert c.status() == binding.SE_DEV_BAD_LENGTH
    assert bool(c.out[5:11].isnan().all())
    held(c.out[:5], want[:5], tol[:5], "out")
    held(c.out[11:], want[11:], tol[11:], "out")
    b.seq_lens[1] = 16 * b.max_pages + 1
    c.chunk()
    assert c.status() == binding.SE_DEV_BAD_LENGTH
    b.seq_lens[1] = 36
    b.cu[3] = b.T + 1
    c.chunk()
    assert c.status() == binding.SE_DEV_BAD_LENGTH
    b.cu[3] = b.T
    keep = int(b.page_table[2, 1])
    b.page_table[2, 1] = b.P + 7                     # treated as absent
    c.out.fill_(NAN)
    c.chunk()
    assert c.status() == binding.SE_DEV_BAD_PAGE_ID
    b.page_table[2, 1] = -1
    want, tol, _, _ = ref.attend(b)
    held(c.out, want, tol, "out")
    b.page_table[2, 1] = keep
    check_attention(c)


@pytest.mark.parametrize("new,past,H_q,H_kv,D,absent", [
    ([1], [0], 2, 1, 64, []),
    ([1, 1, 1], [15, 16, 400], 8, 2, 128, []),
    ([300, 0, 77], [0, 0, 0], 8, 2, 128, []),
    ([130, 40], [700, 30], 14, 2, 128, [(0, 3), (0, 4), (1, 0)]),
    ([129], [127], 5, 1, 64, []),
    ([900], [2000], 6, 2, 64, []),
    ([3, 2], [6000, 90], 24, 3, 128, [(0, 17)]),
])
def test_accumulated_weights(new, past, H_q, H_kv, D, absent):
    b = ref.make_batch(71, new, past, H_q, H_kv, D, spare=4, absent=absent)
    c = Calls(b)
    lse = ref.attend(b)[2].float()
    u = torch.rand(b.P, H_kv, 16, device="cuda")
    want, tol = ref.accumulate(b, lse, u)
    c.mass(lse, u)
    torch.cuda.synchronize()
    assert c.status() == 0
    held(u, want, tol, "score_accum")
    # all weights of a row add up to one per query head
    if not absent:
        add = torch.zeros_like(u)
        c.mass(lse, add)
        assert abs(float(add.double().sum()) - sum(new) * H_q) < 1e-4 * sum(new) * H_q


@pytest.mark.parametrize("G", range(1, 9))
def test_accumulated_weights_every_group_size(G):
    b = ref.make_batch(80 + G, [45, 1, 150], [33, 300, 0], 2 * G, 2, 128 if G % 2 else 64)
    c = Calls(b)
    lse = ref.attend(b)[2].float()
    u = torch.zeros(b.P, 2, 16, device="cuda")
    want, tol = ref.accumulate(b, lse, u)
    c.mass(lse, u)
    held(u, want, tol, "score_accum")


def test_accumulated_weights_of_rows_that_see_nothing():
    b = ref.make_batch(91, [20, 5], [0, 30], 8, 2, 128, absent=[(0, 0), (1, 0), (1, 1), (1, 2)])
    c = Calls(b)
    lse = ref.attend(b)[2].float()
    assert bool((lse[:16] == -math.inf).all())
    u = torch.rand(b.P, 2, 16, device="cuda")
    want, tol = ref.accumulate(b, lse, u)
    c.mass(lse, u)
    held(u, want, tol, "score_accum")


@pytest.mark.parametrize("at", range(16))
def test_a_bad_query_reaches_the_tokens_that_it_sees_and_no_others(at):
    b = ref.make_batch(95, [16], [200], 2, 2, 64)
    c = Calls(b)
    lse = ref.attend(b)[2].float()
    for value in (math.nan, math.inf):
        # a NaN query, and a log-sum-exp that makes all of its weights overflow
        x, y = b.qkv.clone(), lse.clone()
        if math.isnan(value):
            b.qkv[at, 0] = value
        else:
            y[at, 0] = -1e4
        u = torch.zeros(b.P, 2, 16, device="cuda")
        c.mass(y, u)
        got = u[b.page_table[0].long()].transpose(0, 1).reshape(2, -1)
        hit = got[0].isnan() if math.isnan(value) else got[0] == value
        assert bool(hit[:200 + at + 1].all()) and bool((got[0, 200 + at + 1:216].abs() <= 16).all())
        assert bool((got[1, :216].abs() <= 16.01).all()) and bool((got[:, 216:] == 0).all())
        b.qkv.copy_(x)


def test_weights_of_many_queries_add_up_without_loss():
    # a token that every query sees alike: with equal logits the weights are 1 / (number of tokens seen)
    n = 12000
    b = ref.make_batch(96, [n], [0], 8, 1, 64, nan_tail=False)
    b.qkv.zero_()
    c = Calls(b)
    seen = torch.arange(1, n + 1, dtype=torch.float64, device="cuda")
    lse = seen.log().float()[:, None].expand(n, 8).contiguous()
    u = torch.zeros(b.P, 1, 16, device="cuda")
    c.mass(lse, u)
    got = u[b.page_table[0].long()].reshape(-1)[:n].double()
    # the logarithm's rounding is the input's: at most 2^-24 * 9.4 relative in a weight.  On top of it the argument of
    # the exponential is rounded twice (2 * 2^-24 * 13.6 in powers of two), the exponential is good to 2^-22, and sums
    # of 32 weights in a chain add 32 * 2^-24
    want = torch.exp(-lse[:, 0].double()).flip(0).cumsum(0).flip(0) * 8
    assert float(((got - want).abs() / want).max()) <= 2 * 2.0 ** -24 * 13.6 + 2.0 ** -22 + 32 * 2.0 ** -24 + 4 * 2.0 ** -24


def rope_inputs(b, axes, rot, seed, far=0):
    g = torch.Generator().manual_seed(seed)
    n = rot // 2
    pos = torch.randint(0, far or 5000, (axes, b.T), generator=g, dtype=torch.int32)
    inv_freq = 10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)
    axis = torch.randint(0, axes, (n,), generator=g, dtype=torch.int32)
    return pos.cuda(), inv_freq.cuda(), axis.cuda()


@pytest.mark.parametrize("name", ["one_token_alone", "one_token_each", "empty_requests", "page_edges", "prompts", "chunk"])
@pytest.mark.parametrize("H_q,H_kv,D,rot,axes,inter", [(8, 2, 128, 128, 3, False), (8, 2, 64, 64, 1, True), (6, 2, 128, 64, 2, False),
                                                       (7, 1, 128, 48, 4, True), (4, 4, 64, 16, 1, False)])
def test_rope_append(name, H_q, H_kv, D, rot, axes, inter):
    new, past = SHAPES[name]
    b = ref.make_batch(101, new, past, H_q, H_kv, D, spare=2)
    c = Calls(b)
    pos, inv_freq, axis = rope_inputs(b, axes, rot, 7)
    k0, v0 = b.k_cache.clone(), b.v_cache.clone()
    q_out, k_out = c.out, torch.full((b.T, H_kv, D), NAN, dtype=torch.bfloat16, device="cuda")
    meta = torch.full((b.P, H_kv, 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
    binding.se_rope_append(c.p, b.q, b.k, b.v, b.cu, b.seq_lens, b.page_table, pos, inv_freq, axis, q_out, b.k_cache, b.v_cache,
                           c.ws, meta=meta, k_out=k_out, interleaved=inter)
    assert c.status() == 0
    n = sum(new)
    for got, x in ((q_out, b.q), (k_out, b.k)):
        want, tol = ref.rotate(x, pos, inv_freq, axis, inter)
        want[n:] = NAN
        held(got, want, tol, "rotation")
    k_want, v_want = k0.clone(), v0.clone()
    touched = torch.zeros(b.P, dtype=torch.bool, device="cuda")
    for r in range(b.B):
        for i in range(new[r]):
            j = past[r] + i
            pid = int(b.page_table[r, j // 16])
            touched[pid] = True
            k_want[pid, :, j % 16] = k_out[b.rows(r)][i]
            v_want[pid, :, j % 16] = b.v[b.rows(r)][i]
    assert torch.equal(b.k_cache.view(torch.int16), k_want.view(torch.int16))
    assert torch.equal(b.v_cache.view(torch.int16), v_want.view(torch.int16))
    rebuilt = torch.full_like(meta, 7.0)
    binding.se_meta_update(c.p, b.k_cache, b.page_table, b.seq_lens, rebuilt, first_tok=torch.zeros(b.B, dtype=torch.int32, device="cuda"))
    rebuilt[~touched] = 7.0
    assert torch.equal(meta.view(torch.int16), rebuilt.view(torch.int16))


@pytest.mark.parametrize("D,inter", [(128, False), (64, True)])
def test_rope_append_of_many_pages(D, inter, monkeypatch):
    monkeypatch.setitem(SHAPES, "many_pages", ([180, 17, 1] * 100, [5, 0, 130] * 100))
    test_rope_append("many_pages", 8, 2, D, D, 2, inter)


def test_rope_far_positions_and_in_place():
    b = ref.make_batch(111, [50], [3], 4, 2, 128)
    c = Calls(b)
    pos, inv_freq, axis = rope_inputs(b, 2, 128, 9, far=(1 << 31) - 1)
    q = b.q.contiguous()
    want, tol = ref.rotate(q, pos, inv_freq, axis, False)
    binding.se_rope_append(c.p, q, b.k, b.v, b.cu, b.seq_lens, b.page_table, pos, inv_freq, axis, q, b.k_cache, b.v_cache, c.ws)
    assert c.status() == 0
    held(q, want, tol, "rotation in place")


def test_rope_reports_absent_pages_and_bad_axes():
    b = ref.make_batch(112, [20, 4], [10, 0], 4, 2, 64, absent=[(0, 1)], nan_tail=False)
    c = Calls(b)
    pos, inv_freq, axis = rope_inputs(b, 2, 64, 9)
    k0 = b.k_cache.clone()
    args = (c.p, b.q, b.k, b.v, b.cu, b.seq_lens, b.page_table, pos, inv_freq, axis, c.out, b.k_cache, b.v_cache, c.ws)
    binding.se_rope_append(*args)
    assert c.status() == binding.SE_DEV_BAD_PAGE_ID
    want, tol = ref.rotate(b.q, pos, inv_freq, axis, False)
    held(c.out, want, tol, "rotation")                     # q is rotated all the same
    table = b.page_table[0].tolist()
    same = [i for i in range(b.P) if i not in (table[0], int(b.page_table[1, 0]))]
    assert torch.equal(b.k_cache[same], k0[same])
    b.page_table[0, 1] = b.P
    binding.se_rope_append(*args)
    assert c.status() == binding.SE_DEV_BAD_PAGE_ID
    assert torch.equal(b.k_cache[same], k0[same])
    axis[3] = 2
    b.page_table[0, 1] = same[0]
    binding.se_rope_append(*args)
    assert c.status() == binding.SE_DEV_BAD_LENGTH
    axis[3] = 1
    b.seq_lens[1] = 3
    c.out.fill_(NAN)
    binding.se_rope_append(*args)
    assert c.status() == binding.SE_DEV_BAD_LENGTH and bool(c.out[20:].isnan().all())


def test_binding_refusals():
    b = ref.make_batch(113, [20, 4], [10, 0], 4, 2, 64)
    c = Calls(b)
    err = binding.SparseEngineError
    with pytest.raises(err):
        binding.se_chunk_attend(c.p, b.q, b.cu[:-1], b.k_cache, b.v_cache, b.page_table, b.seq_lens, c.out, c.ws)
    with pytest.raises(err):
        binding.se_chunk_attend(c.p, b.q.float(), b.cu, b.k_cache, b.v_cache, b.page_table, b.seq_lens, c.out, c.ws)
    with pytest.raises(err):
        binding.se_chunk_attend(c.p, b.q, b.cu, b.k_cache[1:], b.v_cache, b.page_table, b.seq_lens, c.out, c.ws)
    with pytest.raises(err):
        binding.se_chunk_attend(c.p, b.q[:, :, ::2], b.cu, b.k_cache, b.v_cache, b.page_table, b.seq_lens, c.out, c.ws)
    with pytest.raises(err):
        binding.se_chunk_attend(c.p, b.q, b.cu, b.k_cache, b.v_cache, b.page_table, b.seq_lens, c.out, c.ws[:256 - 16])
    with pytest.raises(err):
        binding.se_prompt_attend(c.p, b.q, b.k[:-1], b.v, b.cu, c.out, c.ws)
    with pytest.raises(err):
        binding.se_prompt_attend(c.p, b.q, b.k, b.v, b.cu, c.out.float(), c.ws)
    with pytest.raises(err):
        binding.se_h2o_accumulate(c.p, b.q, b.cu, b.k_cache, b.page_table, b.seq_lens, c.lse[1:], torch.zeros(b.P, 2, 16, device="cuda"), c.ws)
    assert c.status() == 0
    empty = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    binding.se_chunk_attend(c.p, empty, b.cu, b.k_cache, b.v_cache, b.page_table, b.seq_lens, empty, c.ws)      # no rows: nothing to do


def test_equal_inputs_give_equal_bits_on_any_stream_and_in_graphs():
    b = ref.make_batch(121, [200, 3, 1], [2100, 5000, 700], 8, 2, 128)
    c = Calls(b)
    lse = ref.attend(b)[2].float()
    u = torch.zeros(b.P, 2, 16, device="cuda")
    c.chunk()
    c.mass(lse, u)
    out, l0, u0 = c.out.clone(), c.lse.clone(), u.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.out.fill_(NAN)
        c.chunk()
        u.zero_()
        c.mass(lse, u)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, c.out) and torch.equal(l0, c.lse) and torch.equal(u0, u)
    graphs = []
    for _ in range(2):                               # two captured steps that share the workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.chunk()
            u.zero_()
            c.mass(lse, u)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            c.out.fill_(NAN)
            u.fill_(NAN)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, c.out) and torch.equal(l0, c.lse) and torch.equal(u0, u)
    assert c.status() == 0


def test_a_replayed_graph_follows_changed_lengths():
    b = ref.make_batch(122, [30, 10, 24], [70, 300, 0], 8, 2, 64)
    c = Calls(b)
    c.chunk()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.chunk()
    for new in ([1, 60, 3], [0, 0, 64], [40, 0, 24]):
        b.new = new
        b.cu[1:] = torch.cumsum(torch.tensor(new), 0).to("cuda")
        b.total = [max(n, t) for n, t in zip(new, [100, 310, 24])]
        b.total = [min(t, 16 * int((b.page_table[r] >= 0).sum())) for r, t in enumerate(b.total)]
        b.new = [min(n, t) for n, t in zip(new, b.total)]
        b.cu[1:] = torch.cumsum(torch.tensor(b.new), 0).to("cuda")
        b.seq_lens.copy_(torch.tensor(b.total))
        b.k_cache.nan_to_num_(0.5)
        b.v_cache.nan_to_num_(0.5)
        c.out.fill_(NAN)
        c.lse.fill_(NAN)
        g.replay()
        torch.cuda.synchronize()
        out, tol, lse, ltol = ref.attend(b)
        held(c.lse, lse, ltol, "lse")
        held(c.out, out, tol, "out")


def test_calls_at_once_on_two_streams_give_the_same_bits():
    # large enough for pieces that CTAs take as they become free; each stream has its workspace
    b = ref.make_batch(131, [600, 1] * 12 + [1, 2] * 4 + [37], [1400, 4000] * 12 + [4100, 900] * 4 + [0], 32, 8, 64)
    first = Calls(b)
    first.chunk()
    u0 = torch.zeros(b.P, 8, 16, device="cuda")
    first.mass(first.lse, u0)
    torch.cuda.synchronize()
    sides = [(Calls(b), torch.zeros_like(u0), torch.cuda.Stream()) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        for c, u, stream in sides:
            with torch.cuda.stream(stream):
                c.out.fill_(NAN)
                u.zero_()
                c.chunk()
                c.mass(c.lse, u)
    torch.cuda.synchronize()
    for c, u, _ in sides:
        assert torch.equal(c.out, first.out) and torch.equal(c.lse, first.lse) and torch.equal(u, u0)
        assert c.status() == 0


def test_a_page_read_twice_and_by_two_requests():
    # an aliased prefix, and one physical page at two logical positions
    b = ref.make_batch(132, [20, 30], [300, 500], 8, 2, 128)
    b.page_table[1, :10] = b.page_table[0, :10]
    b.page_table[1, 12] = b.page_table[1, 11]
    check_attention(Calls(b))


def test_largest_batch_of_short_requests():
    n = 8192
    b = ref.make_batch(133, [r % 3 for r in range(n)], [0 if r % 5 else 20 for r in range(n)], 2, 1, 64, spare=2)
    c = Calls(b)
    c.chunk()
    torch.cuda.synchronize()
    assert c.status() == 0
    pick = [0, 1, 2, 5, 95, 96, 97, 4096, 8189, 8190, 8191]
    want = {}
    for r in pick:                       # the reference goes request by request: only some of them
        one = ref.Batch(b.H_q, b.H_kv, b.D, [b.new[r]], [b.total[r]], b.new[r], b.max_pages, b.P, b.qkv[b.rows(r)],
                        None, None, b.page_table[r:r + 1], b.k_cache, b.v_cache)
        want[r] = ref.attend(one)
    for r, (out, tol, lse, ltol) in want.items():
        rows = b.rows(r)
        held(c.lse[rows], lse, ltol, "lse of request %d" % r)
        held(c.out[rows], out, tol, "out of request %d" % r)
    assert bool(c.out[:sum(b.new)].isfinite().all()) and bool(c.out[sum(b.new):].isnan().all())
    u = torch.zeros(b.P, 1, 16, device="cuda")
    c.mass(c.lse[:b.T].clone(), u)
    assert abs(float(u.double().sum()) - sum(b.new) * 2) < 1e-4 * sum(b.new) * 2
