"""The bounded waits of the prompt-side kernels: a copy that never completes ends in SE_DEV_WAIT_TIMEOUT, not in a hang.

In the second build of the library (``-DSE_TEST_SHORT_TX``) one copy of every CTA announces 16 bytes more than it delivers: in
attention the first V tile (D = 128) or the first K tile (D = 64), in the accumulated weights the first query tile (D = 128) or the
first pair of K tiles (D = 64).  The warp that needs it gives up after the limit, the
other roles follow, the copying warps wait - bounded again - for what they still have in flight, and the kernel returns."""
import ctypes
import time

import pytest
import torch

import prompt_ref as ref
from paper_2609_39068_b200 import _build, binding
from test_gpu_prompt import Calls

pytestmark = pytest.mark.gpu

# (new, past): CTAs with a tile or two, whose copying warps have nothing left to do when the wait runs out; rings in full use;
# pieces that CTAs take as they become free
BATCHES = {
    "few_tiles": ([40, 3], [100, 200], 8, 2, 128),
    "many_tiles": ([300, 5], [20000, 30000], 8, 2, 128),
    "few_tiles_64": ([40, 3], [100, 200], 8, 2, 64),
    "many_tiles_64": ([300, 5], [20000, 30000], 6, 2, 64),
    "two_sizes": ([64] * 100 + [1] * 20, [1950] * 110 + [2500] * 10, 32, 8, 64),
}


@pytest.fixture
def short(monkeypatch):
    """Switches the binding to the build whose copies announce too much, and back."""
    lib = ctypes.CDLL(_build.build_short_tx())
    product = binding.load()
    for name in ("se_chunk_attend", "se_prompt_attend", "se_h2o_accumulate"):
        f = getattr(lib, name)
        f.argtypes, f.restype = getattr(product, name).argtypes, ctypes.c_int

    def run(call):
        with monkeypatch.context() as m:
            m.setattr(binding, "_lib", lib)
            t0 = time.perf_counter()
            call()
            torch.cuda.synchronize()          # returns: the kernel gave up by itself
            return time.perf_counter() - t0

    # the workspace's size and state are the product's business
    for name in ("se_prompt_workspace_bytes", "se_strerror"):
        setattr(lib, name, getattr(product, name))
    return run


def operators(b):
    c = Calls(b)
    lse = torch.zeros(b.T, b.H_q, device="cuda")
    u = torch.zeros(b.P, b.H_kv, 16, device="cuda")

    def chunk():
        c.chunk()
        return c.out, c.lse

    def prompt():
        c.prompt()
        return c.out, c.lse

    def mass():
        u.zero_()
        c.mass(lse, u)
        return (u,)

    return c, {"chunk": chunk, "prompt": prompt, "mass": mass}


@pytest.mark.parametrize("name", sorted(BATCHES))
@pytest.mark.parametrize("op", ["chunk", "prompt", "mass"])
def test_wait_that_never_completes_times_out(short, name, op):
    new, past, H_q, H_kv, D = BATCHES[name]
    b = ref.make_batch(3, new, past, H_q, H_kv, D, nan_tail=False)
    c, ops = operators(b)
    good = [x.clone() for x in ops[op]()]
    torch.cuda.synchronize()
    assert c.status() == 0
    elapsed = short(ops[op])
    assert 0.15 < elapsed < 10.0, elapsed     # a few wait limits, not forever
    assert c.status() == binding.SE_DEV_WAIT_TIMEOUT
    binding.se_prompt_workspace_init(c.p, c.ws)
    for _ in range(2):
        again = ops[op]()
        torch.cuda.synchronize()
        assert c.status() == 0
        assert all(torch.equal(x, y) for x, y in zip(good, again))


@pytest.mark.parametrize("op", ["chunk", "prompt", "mass"])
def test_after_a_timeout_calls_refuse_until_the_workspace_is_initialised(short, op):
    new, past, H_q, H_kv, D = BATCHES["two_sizes"]
    b = ref.make_batch(3, new, past, H_q, H_kv, D, nan_tail=False)
    c, ops = operators(b)
    good = [x.clone() for x in ops[op]()]
    short(ops[op])
    assert c.status() == binding.SE_DEV_WAIT_TIMEOUT and c.status() == 0      # the reading has cleared the word ...
    for _ in range(2):
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
        outputs = ops[op]()
        torch.cuda.synchronize()
        assert c.status() == binding.SE_DEV_WAIT_TIMEOUT                      # ... but the workspace is not fit for use
        assert all(bool((x == (0.0 if op == "mass" else 7.0)).all()) for x in outputs)
    binding.se_prompt_workspace_init(c.p, c.ws)
    again = ops[op]()
    torch.cuda.synchronize()
    assert c.status() == 0 and all(torch.equal(x, y) for x, y in zip(good, again))


def test_the_mark_is_the_workspace_s_own():
    # set from the host; a workspace beside it goes on, and the append, which counts nothing, goes on with the marked one
    b = ref.make_batch(4, [20, 1], [30, 0], 8, 2, 64)
    marked, other = Calls(b), Calls(b)
    marked.ws[:8].view(torch.int32)[1] = 1
    marked.chunk()
    other.chunk()
    torch.cuda.synchronize()
    assert marked.status() == binding.SE_DEV_WAIT_TIMEOUT and bool(marked.out.isnan().all())
    assert other.status() == 0 and bool(other.out.isfinite().all())
    pos = torch.zeros(1, b.T, dtype=torch.int32, device="cuda")
    freq, axis = torch.ones(32, dtype=torch.float64, device="cuda"), torch.zeros(32, dtype=torch.int32, device="cuda")
    binding.se_rope_append(marked.p, b.q, b.k, b.v, b.cu, b.seq_lens, b.page_table, pos, freq, axis, marked.out, b.k_cache.clone(),
                           b.v_cache.clone(), marked.ws)
    assert marked.status() == 0 and torch.equal(marked.out, b.q)
