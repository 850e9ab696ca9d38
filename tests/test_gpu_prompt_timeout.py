"""The bounded waits of the prompt-side kernels: a copy that never completes ends in SE_DEV_WAIT_TIMEOUT, not in a hang.

In the second build of the library (``-DSE_TEST_SHORT_TX``) the first V tile of every CTA (attention) or its first query tile
(accumulated weights) announces 16 bytes more than its copies deliver.  The warp that needs it gives up after the limit, the
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
