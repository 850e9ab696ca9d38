"""The bounded waits of the 8-bit cache's kernels: a copy that never completes ends in SE_DEV_WAIT_TIMEOUT, not in a hang.

In the second build of the library (``-DSE_TEST_SHORT_TX``) the first copy of one kind of every CTA (decode: of every warp's first
page; chunk attention: K's first tile at D = 64, V's first pages at D = 128) announces 16 bytes more than it delivers.  Whoever
needs it gives up after the limit, the others follow, copies in flight are waited for - bounded again - and the kernel returns."""
import ctypes
import time

import pytest
import torch

from paper_2609_39068_b200 import _build, binding
from test_gpu_kv8 import Chunk, Decode

pytestmark = pytest.mark.gpu


@pytest.fixture
def short(monkeypatch):
    """Switches the binding to the build whose copies announce too much, and back."""
    lib = ctypes.CDLL(_build.build_short_tx())
    product = binding.load()
    for name in ("se_kv8_decode", "se_kv8_chunk_attend"):
        f = getattr(lib, name)
        f.argtypes, f.restype = getattr(product, name).argtypes, ctypes.c_int
    for name in ("se_prompt_workspace_bytes", "se_strerror"):       # the workspace's size and state are the product's business
        setattr(lib, name, getattr(product, name))

    def run(call):
        with monkeypatch.context() as m:
            m.setattr(binding, "_lib", lib)
            t0 = time.perf_counter()
            call()
            torch.cuda.synchronize()                                # returns: the kernel gave up by itself
            return time.perf_counter() - t0
    return run


@pytest.mark.parametrize("make", [
    lambda: Decode(3, [40, 700], 2, 4, 64), lambda: Decode(3, [30000] * 8, 8, 4, 128), lambda: Decode(3, [100] * 300, 2, 8, 128),
    lambda: Chunk(3, [40, 3], [100, 200], 2, 4, 128), lambda: Chunk(3, [300, 5], [20000, 30000], 2, 4, 128),
    lambda: Chunk(3, [40, 3], [100, 200], 2, 4, 64), lambda: Chunk(3, [300, 5], [20000, 30000], 2, 3, 64),
    lambda: Chunk(3, [64] * 100 + [1] * 20, [1950] * 110 + [2500] * 10, 8, 4, 128),
])
def test_wait_that_never_completes_times_out(short, make):
    c = make()
    c.run()
    good = c.out.clone(), c.lse.clone()
    assert binding.se_last_device_status(c.ws) == 0
    elapsed = short(c.run)
    assert 0.15 < elapsed < 10.0, elapsed                           # a few wait limits, not forever
    assert binding.se_last_device_status(c.ws) == binding.SE_DEV_WAIT_TIMEOUT
    binding.se_prompt_workspace_init(c.p, c.ws)
    for _ in range(2):
        c.run()
        assert binding.se_last_device_status(c.ws) == 0
        assert torch.equal(c.out.view(torch.int8), good[0].view(torch.int8)) and torch.equal(c.lse.view(torch.int8), good[1].view(torch.int8))


def test_the_mark_of_a_workspace():
    """A workspace that has to be initialised again: the calls write nothing and say so; set from the host."""
    for c in (Decode(5, [40, 700], 2, 4, 64), Chunk(5, [20, 1], [30, 0], 2, 4, 64)):
        c.ws[:8].view(torch.int32)[1] = 1
        c.run()
        assert binding.se_last_device_status(c.ws) == binding.SE_DEV_WAIT_TIMEOUT and bool(c.out.isnan().all())
        binding.se_prompt_workspace_init(c.p, c.ws)
        c.check()


def test_the_mark_of_a_pages_workspace():
    i32 = dict(dtype=torch.int32, device="cuda")
    p = binding.make_params(2, 4, 4, 64, 3, 10, 1)
    ws = binding.alloc_pages_workspace(p)
    table, lens, refs, one = torch.full((2, 3), -1, **i32), torch.zeros(2, **i32), torch.zeros(10, **i32), torch.full((1,), 77, **i32)
    ws[:8].view(torch.int32)[1] = 1
    binding.se_pages_update(p, table, lens, refs, lens + 5, table, lens, refs, one, ws)
    assert binding.se_last_device_status(ws) == binding.SE_DEV_WAIT_TIMEOUT and one.tolist() == [77] and lens.tolist() == [0, 0]
    binding.se_pages_compact(p, table, lens, refs, table, refs, torch.zeros_like(refs), one, ws)
    assert binding.se_last_device_status(ws) == binding.SE_DEV_WAIT_TIMEOUT and one.tolist() == [77]
    binding.se_pages_workspace_init(p, ws)
    binding.se_pages_update(p, table, lens, refs, lens + 5, table, lens, refs, one, ws)
    assert binding.se_last_device_status(ws) == 0 and one.tolist() == [8] and lens.tolist() == [5, 5] and table[:, 0].tolist() == [0, 1]
