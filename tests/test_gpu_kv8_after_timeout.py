"""After a wait that gave up a workspace has to be initialised again: until then its calls write nothing and say so each time.

Here decode sets that mark itself, in the build of the bounded waits' tests (``-DSE_TEST_SHORT_TX``): its first pages never come."""
import ctypes
import time

import pytest
import torch

from paper_2609_39068_b200 import _build, binding
from test_gpu_kv8 import Chunk, Decode

pytestmark = pytest.mark.gpu


@pytest.fixture
def short(monkeypatch):
    lib, product = ctypes.CDLL(_build.build_short_tx()), binding.load()
    for name in ("se_kv8_decode",):
        f = getattr(lib, name)
        f.argtypes, f.restype = getattr(product, name).argtypes, ctypes.c_int
    for name in ("se_prompt_workspace_bytes", "se_strerror"):
        setattr(lib, name, getattr(product, name))

    def run(call):
        with monkeypatch.context() as m:
            m.setattr(binding, "_lib", lib)
            t0 = time.perf_counter()
            call()
            torch.cuda.synchronize()
            return time.perf_counter() - t0
    return run


@pytest.mark.parametrize("make", [lambda: Decode(3, [40, 700], 2, 4, 64), lambda: Decode(3, [100] * 300, 2, 8, 128)])
def test_decode_marks_its_workspace(short, make):
    c = make()
    c.run()
    good = c.out.clone(), c.lse.clone()
    assert 0.15 < short(c.run) < 10.0
    assert binding.se_last_device_status(c.ws) == binding.SE_DEV_WAIT_TIMEOUT
    chunk = Chunk(5, [20, 1], [30, 0], 2, 4, 64)
    chunk.ws = c.ws if c.ws.numel() >= chunk.ws.numel() else chunk.ws
    for call, out in ((c, c.out), (c, c.out), (chunk, chunk.out)):
        if call is chunk and chunk.ws is not c.ws:
            continue
        out.fill_(7.0)
        call.run()                                                   # the status has been read: only the mark is left
        assert binding.se_last_device_status(c.ws) == binding.SE_DEV_WAIT_TIMEOUT
        assert bool((out == 7.0).all())
    binding.se_prompt_workspace_init(c.p, c.ws)
    for _ in range(2):
        c.run()
        assert binding.se_last_device_status(c.ws) == 0 and torch.equal(c.out, good[0]) and torch.equal(c.lse, good[1])
