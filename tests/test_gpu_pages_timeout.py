"""The page calls' grid-wide barriers are bounded: in the build of the bounded waits' tests (``-DSE_TEST_SHORT_TX``) they wait for one
CTA more than there is, and the kernels return, report SE_DEV_WAIT_TIMEOUT and mark the workspace: until it is initialised again its
calls write nothing and say so each time."""
import ctypes
import time

import pytest
import torch

import pages_ref
from paper_2609_39068_b200 import _build, binding

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture
def short(monkeypatch):
    lib, product = ctypes.CDLL(_build.build_short_tx()), binding.load()
    for name in ("se_pages_update", "se_pages_compact"):
        f = getattr(lib, name)
        f.argtypes, f.restype = getattr(product, name).argtypes, ctypes.c_int
    for name in ("se_pages_workspace_bytes", "se_strerror"):
        setattr(lib, name, getattr(product, name))

    def run(call):
        with monkeypatch.context() as m:
            m.setattr(binding, "_lib", lib)
            t0 = time.perf_counter()
            call()
            torch.cuda.synchronize()
            return time.perf_counter() - t0
    return run


@pytest.mark.parametrize("buffers", [0, 2])
def test_grid_barriers_give_up(short, buffers):
    B, max_pages, P = 40, 100, 3000
    p = binding.make_params(B, 4, 4, 64, max_pages, P, 1)
    ws = binding.alloc_pages_workspace(p)
    pool = binding.page_buffers([torch.randint(0, 99, (P, 64), **I32) for _ in range(buffers)])
    table, lens, refs, free = torch.full((B, max_pages), -1, **I32), torch.zeros(B, **I32), torch.zeros(P, **I32), torch.full((1,), 77, **I32)
    new = torch.arange(B, **I32) * 37
    outs = [torch.full_like(t, 99) for t in (table, lens, refs)]
    where = torch.full_like(refs, 99)
    update = lambda: binding.se_pages_update(p, table, lens, refs, new, *outs, free, ws, buffers=pool)  # noqa: E731
    compact = lambda: binding.se_pages_compact(p, table, lens, refs, outs[0], outs[2], where, free, ws, buffers=pool)  # noqa: E731
    for call in (update, compact):
        assert 0.15 < short(call) < 10.0
        for again in (update, compact):
            assert binding.se_last_device_status(ws) == binding.SE_DEV_WAIT_TIMEOUT
            again()
        assert binding.se_last_device_status(ws) == binding.SE_DEV_WAIT_TIMEOUT
        assert all(bool((t == 99).all()) for t in outs + [where]) and free.tolist() == [77]
        binding.se_pages_workspace_init(p, ws)
    update()
    want = pages_ref.update(table.tolist(), lens.tolist(), refs.tolist(), new.tolist(), None)
    assert binding.se_last_device_status(ws) == 0 and free.tolist() == [want[3]]
    assert outs[0].tolist() == want[0] and outs[1].tolist() == new.tolist() and outs[2].tolist() == want[2]
