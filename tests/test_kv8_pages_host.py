"""The calls of the 8-bit cache and of the page pool: what they refuse before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

import pages_ref
from paper_2609_39068_b200 import binding

OK, ODD, OTHER = ctypes.c_void_p(4096), ctypes.c_void_p(4100), ctypes.c_void_p(8192)
P = binding.make_params(2, 32, 8, 128, 64, 128, 4)
PP = ctypes.byref(P)
ONE = (binding.SePageBuffer * 1)(binding.SePageBuffer(4096, 64))

# name -> (valid argument list, positions of required pointers, positions of optional pointers)
CALLS = {
    "se_kv8_append": ([PP, OK, 4096, OK, 1024, OK, 1024, 4, OK, OK, OK, OK, 3, OK, OK, 128, 0, OTHER, None, OK, OK, OK, None, OK, None],
                      [1, 3, 5, 8, 9, 10, 11, 13, 14, 17, 19, 20, 21, 23], [18, 22]),
    "se_kv8_decode": ([PP, OK, OK, OK, OK, OK, OK, OK, OK, OK, OK, OK, None], [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11], []),
    "se_kv8_chunk_attend": ([PP, OK, 4096, 4, OK, OK, OK, OK, OK, OK, OK, None, OK, None], [1, 4, 5, 6, 7, 8, 9, 10, 12], [11]),
    "se_pages_update": ([PP, OK, OK, OK, None, OK, OTHER, OTHER, OK, OK, ONE, 1, OK, None], [1, 2, 3, 5, 6, 7, 8, 9, 12], [4]),
    "se_pages_compact": ([PP, OK, OK, OK, OK, OK, OK, OK, ONE, 1, OK, None], [1, 2, 3, 4, 5, 6, 7, 10], []),
}


def call(name, args):
    return getattr(binding.load(), name)(*args)


def changed(name, *changes):
    args = list(CALLS[name][0])
    for at, value in changes:
        args[at] = value
    return args


@pytest.mark.parametrize("name", sorted(CALLS))
def test_null_and_misaligned_pointers(name):
    _, required, optional = CALLS[name]
    for i in required:
        assert call(name, changed(name, (i, None))) == -3, i
        assert call(name, changed(name, (i, ODD))) == -4, i
    for i in optional:
        assert call(name, changed(name, (i, ODD))) == -4, i


@pytest.mark.parametrize("name,strides,total", [("se_kv8_append", [(2, 4096), (4, 1024), (6, 1024)], 7), ("se_kv8_chunk_attend", [(2, 4096)], 3)])
def test_strides_and_row_counts(name, strides, total):
    for at, least in strides:
        for bad in (least - 8, least + 4, -least, 1 << 40):
            assert call(name, changed(name, (at, bad))) == -1, (at, bad)
    assert call(name, changed(name, (total, -1))) == -1
    assert call(name, changed(name, (total, 0))) == 0              # nothing to do, nothing launched


def test_append_argument_ranges():
    for at, bad in ((12, 0), (12, 5), (15, 0), (15, 8), (15, 136), (15, 144), (16, 2)):
        assert call("se_kv8_append", changed("se_kv8_append", (at, bad))) == -1, (at, bad)
    assert call("se_kv8_append", changed("se_kv8_append", (17, OK), (2, 6144))) == -1        # q in place on a strided view
    assert call("se_kv8_append", changed("se_kv8_append", (18, OK), (4, 6144))) == -1        # k too


def test_decode_wants_both_of_a_selection():
    assert call("se_kv8_decode", changed("se_kv8_decode", (7, None))) == -3
    assert call("se_kv8_decode", changed("se_kv8_decode", (8, None))) == -3


@pytest.mark.parametrize("name,at", [("se_pages_update", 10), ("se_pages_compact", 8)])
def test_page_buffers(name, at):
    buffers = lambda base, size: (binding.SePageBuffer * 1)(binding.SePageBuffer(base, size))  # noqa: E731
    for n in (-1, 513):
        assert call(name, changed(name, (at + 1, n))) == -1
    assert call(name, changed(name, (at, None))) == -3
    assert call(name, changed(name, (at, buffers(None, 64)))) == -3
    assert call(name, changed(name, (at, buffers(4100, 64)))) == -4
    for size in (0, -16, 2, 66, (1 << 30) + 4):
        assert call(name, changed(name, (at, buffers(4096, size)))) == -1, size


def test_update_with_parents_wants_outputs_of_its_own():
    for at, same in ((6, OK), (7, OK)):
        assert call("se_pages_update", changed("se_pages_update", (4, OK), (at, same))) == -1


@pytest.mark.parametrize("kw", [dict(D=96), dict(H_q=72), dict(B=0), dict(B=8193), dict(max_pages=0), dict(page_size=32), dict(num_phys_pages=0)])
def test_invalid_params(kw):
    base = dict(B=2, H_q=32, H_kv=8, D=128, max_pages=64, num_phys_pages=128, k_max=4, page_size=16)
    base.update(kw)
    p = binding.make_params(**base)
    assert binding.se_pages_workspace_bytes(p) == 0
    assert binding.load().se_pages_workspace_init(ctypes.byref(p), OK, None) in (-1, -2)
    for name in CALLS:
        assert call(name, changed(name, (0, ctypes.byref(p)))) in (-1, -2)
        assert call(name, changed(name, (0, None))) == -3


def test_pages_workspace_is_pure():
    n = binding.se_pages_workspace_bytes(P)
    assert n > 24 * P.num_phys_pages and n % 256 == 0 and n == binding.se_pages_workspace_bytes(P)
    assert binding.load().se_pages_workspace_init(PP, None, None) == -3
    assert binding.load().se_pages_workspace_init(PP, ODD, None) == -4


def test_binding_refusals():
    i32, codes = dict(dtype=torch.int32), torch.zeros(128, 8, 16, 128, dtype=torch.float8_e4m3fn)
    ws = torch.zeros(binding.se_pages_workspace_bytes(P), dtype=torch.uint8)
    table, lens, refs, one = torch.zeros(2, 64, **i32), torch.zeros(2, **i32), torch.zeros(128, **i32), torch.zeros(1, **i32)
    args = [P, table, lens, refs, lens, table, lens, refs, one, ws]
    for at, bad in ((1, torch.zeros(2, 63, **i32)), (2, torch.zeros(3, **i32)), (3, one), (4, one), (5, lens), (6, one), (7, one), (8, lens)):
        with pytest.raises(binding.SparseEngineError, match="must have shape"):
            binding.se_pages_update(*[bad if i == at else x for i, x in enumerate(args)])
    with pytest.raises(binding.SparseEngineError, match="workspace is smaller"):
        binding.se_pages_update(*args[:-1], ws[:100])
    with pytest.raises(binding.SparseEngineError, match="page buffers must be contiguous CUDA tensors"):
        binding.page_buffers([codes])
    prompt_ws = torch.zeros(binding.se_prompt_workspace_bytes(P), dtype=torch.uint8)
    q, out, lse, scales = torch.zeros(2, 32, 128, dtype=torch.bfloat16), torch.zeros(2, 32, 128), torch.zeros(2, 32), torch.zeros(128, 8, 2)
    args = [P, q, codes, codes, scales, table, lens, out, lse, prompt_ws]
    for at, bad in ((1, q[:1]), (2, codes[:5]), (4, scales[..., 0]), (7, out[:, :3]), (8, lse[:1])):
        with pytest.raises(binding.SparseEngineError, match="must have shape"):
            binding.se_kv8_decode(*[bad if i == at else x for i, x in enumerate(args)])
    with pytest.raises(binding.SparseEngineError, match="must be a CUDA tensor"):
        binding.se_kv8_decode(*args)


def test_the_one_page_form_itself():
    """pages_ref on a case that can be followed by hand: a fork, its copy on write, an end and a compaction."""
    table, lens, refs = [[5, 2, -1], [-1] * 3], [20, 0], [0, 0, 1, 0, 0, 1]
    table, lens, refs, free, copies = pages_ref.update(table, lens, refs, [21, 33], [0, 0])
    assert table == [[5, 2, -1], [5, 0, 1]] and copies == [(2, 0)] and refs == [1, 1, 1, 0, 0, 2] and free == 2
    table, lens, refs, free, copies = pages_ref.update(table, lens, refs, [0, 33], [-1, 1])
    assert table == [[-1] * 3, [5, 0, 1]] and refs == [1, 1, 0, 0, 0, 1] and free == 3 and copies == []
    table, refs, where, n, moves = pages_ref.compact(table, lens, refs)
    assert table[1] == [2, 0, 1] and refs == [1, 1, 1, 0, 0, 0] and where == [0, 1, -1, -1, -1, 2] and n == 3 and moves == [(5, 2)]
