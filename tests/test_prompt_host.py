"""Prompt-side calls: what they refuse before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2609_39068_b200 import binding

OK, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4100)
P = binding.make_params(2, 32, 8, 128, 64, 128, 1)
PP = ctypes.byref(P)

# name -> (valid argument list, positions of required pointers, positions of optional pointers)
CALLS = {
    "se_rope_append": ([PP, OK, 4096, OK, 1024, OK, 1024, 4, OK, OK, OK, OK, 3, OK, OK, 128, 0, ctypes.c_void_p(8192), None, OK, OK,
                        None, OK, None], [1, 3, 5, 8, 9, 10, 11, 13, 14, 17, 19, 20, 22], [18, 21]),
    "se_chunk_attend": ([PP, OK, 4096, 4, OK, OK, OK, OK, OK, OK, None, OK, None], [1, 4, 5, 6, 7, 8, 9, 11], [10]),
    "se_prompt_attend": ([PP, OK, 4096, OK, 1024, OK, 1024, 4, OK, OK, None, OK, None], [1, 3, 5, 8, 9, 11], [10]),
    "se_h2o_accumulate": ([PP, OK, 4096, 4, OK, OK, OK, OK, OK, OK, OK, None], [1, 4, 5, 6, 7, 8, 9, 10], []),
}


def call(name, args):
    return getattr(binding.load(), name)(*args)


def changed(name, at, value):
    args = list(CALLS[name][0])
    args[at] = value
    return args


@pytest.mark.parametrize("name", sorted(CALLS))
def test_null_and_misaligned_pointers(name):
    _, required, optional = CALLS[name]
    for i in required:
        assert call(name, changed(name, i, None)) == -3, i
        assert call(name, changed(name, i, ODD)) == -4, i
    for i in optional:
        assert call(name, changed(name, i, ODD)) == -4, i


@pytest.mark.parametrize("name,strides,total", [("se_rope_append", [(2, 4096), (4, 1024), (6, 1024)], 7), ("se_chunk_attend", [(2, 4096)], 3),
                                                ("se_prompt_attend", [(2, 4096), (4, 1024), (6, 1024)], 7), ("se_h2o_accumulate", [(2, 4096)], 3)])
def test_strides_and_row_counts(name, strides, total):
    for at, least in strides:
        for bad in (least - 8, least + 4, -least, 1 << 40):
            assert call(name, changed(name, at, bad)) == -1, (at, bad)
    assert call(name, changed(name, total, -1)) == -1
    assert call(name, changed(name, total, 0)) == 0                # nothing to do, nothing launched


def test_rope_argument_ranges():
    for at, bad in ((12, 0), (12, 5), (15, 0), (15, 8), (15, 136), (15, 144), (16, 2)):
        assert call("se_rope_append", changed("se_rope_append", at, bad)) == -1, (at, bad)
    args = changed("se_rope_append", 17, OK)                      # in place ...
    args[2] = 6144                                                # ... on a strided view
    assert call("se_rope_append", args) == -1


@pytest.mark.parametrize("kw", [dict(D=96), dict(H_q=72), dict(B=0), dict(B=8193), dict(max_pages=0), dict(page_size=32)])
def test_invalid_params(kw):
    base = dict(B=2, H_q=32, H_kv=8, D=128, max_pages=64, num_phys_pages=128, k_max=1, page_size=16)
    base.update(kw)
    p = binding.make_params(**base)
    assert binding.se_prompt_workspace_bytes(p) == 0
    assert binding.load().se_prompt_workspace_init(ctypes.byref(p), OK, None) in (-1, -2)
    for name in CALLS:
        assert call(name, changed(name, 0, ctypes.byref(p))) in (-1, -2)
        assert call(name, changed(name, 0, None)) == -3


def test_workspace_is_pure():
    n = binding.se_prompt_workspace_bytes(P)
    assert n > 0 and n % 256 == 0 and n == binding.se_prompt_workspace_bytes(P)
    assert binding.load().se_prompt_workspace_init(PP, None, None) == -3
    assert binding.load().se_prompt_workspace_init(PP, ODD, None) == -4


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    x = torch.zeros(3, 32, 128, dtype=torch.bfloat16)
    with pytest.raises(binding.SparseEngineError):
        binding._rows(x, 32, 128, "q")
    with pytest.raises(binding.SparseEngineError):
        binding._shape(x, [3, 32, 64], "q")


def test_shapes_are_compared_by_value():
    x = torch.zeros(3, 32, 128, dtype=torch.bfloat16)
    binding._shape(x, (3, 32, 128), "q")
    binding._shape(None, (3, 32, 128), "lse")
    for bad in ((3, 32, 64), (3, 32), (3, 32, 128, 1), (4, 32, 128), ()):
        with pytest.raises(binding.SparseEngineError, match=r"q must have shape \["):
            binding._shape(x, bad, "q")


def test_rotated_keys_in_place_of_a_strided_view():
    # k_out may be k itself only where the rows of both lie at the same places
    args = changed("se_rope_append", 18, OK)
    args[3], args[4] = OK, 6144
    assert call("se_rope_append", args) == -1
