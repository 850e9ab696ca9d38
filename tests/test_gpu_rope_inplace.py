"""se_rope_append writing over its own inputs."""
import pytest
import torch

import prompt_ref as ref
from paper_2609_39068_b200 import binding
from test_gpu_prompt import Calls, held, rope_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,rot,inter", [(128, 128, False), (64, 32, True)])
def test_queries_and_keys_in_place(D, rot, inter):
    b = ref.make_batch(116, [50, 1, 17], [3, 40, 0], 4, 2, D)
    c = Calls(b)
    pos, inv_freq, axis = rope_inputs(b, 2, rot, 9)
    q, k = b.q.contiguous(), b.k.contiguous()
    want = [ref.rotate(x, pos, inv_freq, axis, inter) for x in (q, k)]
    caches = b.k_cache.clone(), b.v_cache.clone()
    k_out = torch.empty_like(k)
    rest = (b.cu, b.seq_lens, b.page_table, pos, inv_freq, axis)
    binding.se_rope_append(c.p, b.q, b.k, b.v, *rest, torch.empty_like(q), *caches, c.ws, k_out=k_out, interleaved=inter)
    binding.se_rope_append(c.p, q, k, b.v, *rest, q, b.k_cache, b.v_cache, c.ws, k_out=k, interleaved=inter)
    assert c.status() == 0
    for got, (x, tol), name in ((q, want[0], "q"), (k, want[1], "k")):
        held(got, x, tol, name + " in place")
    assert torch.equal(k, k_out)
    assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(caches, (b.k_cache, b.v_cache)))
    # a strided k of several rows has no place for its own rotated rows
    wide = torch.zeros(b.T, 4, D, dtype=torch.bfloat16, device="cuda")
    clash = wide.view(-1)[:b.T * 2 * D].view(b.T, 2, D)
    with pytest.raises(binding.SparseEngineError):
        binding.se_rope_append(c.p, q, wide[:, :2], b.v, *rest, q, b.k_cache, b.v_cache, c.ws, k_out=clash, interleaved=inter)
