"""A query row as the sum of two rows of codes (se_kv8_chunk_attend): what the header says of its precision, in exact arithmetic."""
import torch

import kv8_ref as ref


def split(x, top):
    """hi + lo of ``x`` in a row whose largest magnitude is ``top`` (fp64)."""
    e = torch.ceil(torch.log2(top / 448.0))
    e = torch.where(top <= 448.0 * torch.exp2(e - 1), e - 1, e)
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)
    hi = ref.nearest_code(x / torch.exp2(e))
    return (hi + ref.nearest_code(x / torch.exp2(e) - hi)) * torch.exp2(e)


def test_bounds_of_the_split():
    mantissas = torch.arange(128, 256, dtype=torch.float64)          # the significands of bf16
    tops = (mantissas * 2.0 ** 1)[:, None, None]
    x = (mantissas[:, None] * torch.exp2(torch.arange(-24, 2, dtype=torch.float64))).expand(128, -1, -1)
    x = torch.where(x <= tops, x, torch.zeros_like(x))
    err = (split(x, tops) - x).abs()
    assert float(err[(x >= tops / 896)].max()) == 0.0
    assert float((err / tops).max()) <= 2.0 ** -17.8
    # below: 227 * 2^-10 in a row with the maximum 226 lies above 2^-10 of it and is off by 2^-10
    far, top = torch.tensor([227.0 * 2.0 ** -10], dtype=torch.float64), torch.tensor([226.0], dtype=torch.float64)
    assert float(far / top) > 2.0 ** -10 and float((split(far, top) - far).abs()) == 2.0 ** -10
