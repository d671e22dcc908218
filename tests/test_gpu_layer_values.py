"""Attention at values where the order or the width of its arithmetic shows: the type's greatest, infinities."""
import math

import pytest

from tests import layer_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2412_04788_amd import guide
    return guide.Context(0)


def _starts(torch, lengths):
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("heads,kv,d,nq,nk", [(4, 2, 64, 700, 700), (4, 2, 128, 700, 700), (2, 1, 128, 1, 5000), (2, 1, 64, 3, 5000), (128, 8, 128, 512, 5000)])
def test_prompt_greatest_values(ctx, heads, kv, d, nq, nk):
    """Values of 65504 give 65504, by whole kernels, split ones and large tiles, with probabilities that round up."""
    import torch
    x = torch.arange(0.55, 0.69, 2.0 ** -11, dtype=torch.float64).half().double()
    up = x[(((-x).exp().half().double() / (-x).exp()) - 1).argmax()]                 # e^-x is rounded up most: by nearly 2^-11
    q, k, v = (torch.zeros(n, h, d, dtype=torch.float16, device="cuda") for n, h in ((nq, heads), (nk, kv), (nk, kv)))
    q[..., 0], k[..., 0] = 1, -float(up)
    k[::128, :, 0] = 0                                       # (the greatest score of every part of the keys)
    v[..., ::2], v[..., 1::2] = 65504, -65504
    out = torch.zeros_like(q)
    ctx.prompt_attention(q, k, v, _starts(torch, [nq]), _starts(torch, [nk]), out, scale=1.0)
    assert (out[..., ::2] == 65504).all() and (out[..., 1::2] == -65504).all()
