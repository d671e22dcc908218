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


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("heads,kv,d,n", [(4, 2, 64, 300), (17, 1, 128, 300), (4, 1, 128, 9000)])
def test_cache_mean_of_equal_values(ctx, dtype, heads, kv, d, n):
    """A mean of equal values is that value, by one block and by many, with probabilities that are rounded up."""
    import torch
    dt, block = getattr(torch, dtype), 32
    # keys of 0 and of -1, a query of 1: the scale is the score against the latter, its exponential just past a tie above 1/2
    scale = -math.log(0.5 + 1.02 * 2.0 ** (-9 if dt == torch.bfloat16 else -12))
    q = torch.zeros(1, heads, d, dtype=dt, device="cuda")
    q[..., 0] = 1
    k, v = torch.zeros(n, kv, d, dtype=dt, device="cuda"), torch.full((n, kv, d), 1.5, dtype=dt, device="cuda")
    k[..., 0] = -1
    k[::32, :, 0] = 0                                        # (one in every tile)
    pages = -(-n // block)
    codes = torch.zeros(pages, kv, 2, block, d // 2, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(pages, kv, 2, d // 32, block, dtype=torch.uint8, device="cuda")
    ctx.cache_append(k, v, torch.arange(n, device="cuda"), codes, scales)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages)
    out = torch.zeros_like(q)
    need = ctx.cache_attention_workspace_bytes(1, heads, kv, d, pages * block)
    ctx.cache_attention(q, codes, scales, table, torch.tensor([n], dtype=torch.int32, device="cuda"), out,
                        torch.empty(need, dtype=torch.uint8, device="cuda") if need else None, scale=scale)
    assert (out == 1.5).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("heads,kv,d,nq,nk,at", [(4, 2, 64, 700, 700, 5), (4, 2, 128, 700, 700, 300), (2, 1, 128, 3, 5000, 100), (2, 1, 64, 3, 5000, 4999),
                                                 (128, 8, 128, 512, 5000, 5), (128, 8, 128, 512, 5000, 4900)])
@pytest.mark.parametrize("score", [0.0, -200.0])
def test_prompt_infinite_value(ctx, dtype, heads, kv, d, nq, nk, at, score):
    """An infinity gives every row that sees it the same, whether the row sees all of the key's tile or not: an infinity, or a NaN
    where its probability is zero."""
    import torch
    dt = getattr(torch, dtype)
    q, k, v = (torch.zeros(n, h, d, dtype=dt, device="cuda") for n, h in ((nq, heads), (nk, kv), (nk, kv)))
    q[..., 0], k[at, :, 0] = 1, score
    k[at, 0, 0] = 0                                                # (not for the heads of the first KV head)
    v[at, :, 3], v[at, :, d - 1] = math.inf, -math.inf
    out = torch.zeros_like(q)
    ctx.prompt_attention(q, k, v, _starts(torch, [nq]), _starts(torch, [nk]), out, scale=1.0)
    sees = torch.arange(nq, device="cuda") + nk - nq >= at
    want = torch.zeros_like(out)
    want[sees, :, 3], want[sees, :, d - 1] = math.inf, -math.inf
    if score < 0:
        want[sees, heads // kv:, 3], want[sees, heads // kv:, d - 1] = math.nan, math.nan
    assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.nan_to_num(1), want.nan_to_num(1))
