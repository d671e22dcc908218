"""The layer operators at sizes that one launch does not hold, and at the ends of their stated limits."""
import math

import pytest

from tests import layer_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2412_04788_amd import guide
    return guide.Context(0)


@pytest.fixture(autouse=True)
def memory():
    """Tens of gigabytes each: given back before the next."""
    import torch
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def _repeats(torch, got, pattern):
    """Whether the rows of `got` are those of `pattern` over and over."""
    step = (1 << 24) // len(pattern) * len(pattern)
    want = pattern.repeat(step // len(pattern), 1)
    return all(torch.equal(part, want[:len(part)]) for part in got.split(step))


@pytest.mark.parametrize("rows,cols", [((1 << 30) - 1, 1), ((1 << 25) - 1, 1000)])
def test_quantise_of_nearly_2_30_groups(ctx, rows, cols):
    import torch
    some = torch.randn(1009, cols, generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    for part in x.split(1009 << 10):
        part.copy_(some.repeat(1 << 10, 1)[:len(part)])
    groups = -(-cols // 32)
    codes = torch.full((rows, groups * 16), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, groups), 0xAA, dtype=torch.uint8, device="cuda")
    ctx.quantise(x, codes, scales, bits=4)
    want_c, want_s = ref.quantise(some, 4)
    assert _repeats(torch, codes, want_c) and _repeats(torch, scales, want_s)


@pytest.mark.parametrize("rows,d", [((1 << 26) + 3, 1), ((1 << 24) + 5, 1025)])
def test_norm_of_more_rows_than_a_launch_holds(ctx, rows, d):
    """Rows of a wave each, and rows of a block each."""
    import torch
    few = 1009
    gen = torch.Generator("cuda").manual_seed(d)
    some, weight = torch.randn(few, d, generator=gen, device="cuda").half(), torch.randn(d, generator=gen, device="cuda").half()
    x = torch.empty(rows, d, dtype=torch.float16, device="cuda")
    for part in x.split(few << 10):
        part.copy_(some.repeat(1 << 10, 1)[:len(part)])
    groups = -(-d // 32)
    new = lambda n: (torch.full((n, groups * 16), 0xAA, dtype=torch.uint8, device="cuda"), torch.full((n, groups), 0xAA, dtype=torch.uint8, device="cuda"))  # noqa: E731
    want, (codes, scales) = new(few), new(rows)
    ctx.rms_norm(x, weight, codes, scales, residual=x, total=x, bits=4)
    ctx.rms_norm(2 * some, weight, *want, bits=4)
    assert _repeats(torch, codes, want[0]) and _repeats(torch, scales, want[1])
    assert _repeats(torch, x, 2 * some)


def _starts(torch, counts):
    return torch.cat((torch.zeros(1, dtype=torch.int64), torch.tensor(counts).cumsum(0))).int().cuda()


@pytest.mark.parametrize("heads,kv", [(4096, 8), (4100, 1)])
def test_prompts_of_more_blocks_than_a_launch_holds(ctx, heads, kv):
    """4096 sequences of one token, thousands of heads: every head gives its token's value."""
    import torch
    n, d = 4096, 64
    gen = torch.Generator("cuda").manual_seed(heads)
    k, v = (torch.randn(n, kv, d, generator=gen, device="cuda").half() for _ in range(2))
    q = torch.ones(1, heads, d, dtype=torch.float16, device="cuda").repeat(n, 1, 1)
    out = torch.full_like(q, math.nan)
    starts = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    ctx.prompt_attention(q, k, v, starts, starts, out)
    assert torch.equal(out, v.repeat_interleave(heads // kv, 1))


def test_prompts_most_of_which_are_empty(ctx):
    """2^20 sequences of which 128 have a token (with 4096 heads, tiles times heads pass 2^32 if the empty ones count)."""
    import torch
    n, heads, d = 128, 4096, 64
    gen = torch.Generator("cuda").manual_seed(3)
    k, v = (torch.randn(n, 1, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    q = torch.ones(n, heads, d, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, math.nan)
    starts = _starts(torch, [1] * n + [0] * ((1 << 20) - n))
    ctx.prompt_attention(q, k, v, starts, starts, out)
    assert torch.equal(out, v.expand(n, heads, d))


def test_more_tokens_than_a_launch_holds(ctx):
    """2^28 tokens to append and read back, all but the last 1000 of them outside the cache."""
    import torch
    n, d, block, few = (1 << 28) + 7, 128, 16, 1000
    codes = torch.zeros(64, 1, 2, block, d // 2, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(64, 1, 2, d // 32, block, dtype=torch.uint8, device="cuda")
    slots = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    slots[n - few:] = torch.randperm(64 * block, generator=torch.Generator("cuda").manual_seed(2), device="cuda")[:few]
    x = torch.empty(n, 1, d, dtype=torch.bfloat16, device="cuda")                   # 69 GB: keys and values alike
    x[n - few:] = torch.randn(few, 1, d, generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    held = ref.decode(*ref.quantise(x[n - few:, 0], 4), 4, d)
    ctx.cache_append(x, x, slots, codes, scales)
    x.fill_(7)
    ctx.cache_read(slots, codes, scales, x, x)
    assert torch.equal(x[n - few:, 0].double(), held)
    assert not any(part.any() for part in x[:n - few].view(torch.int16).split(1 << 24))


def test_counts_that_32_bits_do_not_hold(ctx):
    """2^32 rows are not none (one row's memory stands for all of them)."""
    import torch
    n = 1 << 32
    rows = lambda c, dt: torch.zeros(1, c, dtype=dt, device="cuda").expand(n, c)  # noqa: E731
    x, w, codes, scales = rows(1, torch.bfloat16), torch.ones(1, dtype=torch.bfloat16, device="cuda"), rows(16, torch.uint8), rows(1, torch.uint8)
    one = torch.zeros(1, 16, dtype=torch.uint8, device="cuda"), torch.zeros(1, 1, dtype=torch.uint8, device="cuda")
    heads = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    many, starts = heads.expand(n, 1, 64), torch.zeros(2, dtype=torch.int32, device="cuda")
    cache = torch.zeros(1, 1, 2, 16, 32, dtype=torch.uint8, device="cuda"), torch.zeros(1, 1, 2, 2, 16, dtype=torch.uint8, device="cuda")
    slots = torch.zeros(1, dtype=torch.int64, device="cuda").expand(n)
    for call in (lambda: ctx.quantise(x, codes, scales, bits=4), lambda: ctx.rms_norm(x, w, codes, scales, bits=4),
                 lambda: ctx.product(codes, scales, *one, x, bits=4), lambda: ctx.product(*one, codes, scales, x.t(), bits=4),
                 lambda: ctx.prompt_attention(many, heads, heads, starts, starts, many), lambda: ctx.prompt_attention(heads, many, many, starts, starts, heads),
                 lambda: ctx.cache_append(many, many, slots, *cache), lambda: ctx.cache_read(slots, *cache, many, many),
                 lambda: ctx.cache_attention(many, *cache, starts[:1].expand(n, 1), starts[:1].expand(n), many)):
        with pytest.raises(ValueError):
            call()


def test_as_many_sequences_as_there_may_be(ctx):
    """2^20 sequences of one token each: their blocks find them in much less time than a walk over them takes (minutes)."""
    import torch
    n, heads, d = 1 << 20, 8, 64
    gen = torch.Generator("cuda").manual_seed(5)
    k, v = (torch.randn(n, 1, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    q = torch.ones(1, heads, d, dtype=torch.bfloat16, device="cuda").expand(n, heads, d).contiguous()
    out = torch.full_like(q, math.nan)
    starts = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    ctx.prompt_attention(q, k, v, starts, starts, out)
    assert torch.equal(out, v.expand(n, heads, d))
