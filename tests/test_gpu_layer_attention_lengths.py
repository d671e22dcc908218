"""Prompt attention over sequences of very different lengths, where long ones are split over blocks and short ones are not."""
import math

import pytest

from tests import layer_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2412_04788_amd import guide
    return guide.Context(0)


def _starts(torch, lengths):
    return torch.cat((torch.zeros(1, dtype=torch.int64), torch.tensor(lengths).cumsum(0))).int().cuda()


# queries and keys of every sequence: fewer blocks than the chip runs (all of them may be split) and more (those of up to 128
# queries may be), rows without keys, sequences without queries or keys, queries up to a tile and beyond
CASES = {
    "one_long": ([1] * 15 + [1], [100] * 15 + [30000]),
    "one_long_first": ([3] + [1] * 30, [26000] + [5] * 30),
    "decode_and_segment": ([1] * 20 + [500] + [1] * 10, [500 + 37 * i for i in range(20)] + [3000] + [9000 - 700 * i for i in range(10)]),
    "tiles": ([128, 129, 127, 1, 0, 256, 2], [9001, 9000, 12000, 7, 400, 100, 0]),
    "more_queries_than_keys": ([100, 128, 90, 60], [20, 0, 20011, 33]),
    "all_split": ([2, 130, 1], [4000, 6000, 300]),
    "no_queries_in_most": ([0] * 70 + [1] + [0] * 20 + [5], [3] * 70 + [17000] + [0] * 20 + [800]),
    "mean_of_unused_rows": ([1], [9000]),
}


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("heads,kv,d", [(32, 8, 128), (40, 4, 64), (20, 20, 128), (8, 1, 64)])
@pytest.mark.parametrize("case", CASES)
def test_prompts_of_different_lengths(ctx, dtype, heads, kv, d, case):
    import torch
    q_len, k_len = CASES[case]
    spare = 700 if case == "mean_of_unused_rows" else 0                    # rows of no sequence, which the host's mean counts
    tq, tk = sum(q_len), sum(k_len)
    gen = torch.Generator("cuda").manual_seed(tk)
    dt = getattr(torch, dtype)
    q, k, v = (torch.randn(n, h, d, generator=gen, device="cuda").to(dt) for n, h in ((tq + spare, heads), (tk, kv), (tk, kv)))
    out = torch.full_like(q, math.nan)
    args = _starts(torch, q_len), _starts(torch, k_len)
    ctx.prompt_attention(q, k, v, *args, out)
    a = b = 0
    for nq, nk in zip(q_len, k_len):
        sees = torch.arange(nk, device="cuda")[None] <= torch.arange(nq, device="cuda")[:, None] + nk - nq
        want, size = ref.attention(q[a:a + nq], k[b:b + nk], v[b:b + nk], sees, d ** -0.5)
        err = (out[a:a + nq].double() - want).abs()
        bound = ref.attention_bound(want, size, v[b:b + nk], nk, dt)
        assert bool((err <= bound).all()), (nq, nk, float((err / bound).max()))
        a, b = a + nq, b + nk
    assert out[tq:].isnan().all()
    again = torch.zeros_like(out)
    ctx.prompt_attention(q, k, v, *args, again)
    assert torch.equal(out[:tq], again[:tq])


def test_a_long_sequence_among_short_ones_is_split(ctx):
    """One query each: 15 over 100 keys and one over 60 000 take no more than a few times what 16 over 4000 do."""
    import torch
    heads, kv, d = 32, 8, 128

    def best(k_len):
        n, tk = len(k_len), sum(k_len)
        q, k = torch.randn(n, heads, d, device="cuda").bfloat16(), torch.randn(tk, kv, d, device="cuda").bfloat16()
        out, starts = torch.empty_like(q), (_starts(torch, [1] * n), _starts(torch, k_len))
        times = []
        for _ in range(20):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            ctx.prompt_attention(q, k, k, *starts, out)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    # whole it takes as long as 60 000 / 4000 = 15 times one of those, in parts of a sixteenth as long as one
    assert best([100] * 15 + [60000]) < 4 * best([4000] * 16)


MANY = {      # heads, KV heads, channels; queries and keys of every sequence; how many sequences to one that is checked
    "short": (4, 2, 64, [i % 6 for i in range(3000)], [(i * 7) % 11 for i in range(3000)], 1),
    "empty_ones_around": (8, 8, 128, [0] * 1000 + [2, 0, 150] * 3 + [0] * 1000, [1] * 1000 + [3, 5, 400] * 3 + [0] * 1000, 1),
    "one_long": (32, 8, 128, [1] * 500, [3] * 440 + [40000] + [5] * 59, 1),
    "few_queries": (2, 1, 64, [0] * 500 + [2, 130], [9] * 500 + [9000, 7000], 1),
    "long_ones": (64, 1, 128, [3] * 400, [4100 + i for i in range(400)], 37),
}


@pytest.mark.parametrize("case", MANY)
def test_many_sequences(ctx, case):
    """Hundreds to thousands of sequences, which blocks find by a table."""
    import torch
    heads, kv, d, q_len, k_len, every = MANY[case]
    gen = torch.Generator("cuda").manual_seed(7)
    q, k, v = (torch.randn(n, h, d, generator=gen, device="cuda").bfloat16() for n, h in ((sum(q_len), heads), (sum(k_len), kv), (sum(k_len), kv)))
    out = torch.full_like(q, math.nan)
    ctx.prompt_attention(q, k, v, _starts(torch, q_len), _starts(torch, k_len), out)
    assert not out.isnan().any()
    a = b = 0
    for i, (nq, nk) in enumerate(zip(q_len, k_len)):
        if nq and i % every == 0:
            sees = torch.arange(nk, device="cuda")[None] <= torch.arange(nq, device="cuda")[:, None] + nk - nq
            want, size = ref.attention(q[a:a + nq], k[b:b + nk], v[b:b + nk], sees, d ** -0.5)
            err, bound = (out[a:a + nq].double() - want).abs(), ref.attention_bound(want, size, v[b:b + nk], nk, torch.bfloat16)
            assert bool((err <= bound).all()), (i, nq, nk, float((err / bound).max()))
        a, b = a + nq, b + nk
