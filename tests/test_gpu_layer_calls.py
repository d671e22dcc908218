"""How the layer operators are called: tensors of one row or token as torch leaves them, streams, captured calls."""
import math

import numpy as np
import pytest

from tests import layer_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2412_04788_amd import guide
    return guide.Context(0)


def _buffers(torch, rows, cols, bits):
    g = -(-cols // 32)
    return (torch.full((rows, g * 4 * bits), 0xAA, dtype=torch.uint8, device="cuda"),
            torch.full((rows, g), 0xAA, dtype=torch.uint8, device="cuda"))


def test_one_row_that_was_a_column(ctx):
    """A column that is turned round is contiguous to torch, whatever the stride of its only row says."""
    import torch
    gen = torch.Generator("cuda").manual_seed(0)
    turned = lambda t: t.new_empty(t.shape[1], 1).copy_(t.t()).t().contiguous()  # noqa: E731
    x, w = torch.randn(1, 96, generator=gen, device="cuda").half(), torch.ones(96, dtype=torch.float16, device="cuda")
    wc, ws = ref.quantise(torch.randn(5, 96, generator=gen, device="cuda"), 4)
    got = []
    for form in (lambda t: t, turned):
        a, b = _buffers(torch, 1, 96, 8), _buffers(torch, 1, 96, 4)
        a, b, total, out = [form(t) for t in a], [form(t) for t in b], form(torch.zeros_like(x)), form(torch.zeros(1, 5, dtype=torch.float16, device="cuda"))
        assert form is not turned or x.shape == form(x).shape and form(x).stride(0) == 1 and a[0].stride(0) == 1
        ctx.rms_norm(form(x), w, *a, residual=form(x), total=total)
        ctx.product(*a, wc, ws, out)
        ctx.quantise(form(x), *b, bits=4)
        got.append((*a, *b, total, out))
    for one, other in zip(*got):
        assert torch.equal(one, other)
    # one sequence's pages
    codes, scales = torch.full((3, 1, 2, 16, 32), 0x22, dtype=torch.uint8, device="cuda"), torch.full((3, 1, 2, 2, 16), 127, dtype=torch.uint8, device="cuda")
    q, out = torch.ones(1, 1, 64, dtype=torch.float16, device="cuda"), torch.zeros(1, 1, 64, dtype=torch.float16, device="cuda")
    pages = turned(torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda"))
    ctx.cache_attention(q, codes, scales, pages, torch.tensor([40], dtype=torch.int32, device="cuda"), out)
    assert (out == 1).all()


@pytest.mark.parametrize("tokens", [9, 700])
def test_append_with_tokens_to_skip_and_tokens_that_share_a_slot(ctx, tokens):
    """Tokens outside the cache are skipped; what shares a slot stays in that slot."""
    import torch
    kv, d, block, pages = 3, 64, 16, -(-tokens // 16) + 1
    gen = torch.Generator("cuda").manual_seed(tokens)
    k, v = (torch.randn(tokens, kv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    slots = torch.randperm(pages * block, generator=gen, device="cuda")[:tokens]
    slots[::3] = -1
    slots[tokens // 2] = pages * block
    shared = int(slots[1])
    slots[tokens - 1], k[tokens - 1] = shared, k[tokens - 1] * 1024
    keep = (slots >= 0) & (slots < pages * block) & (slots != shared)
    codes = torch.full((pages, kv, 2, block, d // 2), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((pages, kv, 2, d // 32, block), 0xFF, dtype=torch.uint8, device="cuda")
    want = codes.clone(), scales.clone()
    page, at = slots[keep] // block, slots[keep] % block
    for which, x in enumerate((k[keep], v[keep])):
        c, s = ref.quantise(x.reshape(-1, d), 4)
        want[0][page, :, which, at], want[1][page, :, which, :, at] = c.view(-1, kv, d // 2), s.view(-1, kv, d // 32)
    ctx.cache_append(k, v, slots, codes, scales)
    for got, right in ((codes.transpose(3, 4), want[0].transpose(3, 4)), (scales, want[1])):
        got[shared // block, ..., shared % block] = 0
        right[shared // block, ..., shared % block] = 0
        assert torch.equal(got, right)


def test_measuring_leaves_the_context_alone(ctx):
    """The caller's models and hardware answer as before after a measurement on the same context."""
    import torch
    from paper_2412_04788_amd import guide, measure, workloads as wl
    g = wl.grid_tiny()
    ctx.set_models(wl.models_array(g.models))
    ctx.set_hardware(wl.hw_array(g.hws))
    grid = guide.GridArg([(a.values, a.geom2_start) for a in g.axes])

    def answers():
        out = {k: torch.zeros(g.size, dtype=torch.float64, device="cuda") for k in ("t_prefill", "t_decode")}
        ctx.eval_grid(grid, 0, g.size, out=out)
        return out
    before = answers()
    small = wl.Model("small", 1, 256, 4, 2, 448, V=32)
    measure.efficiency_samples(ctx, small, wl.Hardware(1e12, 1e12, 1e12, 1e12), [40, 24], 3, 50, 16, repeats=1)
    after = answers()
    assert all(torch.equal(before[k], after[k]) for k in before)


def test_measured_times_are_the_cards(ctx):
    """What the host does between the calls of a pass is not in its times; a pass of more work takes longer."""
    import time
    import torch
    from paper_2412_04788_amd import measure
    x = torch.randn(4096, 4096, device="cuda").bfloat16()
    codes, scales = _buffers(torch, 4096, 4096, 4)

    def run(times):
        def call():
            for _ in range(times):
                time.sleep(0.02)
                ctx.quantise(x, codes, scales, bits=4)
        return call
    one, many = measure._seconds(run(1), 5), measure._seconds(run(10), 5)
    assert one.shape == many.shape == (5,)
    assert (one > 0).all() and np.median(many) < 0.02 and np.median(many) > 3 * np.median(one)


@pytest.mark.parametrize("seqs,length", [(16, 4000), (1, 700), (3, 513), (2, 0)])
def test_cache_attention_is_split_by_lengths_not_by_tables(ctx, seqs, length):
    """With a table of 131 072 tokens a sequence's keys go to as many blocks as with one that it fills: so many parts of every row are
    written to the workspace, which starts with the parts' maxima."""
    import torch
    kv, heads, d, block = 8, 32, 128, 32
    pages = -(-max(length, 1) // block)
    codes = torch.full((pages, kv, 2, block, d // 2), 0x22, dtype=torch.uint8, device="cuda")
    scales = torch.full((pages, kv, 2, d // 32, block), 127, dtype=torch.uint8, device="cuda")
    q, lengths = torch.ones(seqs, heads, d, device="cuda").bfloat16(), torch.full((seqs,), length, dtype=torch.int32, device="cuda")
    for width in (pages, 4096):
        table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(seqs, -(-width // pages))[:, :width].contiguous()
        need, out = ctx.cache_attention_workspace_bytes(seqs, heads, kv, d, width * block), torch.zeros_like(q)
        room = torch.full((max(need // 4, 1),), math.nan, device="cuda")
        ctx.cache_attention(q, codes, scales, table, lengths, out, room)
        assert (out == (1 if length else 0)).all()
        parts = (~room[:need // (4 * (d + 2))].view(seqs * heads, -1).isnan()).sum(1)
        if need:
            assert (parts == max(1, -(-length // 512))).all(), (width, parts)
