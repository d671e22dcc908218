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


def _split_work(torch, ctx, gen):
    """Calls whose parts are kept in the context's memory or a workspace: f(inputs) -> outputs, and their inputs.  A product whose k
    is split, prompt attention of few queries and of one long sequence among many, cache attention in parts."""
    (ac, as_), (wc, ws) = (ref.quantise(torch.randn(r, 8192, generator=gen, device="cuda"), bits) for r, bits in ((93, 8), (512, 4)))
    starts = lambda n: torch.tensor([0, *np.cumsum(n)], dtype=torch.int32, device="cuda")  # noqa: E731
    few, many = ([3], [5000]), ([1] * 70, [9] * 69 + [30000])
    kv, block, lengths = 2, 16, [5000, 0, 700]
    pages = sum(-(-n // block) for n in lengths)
    cache = torch.randint(0, 256, (pages, kv, 2, block, 64), generator=gen, device="cuda", dtype=torch.uint8), \
        torch.randint(120, 130, (pages, kv, 2, 4, block), generator=gen, device="cuda", dtype=torch.uint8)
    table = torch.randint(0, pages, (3, 400), generator=gen, device="cuda", dtype=torch.int32)
    room = torch.empty(ctx.cache_attention_workspace_bytes(3, 8, kv, 128, 400 * block), dtype=torch.uint8, device="cuda")
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    starts_few, starts_many = [starts(n) for n in few], [starts(n) for n in many]

    def product(a, out):
        ctx.product(a, as_, wc, ws, out)

    def prompt(starts):
        return lambda q, k, v, out: ctx.prompt_attention(q, k, v, *starts, out)

    def cached(q, out):
        ctx.cache_attention(q, *cache, table, lens, out, room)
    heads = lambda n, h: torch.randn(n, h, 128, generator=gen, device="cuda").half()  # noqa: E731
    calls = [(product, [ac]), (prompt(starts_few), [heads(3, 8), heads(5000, 2), heads(5000, 2)]),
             (prompt(starts_many), [heads(70, 8), heads(30621, 2), heads(30621, 2)]), (cached, [heads(3, 8)])]
    outs = lambda: [torch.full((93, 512), math.nan, dtype=torch.float16, device="cuda"), *(torch.full_like(c[1][0], math.nan) for c in calls[1:])]  # noqa: E731
    return calls, outs


def test_split_work_on_several_streams(ctx):
    """Calls in turn on two streams, whose parts lie in the same memory: the bits of the same calls on one."""
    import torch
    calls, outs = _split_work(torch, ctx, torch.Generator("cuda").manual_seed(1))
    want = outs()
    for (call, inputs), out in zip(calls, want):
        call(*inputs, out)
    torch.cuda.synchronize()
    assert not any(o.isnan().any() for o in want)
    sides = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        got = [outs() for _ in sides]
        torch.cuda.synchronize()
        for i, (call, inputs) in enumerate(calls):
            for which in range(2):
                with torch.cuda.stream(sides[(i + which) % 2]):
                    call(*inputs, got[which][i])
        torch.cuda.synchronize()
        for each in got:
            assert all(torch.equal(a, b) for a, b in zip(want, each))


def test_split_work_in_a_graph(ctx):
    """Replays with other work of the context in between, checked each time against the calls themselves."""
    import torch
    gen = torch.Generator("cuda").manual_seed(2)
    calls, outs = _split_work(torch, ctx, gen)
    side, kept = torch.cuda.Stream(), outs()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for (call, inputs), out in zip(calls, kept):
            call(*inputs, out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for (call, inputs), out in zip(calls, kept):
                call(*inputs, out)
    torch.cuda.synchronize()
    for _ in range(4):
        for _, inputs in calls:
            for t in inputs:
                t.copy_(t.flatten()[torch.randperm(t.numel(), generator=gen, device="cuda")].view(t.shape))
        want = outs()
        for (call, inputs), out in reversed(list(zip(calls, want))):
            call(*inputs, out)
        for out in kept:
            out.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, kept))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("m,n,k", [(17, 40, 32), (64, 70, 64), (90, 130, 480), (300, 700, 128), (70, 300, 512), (129, 9000, 96), (1300, 7000, 32), (93, 200, 8224), (130, 129, 1056)])
def test_product_reads_its_operands_alone(ctx, bits, m, n, k):
    """Operands in the middle of memory that is no number wherever it is read: behind every row, before the first and after the last.  The
    same bits as from operands by themselves."""
    import torch
    gen = torch.Generator("cuda").manual_seed(m + k)
    (ac, as_), (wc, ws) = (ref.quantise(torch.randn(r, k, generator=gen, device="cuda"), b) for r, b in ((m, bits), (n, 4)))

    def inside(t, pad):
        big = torch.full((t.shape[0] + 300, t.shape[1] + pad), 255, dtype=torch.uint8, device="cuda")
        big[150:150 + t.shape[0], :t.shape[1]] = t
        return big[150:150 + t.shape[0], :t.shape[1]]
    want, got = (torch.full((m, n), math.nan, dtype=torch.float16, device="cuda") for _ in range(2))
    ctx.product(ac, as_, wc, ws, want, bits=bits)
    ctx.product(inside(ac, 16), inside(as_, 5), inside(wc, 32), inside(ws, 1), got, bits=bits)
    assert torch.isfinite(want).all() and torch.equal(want, got)


@pytest.mark.parametrize("seed", [3, 4])
def test_decode_attends_to_every_token(ctx, seed):
    """The attention inside a decode pass of a layer, to within its own rounding: the tokens of the prefill pass and the new one."""
    import torch
    from paper_2412_04788_amd import measure, workloads as wl
    seen = []

    class Watched(measure.Layer):
        def __call__(self, x, residual, attend):
            def watch(q, k, v):
                out = attend(q, k, v)
                seen.append([t.clone() for t in (q, k, v, out)])
                return out
            return super().__call__(x, residual, watch)
    block, prompts = 16, [33, 1, 70]
    table, pages = measure.page_tables([n + 1 for n in prompts], block)
    layer = Watched(ctx, wl.Model("small", 1, 256, 4, 2, 448, V=32), pages, block, seed=seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    rows = lambda n: torch.randn(n, 256, generator=gen, device="cuda").bfloat16()  # noqa: E731
    slots = np.concatenate([measure.token_slots(table, np.full(n, i), np.arange(n), block) for i, n in enumerate(prompts)])
    layer.prefill(rows(104), rows(104), torch.tensor([0, 33, 34, 104], dtype=torch.int32, device="cuda"), torch.from_numpy(slots).cuda())
    new = measure.token_slots(table, np.arange(3), np.array(prompts), block)
    lengths = torch.tensor([n + 1 for n in prompts], dtype=torch.int32, device="cuda")
    layer.decode(rows(3), rows(3), torch.from_numpy(table).cuda(), lengths, torch.from_numpy(new).cuda())
    (_, k, v, _), (q, k1, v1, out) = seen
    held = lambda t: ref.decode(*ref.quantise(t.reshape(-1, t.shape[-1]), 4), 4, t.shape[-1]).view(t.shape)  # noqa: E731
    a = 0
    for i, n in enumerate(prompts):
        kk, vv = held(torch.cat((k[a:a + n], k1[i:i + 1]))), held(torch.cat((v[a:a + n], v1[i:i + 1])))
        want, size = ref.attention(q[i:i + 1], kk, vv, torch.ones(1, n + 1, dtype=torch.bool, device="cuda"), layer.d_h ** -0.5)
        err = (out[i:i + 1].double() - want).abs()
        bound = ref.attention_bound(want, size, vv, n + 1, torch.bfloat16)
        assert bool((err <= bound).all()), float((err / bound).max())
        a += n
