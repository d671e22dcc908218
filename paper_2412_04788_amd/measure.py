"""A decoder layer on the card, and the efficiency samples that its times give.

The performance model prices a layer's tasks at a card's peak and bandwidth, which a sweep multiplies by efficiency samples
(e_c, e_b).  This module runs those tasks -- norms, products with 4-bit weights, prompt attention, a paged 4-bit KV cache and
the attention of single tokens over it -- at a shape of the user's, and compares the time of a prefill pass and of a decode
pass with what the model's tasks would take at the record's rates for the work that these passes do (their own prompts, weights
and cache in 4 bits): e_c is the ratio for the prefill pass (compute bound), e_b for the decode pass (bandwidth bound).  The
pairs go into Context.eval_grid(e_c=..., e_b=...), whose configurations have the model's own widths.

    python -m paper_2412_04788_amd.measure --model dense-7b --prompts 700,300,1048 --batch 16 --context 4096
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import guide, workloads as wl

EPS = 1e-5
CARD = wl.Hardware(2.5e15, 8.0e12, 288 * wl.GIB, 1.53e11)     # MI355X: dense 16-bit matrix rate, HBM3E, one xGMI link
HELD = 17 / 32           # bytes of a value in 4-bit codes with a scale per 32


def _codes(rows: int, cols: int, bits: int):
    """Code and scale buffers of a matrix."""
    groups = -(-cols // guide.MX_GROUP)
    return (torch.empty(rows, groups * 4 * bits, dtype=torch.uint8, device="cuda"),
            torch.empty(rows, groups, dtype=torch.uint8, device="cuda"))


class Layer:
    """One dense decoder layer with random weights in 4-bit codes and its share of a paged 4-bit KV cache.  Positions are not
    encoded (the model prices no such task)."""

    def __init__(self, ctx: guide.Context, model: wl.Model, n_pages: int, kv_block: int, dtype=torch.bfloat16, seed: int = 0):
        if model.E != 1:
            raise ValueError("a dense layer: routed experts are not run here")
        self.ctx, self.model, self.dtype, self.kv_block = ctx, model, dtype, kv_block
        self.d_h = model.d // model.n_h
        self.q_width, self.kv_width = model.n_h * self.d_h, model.n_kv * self.d_h
        gen = torch.Generator("cuda").manual_seed(seed)
        shapes = dict(qkv=(self.q_width + 2 * self.kv_width, model.d), out=(model.d, self.q_width),
                      up=(2 * model.d_ff, model.d), down=(model.d, model.d_ff))
        self.weights = {}
        for name, (n, k) in shapes.items():
            w = (torch.randn(n, k, generator=gen, device="cuda") * k ** -0.5).to(dtype)
            self.weights[name] = _codes(n, k, 4)
            ctx.quantise(w, *self.weights[name], bits=4)
        self.norms = [torch.ones(model.d, dtype=dtype, device="cuda") for _ in range(2)]
        self.codes = torch.empty(n_pages, model.n_kv, 2, kv_block, self.d_h // 2, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(n_pages, model.n_kv, 2, self.d_h // 32, kv_block, dtype=torch.uint8, device="cuda")

    def _product(self, a, name: str):
        n = self.weights[name][0].shape[0]
        out = torch.empty(a[0].shape[0], n, dtype=self.dtype, device="cuda")
        self.ctx.product(*a, *self.weights[name], out)
        return out

    def _quantised(self, x):
        a = _codes(*x.shape, 8)
        self.ctx.quantise(x, *a, bits=8)
        return a

    def _normed(self, x, residual, which: int):
        a, total = _codes(*x.shape, 8), torch.empty_like(x)
        self.ctx.rms_norm(x, self.norms[which], *a, residual=residual, total=total, eps=EPS)
        return a, total

    def __call__(self, x, residual, attend):
        """(x, residual) -> the layer's two outputs of the same shapes; attend(q, k, v) gives the attention's."""
        m = self.model
        a, residual = self._normed(x, residual, 0)
        heads = self._product(a, "qkv").unflatten(-1, (m.n_h + 2 * m.n_kv, self.d_h))
        o = attend(heads[:, :m.n_h], heads[:, m.n_h:m.n_h + m.n_kv], heads[:, m.n_h + m.n_kv:])
        a, residual = self._normed(self._product(self._quantised(o.flatten(1)), "out"), residual, 1)
        gate, up = self._product(a, "up").chunk(2, -1)
        return self._product(self._quantised(torch.nn.functional.silu(gate) * up), "down"), residual

    def prefill(self, x, residual, starts, slots):
        """A pass over packed prompts: rows starts[s] .. of x; their keys and values go to the cache's slots."""
        def attend(q, k, v):
            out = torch.empty(q.shape, dtype=self.dtype, device="cuda")
            self.ctx.prompt_attention(q, k, v, starts, starts, out)
            self.ctx.cache_append(k, v, slots, self.codes, self.scales)
            return out
        return self(x, residual, attend)

    def decode(self, x, residual, pages, lengths, slots):
        """A pass over one new token per sequence, which lengths[s] counts and whose place in the cache is slots[s]."""
        def attend(q, k, v):
            self.ctx.cache_append(k, v, slots, self.codes, self.scales)
            out = torch.empty(q.shape, dtype=self.dtype, device="cuda")
            need = self.ctx.cache_attention_workspace_bytes(q.shape[0], q.shape[1], self.model.n_kv, self.d_h,
                                                            pages.shape[1] * self.kv_block)
            room = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
            self.ctx.cache_attention(q, self.codes, self.scales, pages, lengths, out, room)
            return out
        return self(x, residual, attend)


def page_tables(lengths, kv_block: int):
    """Consecutive pages for sequences of these lengths: (table [n_seq, max_pages] int32, number of pages)."""
    need = [-(-n // kv_block) for n in lengths]
    table, at = np.full((len(lengths), max(need)), -1, dtype=np.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = np.arange(at, at + n)
        at += n
    return table, at


def token_slots(table, sequence, position, kv_block: int):
    """Slots of tokens `position` of sequences `sequence` (arrays)."""
    return table[sequence, position // kv_block].astype(np.int64) * kv_block + position % kv_block


def _replays(run, passes: int, repeats: int):
    """Times of a pass in `repeats` replays, one after the other, of a graph of `passes` of them."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()                                                # (what is captured follows a call on the same stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for _ in range(passes):
                run()
        marks = [torch.cuda.Event(enable_timing=True) for _ in range(repeats + 1)]
        graph.replay(), graph.replay()
        marks[0].record()
        for m in marks[1:]:
            graph.replay()
            m.record()
        side.synchronize()
    return np.array([a.elapsed_time(b) * 1e-3 / passes for a, b in zip(marks, marks[1:])])


def _seconds(run, repeats: int):
    """Times of `repeats` passes as a program that captures them runs them: the host's part in the calls is not in them.  A replay
    costs the host some 40 us; of passes shorter than that a graph holds sixteen, and a time is their mean."""
    return _replays(run, 1 if np.median(_replays(run, 1, 5)) > 1e-4 else 16, repeats)


def roofline(model: wl.Model, hw: wl.Hardware, tokens: float, pairs: float, keys: float, weight_bytes: float = 0.5, kv_bytes: float = 2.0):
    """Seconds of one dense layer's tasks on one GPU at the record's rates, as guide.h's performance model has them (roofline): a pass
    over `tokens` tokens with `pairs` query-key pairs that reads `keys` cached tokens.  The widths, in bytes of a weight and of a
    cached element, are the model's at wbits = 4 unless others are given; activations are two bytes."""
    d, d_h, t = model.d, model.d // model.n_h, tokens
    dq, dkv, ff = model.n_h * d_h, model.n_kv * d_h, model.d_ff
    w = lambda n: weight_bytes * n  # noqa: E731
    tasks = ((2 * t * d * (dq + 2 * dkv), w(d * (dq + 2 * dkv)) + 2 * t * d + 2 * t * (dq + 2 * dkv)),      # qkv
             (4 * dq * pairs, 4 * t * dq + 2 * kv_bytes * dkv * keys),                                       # attention
             (2 * t * dq * d, w(dq * d) + 2 * t * dq + 2 * t * d),                                           # out-proj
             (4 * t * d * ff, w(2 * d * ff) + 2 * t * d + 4 * t * ff),                                       # ffn-up
             (2 * t * ff * d, w(ff * d) + 2 * t * ff + 2 * t * d),                                           # ffn-down
             (0, 8 * t * d))                                                                                 # norms
    return sum(max(f / hw.peak_flops, b / hw.hbm_bw) for f, b in tasks)


def nominal(model: wl.Model, hw: wl.Hardware, prompts, batch: int, context: int):
    """(prefill, decode) seconds, at the record's rates, of what the passes do: a pass over prompts of these lengths, whose queries see
    themselves and the keys before them (the sweep's model counts every pair of a prompt), and a step of `batch` tokens at
    `context` that reads its cache in 4 bits (the sweep's model: two bytes an element)."""
    tokens, pairs = sum(prompts), sum(n * (n + 1) / 2 for n in prompts)
    return (roofline(model, hw, tokens, pairs, tokens, HELD), roofline(model, hw, batch, batch * context, batch * context, HELD, HELD))


def efficiency_samples(ctx: guide.Context, model: wl.Model, hw: wl.Hardware, prompts, batch: int, context: int, kv_block: int = 32,
                       repeats: int = 16, dtype=torch.bfloat16):
    """Times of a prefill pass over `prompts` and of a decode pass of `batch` tokens at `context` cached ones, and the samples
    (e_c, e_b) that they give: a dict of arrays of `repeats`."""
    prompts = list(prompts)
    table, n_pages = page_tables([context] * batch, kv_block)
    fill, fill_pages = page_tables(prompts, kv_block)
    layer = Layer(ctx, model, max(n_pages, fill_pages), kv_block, dtype)
    gen = torch.Generator("cuda").manual_seed(1)
    rows = lambda n: torch.randn(n, model.d, generator=gen, device="cuda").to(dtype)
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()

    # the decode pass's cache: every slot filled with keys and values of unit size
    every = torch.arange(layer.codes.shape[0] * kv_block, device="cuda")
    for part in every.split(1 << 16):
        kv = torch.randn(len(part), model.n_kv, layer.d_h, generator=gen, device="cuda").to(dtype)
        ctx.cache_append(kv, kv, part, layer.codes, layer.scales)
    seqs = np.arange(batch)
    x, r = rows(batch), rows(batch)
    pages, lengths = cuda(table), cuda(np.full(batch, context, dtype=np.int32))
    new = cuda(token_slots(table, seqs, np.full(batch, context - 1), kv_block))
    t_decode = _seconds(lambda: layer.decode(x, r, pages, lengths, new), repeats)

    total = sum(prompts)
    starts = cuda(np.concatenate([[0], np.cumsum(prompts)]).astype(np.int32))
    slots = cuda(np.concatenate([token_slots(fill, np.full(n, i), np.arange(n), kv_block) for i, n in enumerate(prompts)]))
    px, pr = rows(total), rows(total)
    t_prefill = _seconds(lambda: layer.prefill(px, pr, starts, slots), repeats)

    m_prefill, m_decode = nominal(model, hw, prompts, batch, context)
    return dict(t_prefill=t_prefill, t_decode=t_decode, m_prefill=m_prefill, m_decode=m_decode, e_c=m_prefill / t_prefill,
                e_b=m_decode / t_decode)


def arguments(argv=None):
    """(options, hardware record) of the command line."""
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--model", default=wl.DENSE_7B.name, choices=[m.name for m in wl.MODELS_FULL if m.E == 1])
    ap.add_argument("--prompts", default="700,300,1048", help="prompt lengths of the prefill pass")
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--context", type=int, default=4096, help="cached tokens of a sequence in the decode pass, the new one among them")
    ap.add_argument("--kv-block", type=int, default=32)
    ap.add_argument("--repeats", type=int, default=16, help="samples, 2 to 64 (what a sweep takes)")
    ap.add_argument("--peak", type=float, default=CARD.peak_flops, help="FLOP/s of the record that the samples are relative to (the sweep's)")
    ap.add_argument("--bandwidth", type=float, default=CARD.hbm_bw, help="its bytes/s")
    a = ap.parse_args(argv)
    if not a.peak > 0 or not a.bandwidth > 0:
        ap.error("--peak and --bandwidth are above zero")
    if not 2 <= a.repeats <= 64:
        ap.error("--repeats: 2 to 64")
    return a, wl.Hardware(a.peak, a.bandwidth, CARD.cap_bytes, CARD.link_bw)


def main():
    a, hw = arguments()
    model, = [m for m in wl.MODELS_FULL if m.name == a.model]
    ctx = guide.Context(0)
    got = efficiency_samples(ctx, model, hw, [int(n) for n in a.prompts.split(",")], a.batch, a.context, a.kv_block, a.repeats)
    for name in ("prefill", "decode"):
        print(f"{name}: median {np.median(got['t_' + name]) * 1e6:.1f} us a layer, {got['m_' + name] * 1e6:.1f} us at the record's nominal rates")
    print(f"e_c median {np.median(got['e_c']):.3f}, e_b median {np.median(got['e_b']):.3f}")

    # a sweep on the measured samples
    g = wl.grid_tiny()
    ctx.set_models(wl.models_array([model]))
    ctx.set_hardware(wl.hw_array([hw]))
    grid = guide.GridArg([(x.values, x.geom2_start) for x in g.axes])
    stats = {k: torch.empty(g.size, dtype=torch.float64, device="cuda") for k in ("ttft_mean", "ttft_p10", "ttft_p90")}
    ctx.eval_grid(grid, 0, g.size, stats=stats, e_c=got["e_c"], e_b=got["e_b"])
    best = int(stats["ttft_mean"].argmin())
    print(f"least mean TTFT of {g.size} configurations: {stats['ttft_mean'][best]:.6f} s (p10 {stats['ttft_p10'][best]:.6f}, "
          f"p90 {stats['ttft_p90'][best]:.6f}) at index {best}")


if __name__ == "__main__":
    main()
