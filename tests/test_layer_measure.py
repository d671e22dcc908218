"""CPU-only: what measure.py prices a layer's passes at, against the performance model."""
import numpy as np
import pytest

from paper_2412_04788_amd import measure, workloads as wl

HWS = (wl.HW_TINY, wl.Hardware(2.5e15, 8e12, 288 * wl.GIB, 1e12), wl.Hardware(3e14, 6e12, 80 * wl.GIB, 1e12))


@pytest.mark.parametrize("model", [m for m in wl.MODELS_FULL if m.E == 1], ids=lambda m: m.name)
@pytest.mark.parametrize("batch,s_in", [(1, 128), (16, 700), (3, 4096)])
def test_roofline_is_the_models(ora, model, batch, s_in):
    """A prefill of equal prompts (whose every pair the model counts) and a decode step, to the last bits."""
    one = wl.Model("layer", 1, model.d, model.n_h, model.n_kv, model.d_ff, V=1)
    for hw in HWS:
        axes = [np.array([v], dtype=np.uint64) for v in (0, 0, batch, s_in, 2, 1, 4, 16, batch * s_in)]
        want = ora.eval_grid(ora.Grid(wl.models_array([one]), wl.hw_array([hw]), axes))
        head = lambda n: max(2 * n * model.d / hw.peak_flops, (0.5 * model.d + 2 * n * model.d + 2 * n) / hw.hbm_bw)  # noqa: E731
        prefill = measure.roofline(model, hw, batch * s_in, batch * s_in ** 2, batch * s_in) + head(batch)
        decode = measure.roofline(model, hw, batch, batch * (s_in + 1), batch * (s_in + 1)) + head(batch)
        np.testing.assert_allclose([prefill, decode], [want["t_prefill"][0], want["t_decode"][0]], rtol=1e-12)


def test_prompts_count_at_their_own_lengths():
    """Where operations are all that costs, a pass over prompts costs the products' and the visible pairs'."""
    m, hw = wl.DENSE_70B, wl.Hardware(1e15, 1e30, 1e12, 1e12)
    d_h = m.d // m.n_h
    product = 2 * (m.d * (m.n_h + 2 * m.n_kv) * d_h + m.n_h * d_h * m.d + 3 * m.d * m.d_ff)
    for prompts in ([1], [100, 8000], [700, 300, 1048], [5] * 40):
        visible = sum(i + 1 for n in prompts for i in range(n))
        want = (sum(prompts) * product + visible * 4 * m.n_h * d_h) / hw.peak_flops
        np.testing.assert_allclose(measure.nominal(m, hw, prompts, 1, 1)[0], want, rtol=1e-12)


def test_a_decode_step_is_priced_at_the_bytes_that_it_moves():
    """Where bytes are all that costs: weights and cached tokens at 17 / 32 of a byte a value, as their buffers are large."""
    from paper_2412_04788_amd import guide
    m, hw, batch, context, block = wl.DENSE_7B, wl.Hardware(1e30, 5e12, 1e12, 1e12), 16, 4096, 32
    table, pages = measure.page_tables([context] * batch, block)
    d_h, t = m.d // m.n_h, batch
    cache = pages * m.n_kv * 2 * block * (d_h // 2 + d_h // 32)
    weights = sum(n * (k // 2 + k // guide.MX_GROUP) for n, k in (((m.n_h + 2 * m.n_kv) * d_h, m.d), (m.d, m.n_h * d_h), (2 * m.d_ff, m.d), (m.d, m.d_ff)))
    # activations of two bytes: into and out of every product, q and o of the attention, four passes over the norms
    acts = 2 * t * ((m.d + (m.n_h + 2 * m.n_kv) * d_h) + 2 * m.n_h * d_h + (m.n_h * d_h + m.d) + (m.d + 2 * m.d_ff) + (m.d_ff + m.d) + 4 * m.d)
    want = (cache + weights + acts) / hw.hbm_bw
    np.testing.assert_allclose(measure.nominal(m, hw, [1], batch, context)[1], want, rtol=1e-12)


def test_the_command_measures_against_a_record_of_the_users():
    assert measure.arguments([])[1] == measure.CARD
    a, hw = measure.arguments(["--peak", "1e15", "--bandwidth", "5e12", "--batch", "3"])
    assert (hw.peak_flops, hw.hbm_bw, a.batch) == (1e15, 5e12, 3)
    for bad in (["--peak", "0"], ["--bandwidth", "-1"], ["--bandwidth", "nan"]):
        with pytest.raises(SystemExit):
            measure.arguments(bad)


def test_the_command_takes_as_many_samples_as_a_sweep():
    assert measure.arguments(["--repeats", "64"])[0].repeats == 64
    for bad in ("1", "65"):
        with pytest.raises(SystemExit):
            measure.arguments(["--repeats", bad])
