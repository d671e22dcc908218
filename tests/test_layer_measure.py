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
