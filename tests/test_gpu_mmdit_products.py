"""The stand-in stack with its products and its cache through the library: both streams' products in one call (bf16, 4 bits),
the kept K and V in 4 bits.

Bounds.  bf16 products: those of the stack's test with library products (its arithmetic is bf16 either way).  4 bits: an element's
error is at most half a step, 1 / 6 of the largest of its block at worst and 1 / 8 of itself in the middle of the range, so the
relative error of a product of two such operands is below sqrt(2) / 8 = 0.18; four products lie between a block's input and its
output and the errors of different products are independent: 0.36 in all, tested at 0.5.  The 4-bit cache alone: V's error passes
through an average over keys, at most 1 / 8 of a row; tested at 0.25."""
import numpy as np
import pytest

from gpu_util import dev_bf16, host_f64
from oracle import mmdit_oracle, regione_oracle as orc
from paper_2510_25590_b200 import binding, loop as gloop, synth
from paper_2510_25590_b200.mmdit_scaffold import MMDiTScaffold

pytestmark = pytest.mark.gpu

H, D, C, L, N_TEXT = 2, 128, 16, 2, 40


def _setup(membership="paper", seed=3, **how):
    import torch
    wl = synth.scaled_workload(synth.WORKLOADS[4], grid=(16, 16), n_text=N_TEXT, heads=H)
    lat = synth.make_latents(wl, 0.20, stream=seed)
    ref, planted = lat["ref"], lat["mask"].astype(bool)
    w = synth.make_mmdit_weights(H * D, D, C, N_TEXT, L, seed=seed)
    cos, sin = synth.rope_tables(N_TEXT + 2 * wl.n_img, D)
    om = mmdit_oracle.MMDiTOracle(w, N_TEXT, wl.n_img, wl.n_img, H, D, L, cos, sin, ref, planted, membership)
    gm = MMDiTScaffold({k: dev_bf16(v) for k, v in w.items()}, N_TEXT, wl.n_img, wl.n_img, H, D, L,
                       torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), dev_bf16(ref),
                       torch.from_numpy(planted).cuda(),
                       binding.ROWS_PAPER if membership == "paper" else binding.ROWS_EDITED_QUERIES, **how)
    x = synth.bf16_round(np.random.default_rng(seed).standard_normal(ref.shape).astype(np.float32))
    return wl, om, gm, ref, planted, x


def _rel(got, want):
    return float(np.sqrt(np.mean((got - want) ** 2)) / np.sqrt(np.mean(want ** 2)))


def _steps(membership, **how):
    """Errors of a full step and of the region step behind it against the oracle's stack, inside the planted region."""
    wl, om, gm, ref, planted, x = _setup(membership, **how)
    t, dt = 0.75, 1.0 / 28.0
    lp = gloop.RegionELoop(1, wl.n_img, C, gloop.LoopConfig("F", 1, [t, t - dt], [1.0, 1.0], 0.05, binding.METRIC_L2, 0.1))
    gm.bind(lp)
    v_gpu, v_orc = gm.full(dev_bf16(x), t, True), om.full(x, t)
    binding.partition(dev_bf16(x), v_gpu, dev_bf16(ref), t, binding.METRIC_L2, 0.1, lp.mask, lp.edit_idx, lp.keep_idx, lp.slot,
                      lp.n_edit)
    p = orc.partition(x, synth.bf16_round(v_orc.astype(np.float32)), ref, np.float32(t), orc.L2, np.float32(0.1))
    assert np.array_equal(p["mask"].astype(bool), planted) and np.array_equal(lp.mask.cpu().numpy().astype(bool), planted)
    ne = int(p["n_edit"][0])
    x_e = np.zeros_like(x); x_e[0, :ne] = x[0, p["edit_idx"][0, :ne]] * 0.9
    x_e = synth.bf16_round(x_e.astype(np.float32))
    ve_gpu = gm.region(dev_bf16(x_e), t - dt, lp.edit_idx, lp.n_edit)
    ve_orc = om.region(x_e, t - dt, p["edit_idx"], p["n_edit"])
    assert int(gm.dev_status[0]) == 0
    inside = planted[0]
    return _rel(host_f64(v_gpu)[0, inside], v_orc[0, inside]), _rel(host_f64(ve_gpu)[0, :ne], ve_orc[0, :ne])


@pytest.mark.parametrize("membership", ["paper", "edited_queries"])
def test_bf16_products_of_both_streams_in_one_call(membership):
    full, region = _steps(membership, products="grouped")
    assert full < 3e-2 and region < 3e-2


def test_4_bit_products():
    full, region = _steps("paper", products="mxfp4")
    assert 0 < full < 0.5 and 0 < region < 0.5


def test_4_bit_cache():
    full, region = _steps("paper", products="grouped", cache="mxfp4")
    assert full < 3e-2 and region < 0.25


@pytest.mark.parametrize("how", [dict(products="grouped"), dict(products="mxfp4", cache="mxfp4")])
def test_the_sampler_loop_runs_around_it(how):
    import torch
    wl, om, gm, ref, planted, x = _setup(seed=5, **how)
    kinds, after = gloop.alternating_schedule()
    T = len(kinds)
    cfg = gloop.LoopConfig(kinds, after, [1.0 - k / T for k in range(T + 1)], [1.0] * (T + 1), 0.05, binding.METRIC_L2, 0.1)
    lp = gloop.RegionELoop(1, wl.n_img, C, cfg)
    gm.bind(lp)
    out, trace = lp.run(dev_bf16(x), dev_bf16(ref), gm)
    torch.cuda.synchronize()
    assert int(lp.dev_status[0]) == 0 and int(gm.dev_status[0]) == 0
    assert torch.isfinite(out.float()).all() and trace.model_region_calls > 0
    assert np.array_equal(lp.mask.cpu().numpy().astype(bool), planted)


def test_unknown_products_are_refused():
    with pytest.raises(binding.RegionEError):
        _setup(products="fp8")
