"""The stand-in stack with its norms, its positions and its adapters through the library: layer norm, rotary positions and products with
adapters as a transformer block uses them one after the other, in full and region steps, against the oracle's stack with the same
angles and with the adapters folded into its weights.

Bounds: those of the stack's test with library products, its arithmetic is bf16 either way; a lost adapter, the other stream's adapter and
coordinates in another order are outside them."""
import numpy as np
import pytest

from gpu_util import dev_bf16, host_f64
from oracle import mmdit_oracle, regione_oracle as orc
from paper_2510_25590_b200 import binding, loop as gloop, synth
from paper_2510_25590_b200.mmdit_scaffold import MMDiTScaffold

pytestmark = pytest.mark.gpu

H, D, C, L, N_TEXT, RANK = 2, 128, 16, 2, 40, 16
WIDTHS = (16, 56, 56)
MATCH = 3e-2


def _places(side):
    """(image or text, row, column) of text, image and reference tokens."""
    grid = np.stack(np.meshgrid(np.arange(side), np.arange(side), indexing="ij"), -1).reshape(-1, 2)
    image = np.concatenate([np.zeros((len(grid), 1)), grid], 1)
    ref = np.concatenate([np.ones((len(grid), 1)), grid], 1)
    return np.concatenate([np.zeros((N_TEXT, 3)), image, ref]).astype(np.float32)


def _setup(membership="paper", seed=3, norms="fused", axes=True, adapters=True, products="grouped"):
    import torch
    wl = synth.scaled_workload(synth.WORKLOADS[4], grid=(16, 16), n_text=N_TEXT, heads=H)
    lat = synth.make_latents(wl, 0.20, stream=seed)
    ref, planted = lat["ref"], lat["mask"].astype(bool)
    w = synth.make_mmdit_weights(H * D, D, C, N_TEXT, L, seed=seed)
    freq, axis = binding.rotary_frequencies(WIDTHS)
    places = _places(16)
    if axes:
        angle = places.astype(np.float64)[:, axis] * np.asarray(freq)
        cos, sin = np.cos(angle), np.sin(angle)
    else:
        cos, sin = synth.rope_tables(N_TEXT + 2 * wl.n_img, D)
    folded, factors, of, scale = dict(w), {}, (1, 0), (1.5, 0.75, 1.0)
    if adapters:
        rng = np.random.default_rng(seed + 100)
        hd = H * D
        for l in range(L):
            for name, K, N in [(f"q{l}", hd, hd), (f"v{l}", hd, hd), (f"o{l}", hd, hd), (f"fc1_{l}", hd, w[f"fc1_{l}_0"].shape[1]),
                               (f"fc2_{l}", w[f"fc1_{l}_0"].shape[1], hd)]:
                a = synth.bf16_round((rng.standard_normal((3, RANK, K)) * K ** -0.5).astype(np.float32))
                b = synth.bf16_round((rng.standard_normal((3, N, RANK)) * 0.5 * RANK ** -0.5).astype(np.float32))
                factors[name] = a, b
                for s in (0, 1):
                    more = (scale[of[s]] * (b[of[s]].astype(np.float64) @ a[of[s]].astype(np.float64))).T
                    if name[0] in "qv":
                        j, key = "qkv".index(name[0]), f"qkv{l}_{s}"
                        folded[key] = np.array(folded[key], np.float64)
                        folded[key][:, j * hd:(j + 1) * hd] += more
                    else:
                        folded[f"{name}_{s}"] = np.asarray(folded[f"{name}_{s}"], np.float64) + more
    om = mmdit_oracle.MMDiTOracle(folded, N_TEXT, wl.n_img, wl.n_img, H, D, L, cos, sin, ref, planted, membership)
    how = dict(products=products, norms=norms)
    tables = (None, None) if axes else tuple(torch.from_numpy(t).cuda() for t in (cos, sin))
    if axes:
        how.update(positions=torch.from_numpy(places).cuda(), rotary=(freq, axis))
    if adapters:
        how["adapters"] = ({k: (dev_bf16(a), dev_bf16(b)) for k, (a, b) in factors.items()},
                           torch.tensor(of, dtype=torch.int32, device="cuda"), torch.tensor(scale, dtype=torch.float32, device="cuda"))
    gm = MMDiTScaffold({k: dev_bf16(v) for k, v in w.items()}, N_TEXT, wl.n_img, wl.n_img, H, D, L, *tables, dev_bf16(ref),
                       torch.from_numpy(planted).cuda(), binding.ROWS_PAPER if membership == "paper" else binding.ROWS_EDITED_QUERIES, **how)
    x = synth.bf16_round(np.random.default_rng(seed).standard_normal(ref.shape).astype(np.float32))
    return wl, om, gm, ref, planted, x


def _rel(got, want):
    return float(np.sqrt(np.mean((got - want) ** 2)) / np.sqrt(np.mean(want ** 2)))


def _steps(setup):
    """Errors of a full step and of the region step behind it against the oracle's stack, inside the planted region."""
    wl, om, gm, ref, planted, x = setup
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
@pytest.mark.parametrize("how", [dict(), dict(adapters=False, products="torch"), dict(axes=False, adapters=False), dict(norms="torch"),
                                 dict(norms="torch", adapters=False, products="torch")],
                         ids=["all", "norms_and_positions", "norms", "positions_and_adapters", "positions"])
def test_steps_match_the_oracles_stack(how, membership):
    full, region = _steps(_setup(membership, **how))
    assert full < MATCH and region < MATCH


@pytest.mark.parametrize("lost", ["adapter", "stream", "axes"])
def test_what_is_lost_shows(lost):
    """A mistake planted in the oracle: no adapters, those of the other stream, or rows and columns exchanged."""
    wl, om, gm, ref, planted, x = setup = _setup()
    if lost == "adapter":
        om.w.update({k: np.asarray(v, np.float64) for k, v in synth.make_mmdit_weights(H * D, D, C, N_TEXT, L, seed=3).items()})
    elif lost == "stream":
        plain = synth.make_mmdit_weights(H * D, D, C, N_TEXT, L, seed=3)
        for l in range(L):
            for name in (f"qkv{l}", f"o{l}", f"fc1_{l}", f"fc2_{l}"):
                more = [om.w[f"{name}_{s}"] - plain[f"{name}_{s}"] for s in (0, 1)]
                for s in (0, 1):
                    om.w[f"{name}_{s}"] = plain[f"{name}_{s}"] + more[1 - s]
    else:
        places = _places(16)[:, [0, 2, 1]].astype(np.float64)
        freq, axis = binding.rotary_frequencies(WIDTHS)
        angle = places[:, axis] * np.asarray(freq)
        om.cos, om.sin = np.cos(angle), np.sin(angle)
    t = 0.75
    full = _rel(host_f64(gm.full(dev_bf16(x), t, False))[0, planted[0]], om.full(x, t)[0, planted[0]])
    assert full > MATCH                                                # what shows is what the match's own bound refuses, no more and no less


def test_the_sampler_loop_runs_around_it():
    import torch
    wl, om, gm, ref, planted, x = _setup(seed=5)
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


def test_what_does_not_go_together_is_refused():
    for how in (dict(norms="rms"), dict(products="torch"), dict(products="mxfp4")):
        with pytest.raises(binding.RegionEError):
            _setup(**how)
