"""What the bounds of the 4-bit stack's GPU tests tell apart: the oracle's stack in 4 bits against the same stack with a mistake planted in
it (CPU only).  The bounds themselves are derived beside ``BOUND`` and ``CACHE_BOUND``."""
import numpy as np
import pytest

from oracle import mmdit_oracle, regione_oracle as orc
from paper_2510_25590_b200 import synth

H, D, C, L, N_TEXT = 2, 128, 16, 2, 40

# Relative error of a velocity with 4-bit products, both sides quantised.  Rows in front of a quantisation differ by their bf16 roundings:
# h, the modulation, the normalised rows, each off by 2^-9 of itself at most and 2^-9 / sqrt(3) on the average, about 2^-8 / sqrt(3)
# together.  Where that moves an element over the middle between two codes, its value moves by a whole step, 0.25 to 0.5 of
# itself, 0.35 on the average: sqrt(0.35 * 2^-8 / sqrt(3)) = 0.028 of a row.  Eight products (four in each of two blocks) with independent
# errors: sqrt(8) * 0.028 = 0.08.
BOUND = 0.08
# With bf16 products and a 4-bit cache: a stored element moves by a step as above, 0.028 of a row, and reaches the output through an
# average over keys and one of four products a block: 0.01, beside the bf16 roundings of the stack itself, which its own test bounds by this.
CACHE_BOUND = 3e-2


def model(cls=mmdit_oracle.MMDiTOracle, membership="paper", seed=3, **how):
    wl = synth.scaled_workload(synth.WORKLOADS[4], grid=(16, 16), n_text=N_TEXT, heads=H)
    lat = synth.make_latents(wl, 0.20, stream=seed)
    ref, planted = lat["ref"], lat["mask"].astype(bool)
    w = synth.make_mmdit_weights(H * D, D, C, N_TEXT, L, seed=seed)
    cos, sin = synth.rope_tables(N_TEXT + 2 * wl.n_img, D)
    m = cls(w, N_TEXT, wl.n_img, wl.n_img, H, D, L, cos, sin, ref, planted, membership, **how)
    x = synth.bf16_round(np.random.default_rng(seed).standard_normal(ref.shape).astype(np.float32))
    return m, ref, planted, x


def steps(m, ref, planted, x, t=0.75, dt=1.0 / 28.0):
    """Velocities of a full step and of the region step behind it, inside the planted region."""
    v = m.full(x, t)
    e = np.flatnonzero(planted[0])
    x_e = np.zeros_like(x); x_e[0, :len(e)] = x[0, e] * 0.9
    idx = np.zeros((1, planted.shape[1]), np.int64); idx[0, :len(e)] = e
    ve = m.region(synth.bf16_round(x_e.astype(np.float32)), t - dt, idx, [len(e)])
    return v[0, planted[0]], ve[0, :len(e)]


def rel(got, want):
    return float(np.sqrt(np.mean((got - want) ** 2)) / np.sqrt(np.mean(want ** 2)))


def planted_mistake(kind, product):
    """The stack with one of its products zeroed or taken with the other stream's weights."""
    class Mistaken(mmdit_oracle.MMDiTOracle):
        def _per_stream(self, x, streams, name):
            hit = name.startswith(product)
            y = super()._per_stream(x, 1 - streams if hit and kind == "other stream" else streams, name)
            return 0.0 * y if hit and kind == "zero" else y
    return Mistaken


@pytest.fixture(scope="module")
def right():
    return steps(*model(products="mxfp4"))


@pytest.mark.parametrize("kind", ["zero", "other stream"])
@pytest.mark.parametrize("product", ["qkv", "o", "fc1", "fc2"])
def test_a_wrong_product_is_outside_the_bound(right, kind, product):
    full, region = steps(*model(planted_mistake(kind, product), products="mxfp4"))
    assert rel(full, right[0]) > 2 * BOUND and rel(region, right[1]) > 2 * BOUND


@pytest.mark.parametrize("lost", ["k", "v", "kv"])
def test_a_lost_cache_is_outside_the_bound(lost, monkeypatch):
    want = steps(*model(cache="mxfp4"))[1]
    store = orc.rikv_store

    def losing(*a):
        k, v = store(*a)
        return 0.0 * k if "k" in lost else k, 0.0 * v if "v" in lost else v
    monkeypatch.setattr(orc, "rikv_store", losing)
    assert rel(steps(*model(cache="mxfp4"))[1], want) > 2 * CACHE_BOUND


def test_what_the_format_takes():
    """4-bit products are another function than exact ones, a 4-bit cache nearly the same."""
    exact, four = steps(*model()), steps(*model(products="mxfp4"))
    assert all(0.05 < rel(a, b) < 0.5 for a, b in zip(four, exact))
    assert rel(steps(*model(cache="mxfp4"))[1], exact[1]) < CACHE_BOUND


def test_bf16_rounding():
    x = np.concatenate([np.random.default_rng(0).standard_normal(1000).astype(np.float32) * np.float32(2.0) ** np.arange(-50, 50).repeat(10),
                        np.float32([0.0, -0.0, 1.00390625, 1.01171875, 1.9999, -1.00390625])])
    assert np.array_equal(mmdit_oracle._bf16(x), synth.bf16_round(x).astype(np.float64))
