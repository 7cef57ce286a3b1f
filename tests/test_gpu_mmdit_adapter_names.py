"""The stand-in stack with adapters beside the products that the test of its blocks leaves without: K's projection and the modulation's rows."""
import numpy as np
import pytest

from gpu_util import dev_bf16
from paper_2510_25590_b200 import binding, synth
from test_gpu_mmdit_block import L, MATCH, RANK, _setup, _steps

pytestmark = pytest.mark.gpu


def _with_adapters(lost=False):
    import torch
    wl, om, gm, ref, planted, x = setup = _setup(adapters=False)
    rng, hd, of = np.random.default_rng(8), gm.hidden, (1, 0)
    om.w, factors = dict(om.w), {}
    for l in range(L):
        for name, N, key, cols in ((f"k{l}", hd, f"qkv{l}", slice(hd, 2 * hd)), (f"mod{l}", 6 * hd, f"mod{l}", slice(None))):
            a = synth.bf16_round((rng.standard_normal((2, RANK, hd)) * hd ** -0.5).astype(np.float32))
            b = synth.bf16_round((rng.standard_normal((2, N, RANK)) * RANK ** -0.5).astype(np.float32))
            factors[name] = dev_bf16(a), dev_bf16(b)
            for s in (0, 1):
                w = np.array(om.w[f"{key}_{s}"], np.float64)
                w[:, cols] += 0.0 if lost else (b[of[s]].astype(np.float64) @ a[of[s]].astype(np.float64)).T
                om.w[f"{key}_{s}"] = w
    gm.adapters = factors, torch.tensor(of, dtype=torch.int32, device="cuda"), None
    need = max(binding.adapter_matmul_workspace(gm.n_full, 2, hd, b.shape[1], RANK) for _, b in factors.values())
    gm.adapter_workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
    return setup


def test_adapters_of_k_and_of_the_modulation():
    full, region = _steps(_with_adapters())
    assert full < MATCH and region < MATCH


def test_lost_ones_show():
    full, _ = _steps(_with_adapters(lost=True))
    assert full > MATCH
