"""The stand-in stack with 4-bit products and a 4-bit cache against the oracle's stack with the same operands quantised, and what it
multiplies and attends over, step by step.  The bounds of the whole stack are derived, and shown to leave planted mistakes outside, in
the oracle's own test."""
import numpy as np
import pytest

from gpu_util import dev_bf16, host_f64
from oracle import regione_oracle as orc
from paper_2510_25590_b200 import binding, loop as gloop, synth
from paper_2510_25590_b200.mmdit_scaffold import MMDiTScaffold
from test_oracle_mmdit_4bit import BOUND, C, CACHE_BOUND, D, H, L, N_TEXT, model, rel, steps

pytestmark = pytest.mark.gpu


def _scaffold(membership, **how):
    import torch
    om, ref, planted, x = model(membership=membership)
    w = synth.make_mmdit_weights(H * D, D, C, N_TEXT, L, seed=3)
    gm = MMDiTScaffold({k: dev_bf16(v) for k, v in w.items()}, N_TEXT, om.n_img, om.n_img, H, D, L,
                       torch.from_numpy(om.cos.astype(np.float32)).cuda(), torch.from_numpy(om.sin.astype(np.float32)).cuda(),
                       dev_bf16(ref), torch.from_numpy(planted).cuda(),
                       binding.ROWS_PAPER if membership == "paper" else binding.ROWS_EDITED_QUERIES, **how)
    return gm, w, ref, planted, x


def _run(gm, ref, planted, x, t=0.75, dt=1.0 / 28.0):
    """As ``steps`` of the oracle's test: the same latents, the planted tokens edited."""
    lp = gloop.RegionELoop(1, gm.n_img, C, gloop.LoopConfig("F", 1, [t, t - dt], [1.0, 1.0], 0.05, binding.METRIC_L2, 0.1))
    gm.bind(lp)
    v = gm.full(dev_bf16(x), t, True)
    binding.partition(dev_bf16(x), v, dev_bf16(ref), t, binding.METRIC_L2, 0.1, lp.mask, lp.edit_idx, lp.keep_idx, lp.slot, lp.n_edit)
    assert np.array_equal(lp.mask.cpu().numpy().astype(bool), planted)
    e = np.flatnonzero(planted[0])
    x_e = np.zeros_like(x); x_e[0, :len(e)] = x[0, e] * 0.9
    ve = gm.region(dev_bf16(synth.bf16_round(x_e.astype(np.float32))), t - dt, lp.edit_idx, lp.n_edit)
    assert int(gm.dev_status[0]) == 0
    return host_f64(v)[0, planted[0]], host_f64(ve)[0, :len(e)]


@pytest.mark.parametrize("membership", ["paper", "edited_queries"])
@pytest.mark.parametrize("how,oracle,bound", [(dict(products="mxfp4"), dict(products="mxfp4"), BOUND),
                                              (dict(products="grouped", cache="mxfp4"), dict(cache="mxfp4"), CACHE_BOUND),
                                              (dict(products="torch", cache="mxfp4"), dict(cache="mxfp4"), CACHE_BOUND),
                                              (dict(products="mxfp4", cache="mxfp4"), dict(products="mxfp4", cache="mxfp4"), BOUND)],
                         ids=["products", "cache", "cache-torch", "both"])
def test_against_the_oracles_stack_in_4_bits(how, oracle, bound, membership):
    gm, w, ref, planted, x = _scaffold(membership, **how)
    got, want = _run(gm, ref, planted, x), steps(*model(membership=membership, **oracle))
    assert rel(got[0], want[0]) < bound and rel(got[1], want[1]) < bound


def _gelu(y):
    return 0.5 * y * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (y + 0.044715 * y ** 3)))


def test_every_product_of_the_steps(monkeypatch):
    """Operands are what the oracle quantises of the rows and of the weights of the rows' stream, the sums what they give: half a bf16
    step, and K additions of at most 2^-23 of the sum of magnitudes (times gelu's slope, at most 1.13, and 2^-14 for its own steps)."""
    gm, w, ref, planted, x = _scaffold("paper", products="mxfp4")
    operands, products = [], []
    operand, product = gm._operand, gm._product

    def spy_operand(a):
        out = operand(a)
        operands.append((host_f64(a), *(o.cpu().numpy() for o in out)))
        return out

    def spy_product(op, name, ranges, out, activation=binding.ACT_NONE):
        r = product(op, name, ranges, out, activation)
        if isinstance(op, tuple):
            products.append((*(o.cpu().numpy() for o in op), name, [v.cpu().numpy() for v in ranges], host_f64(out), activation))
        return r
    monkeypatch.setattr(gm, "_operand", spy_operand)
    monkeypatch.setattr(gm, "_product", spy_product)
    _run(gm, ref, planted, x)
    assert len(operands) == 2 * L * 4 and len(products) == 2 * L * 6          # two steps; Q, K and V share their rows
    for a, codes, scales in operands:
        c, s = orc.mxfp4_quantize(a)
        assert np.array_equal(scales, s) and np.array_equal(orc.mxfp4_dequantize(codes, scales), orc.mxfp4_dequantize(c, s))
    for codes, scales, name, (begin, end), out, activation in products:
        assert begin.tolist() == [0, N_TEXT] and end.tolist() == [N_TEXT, len(out)]
        rows = orc.mxfp4_dequantize(codes, scales)
        for s, (b, e) in enumerate(zip(begin, end)):
            if name[0] in "qkv":
                j = "qkv".index(name[0])
                weight = w[f"qkv{name[1:]}_{s}"][:, j * H * D:(j + 1) * H * D]
            else:
                weight = w[f"{name}_{s}"]
            weight = orc.mxfp4_dequantize(*orc.mxfp4_quantize(weight.T))
            y, sums = rows[b:e] @ weight.T, np.abs(rows[b:e]) @ np.abs(weight.T)
            act = activation == binding.ACT_GELU_TANH
            assert act == name.startswith("fc1")
            want = _gelu(y) if act else y
            bound = (2.0 ** -8 + (2.0 ** -14 if act else 0.0)) * np.abs(want) + 1.13 * weight.shape[1] * 2.0 ** -23 * sums + 1e-30
            assert np.all(np.abs(out[b:e] - want) <= bound), (name, s)


@pytest.mark.parametrize("membership", ["paper", "edited_queries"])
def test_what_the_region_step_attends_over(monkeypatch, membership):
    """The kept rows of every block, quantised as the oracle quantises them: bit-exact."""
    gm, w, ref, planted, x = _scaffold(membership, products="grouped", cache="mxfp4")
    seen = []
    attention = binding.region_attention

    def spy(q, k, v, k_cache, v_cache, *rest, **kw):
        if k_cache is not None:
            seen.append((host_f64(k_cache), host_f64(v_cache)))
        return attention(q, k, v, k_cache, v_cache, *rest, **kw)
    monkeypatch.setattr(binding, "region_attention", spy)
    _run(gm, ref, planted, x)
    n = int(gm.n_cache[0])
    rows = gm.cache_rows[0, :n].cpu().numpy()
    kept = np.setdiff1d(np.arange(gm.n_full), gm.query_rows[0, :int(gm.n_query[0])].cpu().numpy())
    assert np.array_equal(rows, kept) and len(seen) == L
    for l, caches in enumerate(seen):
        for cache, full in zip(caches, (gm.k_full[l], gm.v_full[l])):
            c, s = orc.mxfp4_quantize(host_f64(full)[0, rows])
            assert np.array_equal(cache[0, :n], orc.mxfp4_dequantize(c, s))
