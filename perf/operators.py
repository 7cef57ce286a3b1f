"""Matrix products of ragged groups of rows, and the 4-bit microscaled format, as cases that can be timed and compared.

``kind`` names the operator:

  grouped    product of groups of bf16 rows with the weight set of their group, bias and activation fused
  linear4    the same layer in 4 bits: the rows are quantised, then multiplied with weights quantised beforehand
  quantize   rows to 4-bit codes with a scale per 32 elements, and back
  cache      the Region-Instruction KV cache in that format: stored at a full step, widened in front of a region step

``layout`` says where the groups of a product come from: ``streams`` are the text and the image rows of ``batch`` requests (two
weight sets; a request has room for ``image`` image rows, of which a seeded part is live), ``experts`` are the rows of
``tokens`` tokens sorted by expert, ``top`` experts each, unevenly and some experts empty.

Where ``own`` is false the operators run in plain torch operations, in 32 bits.
"""
import math

import numpy as np
import torch

own = False

BF, F32, F64, I32, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8
MOST_FLOPS = 1.03e12              # a drawn case costs no more than the largest listed ones
MOST_BYTES = 7.2e8


def listed():
    return [
        # modulation of one block: a single row per stream, the weights pass through once
        dict(name="grouped_one_row", kind="grouped", layout="streams", batch=1, text=1, image=1, K=1024, N=6144, gelu=False),
        # Q, K and V of a region step: text rows and a fifth of a 64 x 64 token image
        dict(name="grouped_region_qkv", kind="grouped", layout="streams", batch=1, text=256, image=1024, K=2048, N=6144,
             gelu=False),
        # first product of the feed-forward part in a full step of two images with their references
        dict(name="grouped_full_ffn", kind="grouped", layout="streams", batch=2, text=512, image=8192, K=2048, N=8192, gelu=True),
        # a mixture layer: 64 experts, 8 for each of 512 tokens
        dict(name="grouped_experts", kind="grouped", layout="experts", experts=64, tokens=512, top=8, K=2048, N=1408, gelu=True),
        # the same layers in 4 bits
        dict(name="linear4_one_row", kind="linear4", layout="streams", batch=1, text=1, image=1, K=1024, N=6144, gelu=False),
        dict(name="linear4_region_qkv", kind="linear4", layout="streams", batch=1, text=256, image=1024, K=2048, N=6144,
             gelu=False),
        dict(name="linear4_full_ffn", kind="linear4", layout="streams", batch=2, text=512, image=8192, K=4096, N=8192, gelu=True),
        # few tokens in a mixture layer: most of the time goes into weights that meet one or two rows
        dict(name="linear4_experts_few", kind="linear4", layout="experts", experts=48, tokens=17, top=4, K=4096, N=1536,
             gelu=False),
        # activations of a region step, gathered by the row list; the weights of a feed-forward layer when they are laid out
        dict(name="quantize_rows", kind="quantize", batch=1, src=8704, rows=1075, K=2048, gather=True),
        dict(name="quantize_weights", kind="quantize", batch=1, src=16384, rows=16384, K=8192, gather=False),
        # one layer's cache: 1024 x 1024 edit with its reference; four larger edits with heads of 64
        dict(name="cache_one", kind="cache", batch=1, full=8704, rows=7885, H=24, D=128),
        dict(name="cache_batch", kind="cache", batch=4, full=18944, rows=17562, H=16, D=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["grouped", "grouped", "linear4", "linear4", "quantize", "cache"])
        if kind in ("grouped", "linear4"):
            step = 8 if kind == "grouped" else 128
            case = dict(kind=kind, K=step * max(1, _log_int(rng, 256, 8192) // step), N=8 * _log_int(rng, 8, 2048),
                        gelu=rng.random() < 0.5)
            if rng.random() < 0.5:
                case.update(layout="streams", batch=rng.choice([1, 1, 2, 4]), text=_log_int(rng, 1, 1024),
                            image=_log_int(rng, 1, 9216))
            else:
                experts = rng.randint(3, 130)
                case.update(layout="experts", experts=experts, tokens=_log_int(rng, 1, 4096), top=rng.randint(1, min(8, experts)))
        elif kind == "quantize":
            gather = rng.random() < 0.5
            rows = _log_int(rng, 1, 16384)
            case = dict(kind=kind, batch=rng.choice([1, 1, 3]), src=rows + (_log_int(rng, 1, 4096) if gather else 0), rows=rows,
                        K=32 * _log_int(rng, 1, 256), gather=gather)
        else:
            full = _log_int(rng, 16, 18944)
            case = dict(kind=kind, batch=rng.choice([1, 1, 2, 4]), full=full, rows=rng.randint(1, full),
                        H=rng.choice([3, 4, 16, 24]), D=rng.choice([64, 128]))
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


def _groups(case, seed):
    """[(first row, row behind the last, weight set)] and the rows of the buffers."""
    if case["layout"] == "streams":
        rng = np.random.default_rng([seed, 1])
        room, out = case["text"] + case["image"], []
        for b in range(case["batch"]):
            live = case["image"] if case["batch"] == 1 else int(rng.integers(max(1, case["image"] * 3 // 4), case["image"] + 1))
            mid = b * room + case["text"]
            out += [(b * room, mid, 0), (mid, mid + live, 1)]
        return out, case["batch"] * room, 2
    rng = np.random.default_rng([seed, 2])
    E = case["experts"]
    liking = rng.dirichlet(np.full(E, 1.5))                       # some experts are asked for far more than others
    count = np.zeros(E, int)
    for _ in range(case["tokens"]):
        count[np.argsort(np.log(liking) + rng.gumbel(size=E))[-case["top"]:]] += 1
    end = np.cumsum(count)
    return [(int(e - c), int(e), i) for i, (e, c) in enumerate(zip(end, count))], int(end[-1]), E


def work(case):
    if case["kind"] in ("grouped", "linear4"):
        groups = [g for g in _groups(case, 0)[0] if g[1] > g[0]]      # (other seeds: nearly as many rows and experts)
        rows, sets = sum(e - b for b, e, _ in groups), len({i for _, _, i in groups})
        K, N = case["K"], case["N"]
        weight = 2.0 if case["kind"] == "grouped" else 17.0 / 32
        return {"bytes": rows * K * 2 + sets * N * K * weight + sets * N * 2 + rows * N * 2, "flops": 2.0 * rows * N * K}
    if case["kind"] == "quantize":
        n = case["batch"] * case["rows"] * case["K"]
    else:
        n = 2 * case["batch"] * case["rows"] * case["H"] * case["D"]
    return {"bytes": n * (2 + 17.0 / 32) + n * (2 + 17.0 / 32), "flops": 4.0 * n}


def _normal(gen, shape, std=1.0):
    return (torch.randn(shape, device="cuda", dtype=F32, generator=gen) * std).to(BF)


def _pow2(k):
    """2^k as fp32, from its bits; -127 < k < 128."""
    return ((k.int() + 127) << 23).view(F32)


def _codes(x):
    """Plain quantisation of bf16 x [..., K]: element values over their scale [..., K/32, 32] and k of the scale 2^k."""
    blocks = x.float().unflatten(-1, (-1, 32))
    m, e = torch.frexp(blocks.abs().amax(-1))
    k = torch.where(m == 0, 0, (e - 3 + (m > 0.75)).clamp(min=-127))
    y = blocks * _pow2(-k).unsqueeze(-1)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.round(a / step) * step * torch.sign(y), k


def _widen(q, k):
    return (q * _pow2(k).unsqueeze(-1)).flatten(-2)


def _pack(q, k):
    """The plain codes as bytes: two E2M1 codes to a byte, the earlier element in the low half; E8M0 scales."""
    a = q.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(U8) | (torch.signbit(q).to(U8) << 3)
    code = code.flatten(-2)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous(), (k + 127).to(U8)


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    s = dict(case)
    if case["kind"] in ("grouped", "linear4"):
        groups, rows, sets = _groups(case, seed)
        K, N = case["K"], case["N"]
        s["groups"] = groups
        s["begin"] = torch.tensor([g[0] for g in groups], dtype=I32, device="cuda")
        s["end"] = torch.tensor([g[1] for g in groups], dtype=I32, device="cuda")
        s["x"] = _normal(gen, (rows, K))                              # rows behind a normalisation
        w = _normal(gen, (sets, N, K), K ** -0.5)
        s["bias"] = _normal(gen, (sets, N), 0.1)
        s["out"] = torch.zeros((rows, N), dtype=BF, device="cuda")
        if case["kind"] == "grouped":
            s["w"] = w
        else:
            # the weights are quantised once, when a model is loaded
            s["w_q"] = torch.empty((sets, N, K // 2), dtype=U8, device="cuda")
            s["w_scale"] = torch.empty((sets, N, K // 32), dtype=U8, device="cuda")
            for i in range(sets):
                s["w_q"][i], s["w_scale"][i] = _pack(*_codes(w[i]))
            s["x_q"] = torch.empty((1, rows, K // 2), dtype=U8, device="cuda")
            s["x_scale"] = torch.empty((1, rows, K // 32), dtype=U8, device="cuda")
    elif case["kind"] == "quantize":
        B, rows, K = case["batch"], case["rows"], case["K"]
        s["x"] = _normal(gen, (B, case["src"], K)) * torch.exp2(torch.randint(-6, 5, (B, case["src"], 1), device="cuda",
                                                                             generator=gen).float()).to(BF)
        s["idx"] = None
        if case["gather"]:
            s["idx"] = torch.stack([torch.randperm(case["src"], device="cuda", generator=gen)[:rows].sort().values
                                    for _ in range(B)]).to(I32)
        s["codes"] = torch.empty((B, rows, K // 2), dtype=U8, device="cuda")
        s["scales"] = torch.empty((B, rows, K // 32), dtype=U8, device="cuda")
        s["out"] = torch.empty((B, rows, K), dtype=BF, device="cuda")
    else:
        B, rows, H, D = (case[k] for k in ("batch", "rows", "H", "D"))
        s["k"] = _normal(gen, (B, case["full"], H, D), D ** -0.5)     # normalised keys
        s["v"] = _normal(gen, (B, case["full"], H, D))
        s["keep"] = torch.stack([torch.randperm(case["full"], device="cuda", generator=gen)[:rows].sort().values
                                 for _ in range(B)]).to(I32)
        s["n"] = torch.full((B,), rows, dtype=I32, device="cuda")
        for name in ("k", "v"):
            s[name + "_q"] = torch.empty((B, rows, H, D // 2), dtype=U8, device="cuda")
            s[name + "_scale"] = torch.empty((B, rows, H, D // 32), dtype=U8, device="cuda")
            s[name + "_cache"] = torch.empty((B, rows, H, D), dtype=BF, device="cuda")
    return s


def _gelu(x):
    return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))


def _weights(s, i):
    """Weight set i of a 4-bit layer, widened."""
    b = s["w_q"][i].int()
    code = torch.stack([b & 15, b >> 4], -1).flatten(-2)
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=b.device)
    return _widen(table[code].unflatten(-1, (-1, 32)), s["w_scale"][i].int() - 127)


def _run_plain(s):
    if s["kind"] in ("grouped", "linear4"):
        for b, e, i in s["groups"]:
            if e > b:
                if s["kind"] == "grouped":
                    y = s["x"][b:e].float() @ s["w"][i].float().T
                else:
                    y = _widen(*_codes(s["x"][b:e])) @ _weights(s, i).T
                y += s["bias"][i].float()
                s["out"][b:e] = (_gelu(y) if s["gelu"] else y).to(BF)
        return s["out"]
    if s["kind"] == "quantize":
        for b in range(s["batch"]):
            x = s["x"][b] if s["idx"] is None else s["x"][b][s["idx"][b].long()]
            s["out"][b] = _widen(*_codes(x)).to(BF)
        return s["out"]
    for b in range(s["batch"]):
        keep = s["keep"][b].long()
        s["k_cache"][b] = _widen(*_codes(s["k"][b][keep])).to(BF)
        s["v_cache"][b] = _widen(*_codes(s["v"][b][keep])).to(BF)
    return s["k_cache"], s["v_cache"]


def _run_own(s):
    from paper_2510_25590_b200 import binding
    if s["kind"] in ("grouped", "linear4"):
        act = binding.ACT_GELU_TANH if s["gelu"] else binding.ACT_NONE
        if s["kind"] == "grouped":
            binding.grouped_matmul(s["x"], s["w"], s["begin"], s["end"], s["out"], bias=s["bias"], activation=act)
        else:
            binding.mxfp4_quantize(s["x"][None], s["x_q"], s["x_scale"])
            binding.mxfp4_grouped_matmul(s["x_q"][0], s["x_scale"][0], s["w_q"], s["w_scale"], s["begin"], s["end"], s["out"],
                                         bias=s["bias"], activation=act)
        return s["out"]
    if s["kind"] == "quantize":
        binding.mxfp4_quantize(s["x"], s["codes"], s["scales"], idx=s["idx"])
        binding.mxfp4_dequantize(s["codes"], s["scales"], s["out"])
        return s["out"]
    binding.rikv_store_mxfp4(s["k"], s["v"], s["keep"], s["n"], s["k_q"], s["v_q"], s["k_scale"], s["v_scale"])
    binding.rikv_load_mxfp4(s["k_q"], s["v_q"], s["k_scale"], s["v_scale"], s["n"], s["k_cache"], s["v_cache"])
    return s["k_cache"], s["v_cache"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _nearest(x):
    """The format from its definition, in 64 bits: the scale by search, the element by its distance to every value."""
    v = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=F64, device=x.device)
    mid, even = (v[1:] + v[:-1]) / 2, torch.arange(7, device=x.device) % 2 == 0
    out = torch.empty(x.shape, dtype=F64, device=x.device)
    for i in range(0, x.shape[0], 1024):
        t = x[i:i + 1024].double().unflatten(-1, (-1, 32))
        top = t.abs().amax(-1, keepdim=True)
        k = torch.ceil(torch.log2(torch.where(top == 0, 6.0, top) / 6))
        k = torch.where(top <= 6 * torch.exp2(k - 1), k - 1, k)
        k = torch.where(top > 6 * torch.exp2(k), k + 1, k)
        k = torch.where(top == 0, 0.0, k.clamp(min=-127))
        a = t.abs() * torch.exp2(-k)
        code = torch.zeros_like(a, dtype=torch.long)
        for j in range(7):                                          # between two values: up behind the middle, on it to the even code
            code += (a > mid[j]) | ((a == mid[j]) & ~even[j])
        out[i:i + 1024] = (v[code] * torch.sign(t) * torch.exp2(k)).flatten(-2)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("grouped", "linear4"):
        out = torch.zeros(s["out"].shape, dtype=F64, device="cuda")
        for b, e, i in s["groups"]:
            if e == b:
                continue
            if case["kind"] == "grouped":
                x, w = s["x"][b:e].double(), s["w"][i].double()
            else:
                x, c = _nearest(s["x"][b:e]), s["w_q"][i].long()
                c = torch.stack([c % 16, c // 16], -1).flatten(-2)
                mag, ex = (c % 8).double(), torch.clamp(c % 8 // 2, min=1).double()
                frac = torch.where(c % 8 < 2, mag / 2, 1 + (c % 2) / 2)          # subnormal below 1, else 1.0 or 1.5
                w = torch.where(c >= 8, -1.0, 1.0) * frac * torch.exp2(ex - 1)
                w = w * torch.exp2(s["w_scale"][i].double() - 127).repeat_interleave(32, -1)
            for j in range(0, e - b, 4096):
                y = torch.matmul(x[j:j + 4096], w.T) + s["bias"][i].double()
                if case["gelu"]:
                    z = math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)
                    y = y / (1 + torch.exp(-2 * z))
                out[b + j:b + j + y.shape[0]] = y
        return out
    if case["kind"] == "quantize":
        pick = lambda b: s["x"][b] if s["idx"] is None else s["x"][b].index_select(0, s["idx"][b].long())
        return torch.stack([_nearest(pick(b)) for b in range(case["batch"])])
    side = lambda x: torch.stack([_nearest(x[b].index_select(0, s["keep"][b].long()).flatten(1)).view(-1, case["H"], case["D"])
                                  for b in range(case["batch"])])
    return side(s["k"]), side(s["v"])
