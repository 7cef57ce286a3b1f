"""What a transformer block does between its attention and its plain products, as cases that can be timed and compared.

``kind`` names the operator:

  norm       layer normalisation with the scale and shift of the row's group (``affine``: one weight and bias for all rows), behind
             the gated residual update of the rows where ``residual`` is true
  norm_grad  its backward pass, with the sums over the rows that are the gradients of scale, shift and gate
  rotary     rotary positions with several axes for Q and K, behind their per-head normalisation (``inverse``: the gradient of
             the rotation alone)
  adapters   product of groups of rows with the weight set of their group, and beside it the low-rank adapter of their group

``layout`` says where the groups come from: ``streams`` are the text and the image rows of ``batch`` requests (a request has room for
``image`` image rows, of which a seeded part is live), ``tokens`` are requests of one row each.

Where ``own`` is false the operators run in plain torch operations, in 32 bits (angles in 64).
"""
import math

import numpy as np
import torch

own = False

BF, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
MOST_FLOPS = 6.2e11               # a drawn case costs no more than the largest listed ones
MOST_BYTES = 1.2e9
EPS = 1e-6


def listed():
    return [
        # one row per stream: the latency of a call
        dict(name="norm_one_row", kind="norm", layout="streams", batch=1, text=1, image=1, C=1024, residual=False, affine=False),
        # between attention and feed-forward of a region step: text rows and a fifth of a 64 x 64 token image
        dict(name="norm_region", kind="norm", layout="streams", batch=1, text=256, image=819, C=2048, residual=True, affine=False),
        # the same in a full step of four images with their references
        dict(name="norm_full", kind="norm", layout="streams", batch=4, text=512, image=8192, C=4096, residual=True, affine=False),
        # gradients of a small layer with a weight and bias of its own, one image with its text
        dict(name="norm_grad_affine", kind="norm_grad", layout="streams", batch=1, text=77, image=1024, C=1536, residual=False, affine=True),
        # gradients of a modulated norm behind a gated residual, two images with their references
        dict(name="norm_grad_full", kind="norm_grad", layout="streams", batch=2, text=512, image=8192, C=2048, residual=True, affine=False),
        # a single new row for each of a few requests
        dict(name="rotary_one_row", kind="rotary", batch=17, src=1, rows=1, gather=False, Hq=8, Hk=8, widths="16 56 56",
             halves=False, normalise=True, inverse=False),
        # region step: the recomputed rows of an image and its text, gathered by the row list
        dict(name="rotary_region", kind="rotary", batch=1, src=8704, rows=1075, gather=True, Hq=16, Hk=16, widths="16 56 56",
             halves=False, normalise=True, inverse=False),
        # two clips of 17 frames of 30 x 45 tokens with their text, four heads of queries to one of keys
        dict(name="rotary_video", kind="rotary", batch=2, src=23176, rows=23176, gather=False, Hq=16, Hk=4, widths="16 24 24",
             halves=True, normalise=True, inverse=False),
        # the rotation's gradient, at an odd head dimension and odd lengths
        dict(name="rotary_grad", kind="rotary", batch=3, src=4099, rows=4099, gather=False, Hq=13, Hk=13, widths="32 32 32",
             halves=False, normalise=False, inverse=True),
        # 64 requests with one row each, most with an adapter
        dict(name="adapters_tokens", kind="adapters", layout="tokens", batch=64, K=2048, N=6144, rank=16, adapters=24, gelu=False),
        # Q, K and V of a region step of four requests, each with adapters of its own for text and image
        dict(name="adapters_region", kind="adapters", layout="streams", batch=4, text=77, image=1024, K=2048, N=6144, rank=32, adapters=8,
             gelu=False),
        # first product of the feed-forward part in a full step of two images with their references
        dict(name="adapters_full", kind="adapters", layout="streams", batch=2, text=512, image=8192, K=2048, N=8192, rank=64, adapters=4,
             gelu=True),
    ]


def _widths(case):
    """Elements of a head that turn with each axis."""
    return [int(w) for w in case["widths"].split()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm_grad", "rotary", "adapters", "adapters"])
        if kind in ("norm", "norm_grad"):
            case = dict(kind=kind, layout="streams", batch=rng.choice([1, 1, 2, 4]), text=_log_int(rng, 1, 1024), image=_log_int(rng, 1, 9216),
                        C=8 * _log_int(rng, 16, 1024), residual=rng.random() < 0.5, affine=rng.random() < 0.3)
        elif kind == "rotary":
            src = _log_int(rng, 1, 24000)
            gather, inverse = rng.random() < 0.5, rng.random() < 0.25
            heads = rng.choice([1, 3, 8, 16, 24])
            case = dict(kind=kind, batch=rng.choice([1, 1, 2, 5]), src=src, rows=rng.randint(1, src) if gather else src, gather=gather,
                        Hq=heads, Hk=rng.choice([heads, 1]),
                        widths=rng.choice(["16 56 56", "16 24 24", "32 32 32", "44 42 42", "64 64", "64", "16 16 16 16"]),
                        halves=rng.random() < 0.5, normalise=not inverse and rng.random() < 0.7, inverse=inverse)
        else:
            case = dict(kind=kind, K=8 * _log_int(rng, 32, 1024), N=8 * _log_int(rng, 8, 1024), rank=8 * _log_int(rng, 1, 16),
                        adapters=_log_int(rng, 1, 48), gelu=rng.random() < 0.5)
            if rng.random() < 0.5:
                case.update(layout="streams", batch=rng.choice([1, 2, 4, 8]), text=_log_int(rng, 1, 1024), image=_log_int(rng, 1, 9216))
            else:
                case.update(layout="tokens", batch=_log_int(rng, 1, 256))
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


def _groups(case, seed):
    """[(first row, row behind the last)] and the rows of the buffers."""
    if case["layout"] == "tokens":
        return [(b, b + 1) for b in range(case["batch"])], case["batch"]
    rng = np.random.default_rng([seed, 1])
    room, out = case["text"] + case["image"], []
    for b in range(case["batch"]):
        live = case["image"] if case["batch"] == 1 else int(rng.integers(max(1, case["image"] * 3 // 4), case["image"] + 1))
        mid = b * room + case["text"]
        out += [(b * room, mid), (mid, mid + live)]
    return out, case["batch"] * room


def _sets(case):
    """Weight or parameter sets: group g has set g mod this."""
    if case["kind"] == "adapters":
        return 2 if case["layout"] == "streams" else 1
    return 1 if case["affine"] else 2 * case["batch"]


def _adapter_of(case, seed):
    """The groups' adapters; an eighth of the requests have none."""
    rng = np.random.default_rng([seed, 2])
    groups = len(_groups(case, seed)[0])
    return [int(a) for a in np.where(rng.random(groups) < 0.125, -1, rng.integers(0, case["adapters"], groups))]


def work(case):
    kind = case["kind"]
    if kind == "rotary":
        D, rows = sum(_widths(case)), case["batch"] * case["rows"]
        n = rows * (case["Hq"] + case["Hk"]) * D
        return {"bytes": 4.0 * n + rows * 4 * (len(_widths(case)) + case["gather"]), "flops": (7.0 if case["normalise"] else 3.0) * n}
    groups = _groups(case, 0)[0]                                   # (other seeds: nearly as many rows)
    rows = sum(e - b for b, e in groups)
    if kind == "norm":
        n, params = rows * case["C"], _sets(case) * case["C"]
        return {"bytes": n * (8.0 if case["residual"] else 4.0) + params * (6.0 if case["residual"] else 4.0),
                "flops": n * (9.0 if case["residual"] else 7.0)}
    if kind == "norm_grad":
        n, params = rows * case["C"], _sets(case) * case["C"]
        return {"bytes": n * (12.0 if case["residual"] else 6.0) + 8.0 * rows + params * (16.0 if case["residual"] else 10.0),
                "flops": n * (17.0 if case["residual"] else 13.0)}
    K, N, R = case["K"], case["N"], case["rank"]
    on = [(g, a) for g, a in zip(groups, _adapter_of(case, 0)) if a >= 0]
    adapted = sum(e - b for (b, e), _ in on)
    return {"bytes": 2.0 * (rows * (K + N) + _sets(case) * N * (K + 1) + len({a for _, a in on}) * R * (K + N)),
            "flops": 2.0 * rows * N * K + 2.0 * adapted * R * (K + N)}


def _normal(gen, shape, std=1.0):
    return (torch.randn(shape, device="cuda", dtype=F32, generator=gen) * std).to(BF)


def _frequencies(widths):
    """Radians a unit of position for every pair of a head, and the axis it turns with."""
    return ([10000.0 ** (-2.0 * i / w) for w in widths for i in range(w // 2)], [a for a, w in enumerate(widths) for i in range(w // 2)])


def _positions(case, gen):
    """[batch, src, axes]: on a grid of frames, rows and columns; a quarter of the requests have a resized image, whose places lie between
    whole numbers."""
    axes, src = len(_widths(case)), case["src"]
    i = torch.arange(src, device="cuda")
    side = max(1, int(math.sqrt(min(src, 4096))))
    at = [i // (side * side), i // side % side, i % side, i % 7][:axes] if axes > 1 else [i]
    grid = torch.stack(at, -1).float().expand(case["batch"], -1, -1).contiguous()
    start = torch.randint(0, 64, (case["batch"], 1, axes), device="cuda", generator=gen).float()
    resized = torch.rand((case["batch"], 1, 1), device="cuda", generator=gen) < 0.25
    return torch.where(resized, grid * 0.8125, grid) + start


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    s = dict(case)
    if case["kind"] == "rotary":
        B, D = case["batch"], sum(_widths(case))
        s["freq"], s["axis"] = _frequencies(_widths(case))
        s["positions"] = _positions(case, gen)
        s["q"], s["k"] = (_normal(gen, (B, case["src"], case[h], D)) for h in ("Hq", "Hk"))
        s["q_weight"], s["k_weight"] = ((1.0 + 0.2 * torch.randn(D, device="cuda", generator=gen)).to(BF) for _ in range(2))
        s["idx"] = None
        if case["gather"]:
            s["idx"] = torch.stack([torch.randperm(case["src"], device="cuda", generator=gen)[:case["rows"]].sort().values
                                    for _ in range(B)]).to(I32)
        s["q_out"], s["k_out"] = (torch.zeros((B, case["rows"], case[h], D), dtype=BF, device="cuda") for h in ("Hq", "Hk"))
        return s
    s["groups"], rows = _groups(case, seed)
    s["begin"] = torch.tensor([g[0] for g in s["groups"]], dtype=I32, device="cuda")
    s["end"] = torch.tensor([g[1] for g in s["groups"]], dtype=I32, device="cuda")
    sets = _sets(case)
    if case["kind"] == "adapters":
        K, N, R, n = case["K"], case["N"], case["rank"], case["adapters"]
        s["adapter_of"] = _adapter_of(case, seed)
        s["adapter"] = torch.tensor(s["adapter_of"], dtype=I32, device="cuda")
        s["x"] = _normal(gen, (rows, K))
        s["w"] = _normal(gen, (sets, N, K), K ** -0.5)
        s["bias"] = _normal(gen, (sets, N), 0.1)
        s["a"] = _normal(gen, (n, R, K), K ** -0.5)
        s["b"] = _normal(gen, (n, N, R), 0.25 * R ** -0.5)
        s["scale"] = 0.5 + 1.5 * torch.rand(n, device="cuda", generator=gen)
        s["out"] = torch.zeros((rows, N), dtype=BF, device="cuda")
        if own:
            from paper_2510_25590_b200 import binding
            nbytes = binding.adapter_matmul_workspace(rows, len(s["groups"]), K, N, R)
            s["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        return s
    C = case["C"]
    if case["affine"]:
        s["weight"] = (1.0 + 0.2 * torch.randn((1, C), device="cuda", generator=gen)).to(BF)
        s["bias"], s["gate"] = _normal(gen, (1, C), 0.1), _normal(gen, (1, C), 0.5)
    else:
        mods = _normal(gen, (sets, 6 * C), 0.3)                    # what the modulation's product leaves, in six parts
        s["bias"], s["weight"], s["gate"] = mods[:, :C], mods[:, C:2 * C], mods[:, 2 * C:3 * C]
    # residual stream: some channels much larger than the others, and a mean
    s["x"] = (torch.randn((rows, C), device="cuda", generator=gen) * torch.exp(torch.randn(C, device="cuda", generator=gen)) + 0.25).to(BF)
    s["r"] = _normal(gen, (rows, C)) if case["residual"] else None
    s["out"] = torch.zeros((rows, C), dtype=BF, device="cuda")
    s["x_out"] = torch.zeros((rows, C), dtype=BF, device="cuda") if case["residual"] else None
    if case["kind"] == "norm_grad":
        z = s["x"].double()
        s["mean"] = z.mean(-1).float()
        s["rstd"] = torch.rsqrt((z - z.mean(-1, keepdim=True)).square().mean(-1) + EPS).float()
        s["dy"] = _normal(gen, (rows, C), 0.01)
        s["dz"] = _normal(gen, (rows, C), 0.01) if case["residual"] else None
        s["dr"] = torch.zeros((rows, C), dtype=BF, device="cuda") if case["residual"] else None
        s["dweight"], s["dbias"], s["dgate"] = (torch.zeros((sets, C), dtype=F32, device="cuda") for _ in range(3))
        if own:
            from paper_2510_25590_b200 import binding
            nbytes = binding.layer_norm_backward_workspace(rows, len(s["groups"]), C)
            s["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return s


def _gelu(x):
    return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))


def _turn(y, cos, sin, halves):
    out = torch.empty_like(y)
    half = y.shape[-1] // 2
    first, second = (slice(None, half), slice(half, None)) if halves else (slice(0, None, 2), slice(1, None, 2))
    out[..., first] = y[..., first] * cos - y[..., second] * sin
    out[..., second] = y[..., first] * sin + y[..., second] * cos
    return out


def _outputs(s):
    if s["kind"] == "norm":
        return (s["x_out"], s["out"]) if s["residual"] else (s["out"],)
    if s["kind"] == "norm_grad":
        return (s["out"], s["dr"], s["dweight"], s["dbias"], s["dgate"]) if s["residual"] else (s["out"], s["dweight"], s["dbias"])
    return s["out"]


def _run_plain(s):
    kind = s["kind"]
    if kind == "rotary":
        at = s["positions"].double()
        if s["idx"] is not None:
            at = torch.gather(at, 1, s["idx"].long()[..., None].expand(-1, -1, at.shape[2]))
        angle = at[:, :, s["axis"]] * torch.tensor(s["freq"], dtype=F64, device="cuda")
        cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
        for name in ("q", "k"):
            x = s[name].float() if s["idx"] is None else \
                torch.stack([s[name][b][s["idx"][b].long()] for b in range(s["batch"])]).float()
            if s["normalise"]:
                x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s[name + "_weight"].float()
            s[name + "_out"].copy_(_turn(x, cos, -sin if s["inverse"] else sin, s["halves"]))
        return s["q_out"], s["k_out"]
    if kind == "adapters":
        sets = s["w"].shape[0]
        for g, (b, e) in enumerate(s["groups"]):
            i, a = g % sets, s["adapter_of"][g]
            if s["layout"] == "tokens" and g > 0:
                continue                                            # (one weight set: all rows at once, below)
            b, e = (0, s["batch"]) if s["layout"] == "tokens" else (b, e)
            y = s["x"][b:e].float() @ s["w"][i].float().T + s["bias"][i].float()
            if s["layout"] == "tokens":
                on = [r for r in range(e) if s["adapter_of"][r] >= 0]
                which = [s["adapter_of"][r] for r in on]
                u = torch.einsum("rk,rjk->rj", s["x"][on].float(), s["a"][which].float()) * s["scale"][which][:, None]
                y[on] += torch.einsum("rj,rnj->rn", u, s["b"][which].float())
            elif a >= 0:
                y += ((s["x"][b:e].float() @ s["a"][a].float().T) * s["scale"][a]) @ s["b"][a].float().T
            s["out"][b:e] = (_gelu(y) if s["gelu"] else y).to(BF)
        return _outputs(s)
    sets = s["weight"].shape[0]
    for name in ("dweight", "dbias", "dgate"):
        if kind == "norm_grad":
            s[name].zero_()
    for g, (b, e) in enumerate(s["groups"]):
        i = g % sets
        w = s["weight"][i].float() + (0.0 if s["affine"] else 1.0)
        z = s["x"][b:e].float()
        if kind == "norm":
            if s["residual"]:
                s["x_out"][b:e] = (z + s["gate"][i].float() * s["r"][b:e].float()).to(BF)
                z = s["x_out"][b:e].float()
            z = z - z.mean(-1, keepdim=True)
            s["out"][b:e] = (z * torch.rsqrt((z * z).mean(-1, keepdim=True) + EPS) * w + s["bias"][i].float()).to(BF)
            continue
        h, dy = (z - s["mean"][b:e, None]) * s["rstd"][b:e, None], s["dy"][b:e].float()
        a = dy * w
        d = (a - a.mean(-1, keepdim=True) - h * (a * h).mean(-1, keepdim=True)) * s["rstd"][b:e, None]
        if s["residual"]:
            d = d + s["dz"][b:e].float()
            s["dr"][b:e] = (d * s["gate"][i].float()).to(BF)
            s["dgate"][i] += (d * s["r"][b:e].float()).sum(0)
        s["out"][b:e] = d.to(BF)
        s["dweight"][i] += (dy * h).sum(0)
        s["dbias"][i] += dy.sum(0)
    return _outputs(s)


def _run_own(s):
    from paper_2510_25590_b200 import binding
    if s["kind"] == "rotary":
        extra = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS) if s["normalise"] else {}
        binding.rotary_axes(s["q"], s["k"], s["positions"], s["freq"], s["axis"], s["q_out"], s["k_out"],
                            binding.ROPE_HALF if s["halves"] else binding.ROPE_INTERLEAVED, idx=s["idx"], inverse=s["inverse"], **extra)
        return s["q_out"], s["k_out"]
    if s["kind"] == "adapters":
        binding.adapter_matmul(s["x"], s["w"], s["a"], s["b"], s["adapter"], s["begin"], s["end"], s["out"], s["workspace"], scale=s["scale"],
                               bias=s["bias"], activation=binding.ACT_GELU_TANH if s["gelu"] else binding.ACT_NONE)
    elif s["kind"] == "norm":
        extra = dict(residual=s["r"], gate=s["gate"], x_out=s["x_out"]) if s["residual"] else {}
        binding.layer_norm(s["x"], s["weight"], s["bias"], s["begin"], s["end"], s["out"], EPS, modulated=not s["affine"], **extra)
    else:
        extra = dict(dx_out=s["dz"], residual=s["r"], gate=s["gate"], dresidual=s["dr"], dgate=s["dgate"]) if s["residual"] else {}
        binding.layer_norm_backward(s["x"], s["mean"], s["rstd"], s["dy"], s["weight"], s["begin"], s["end"], s["out"], s["dweight"],
                                    s["dbias"], s["workspace"], modulated=not s["affine"], **extra)
    return _outputs(s)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotary":
        D = sum(_widths(case))
        freq = torch.tensor([math.pow(10000.0, -2.0 * i / w) for w in _widths(case) for i in range(w // 2)], dtype=F64, device="cuda")
        axis = torch.tensor([a for a, w in enumerate(_widths(case)) for _ in range(w // 2)], device="cuda")
        out = []
        for name in ("q", "k"):
            side = []
            for b in range(case["batch"]):
                at = torch.arange(case["rows"], device="cuda") if s["idx"] is None else s["idx"][b].long()
                x = s[name][b].index_select(0, at).double()
                if case["normalise"]:
                    x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + EPS) * s[name + "_weight"].double()
                t = s["positions"][b].double().index_select(0, at).index_select(1, axis) * freq
                z = torch.polar(torch.ones_like(t), -t if case["inverse"] else t)[:, None]
                if case["halves"]:
                    y = torch.complex(x[..., :D // 2], x[..., D // 2:]) * z
                    side.append(torch.cat([y.real, y.imag], -1))
                else:
                    side.append(torch.view_as_real(torch.view_as_complex(x.unflatten(-1, (-1, 2)).contiguous()) * z).flatten(-2))
            out.append(torch.stack(side))
        return tuple(out)
    if kind == "adapters":
        out = torch.zeros(s["out"].shape, dtype=F64, device="cuda")
        sets = _sets(case)
        whole = [None] * sets
        for g, ((b, e), a) in enumerate(zip(s["groups"], s["adapter_of"])):
            if whole[g % sets] is None:
                whole[g % sets] = s["w"][g % sets].double()
            x = s["x"][b:e].double()
            y = torch.matmul(x, whole[g % sets].T) + s["bias"][g % sets].double()
            if a >= 0:
                y += torch.matmul(torch.matmul(x, s["a"][a].double().T), s["b"][a].double().T) * s["scale"][a].double()
            if case["gelu"]:
                y = y / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
            out[b:e] = y
        return out
    sets, C = _sets(case), case["C"]
    rows = torch.cat([torch.arange(b, e, device="cuda") for b, e in s["groups"]])
    of = torch.cat([torch.full((e - b,), g % sets, device="cuda") for g, (b, e) in enumerate(s["groups"])])
    full = lambda: torch.zeros((s["x"].shape[0], C), dtype=F64, device="cuda")
    out, x_out, dr = full(), full(), full()
    sums = [torch.zeros((sets, C), dtype=F64, device="cuda") for _ in range(3)]
    for j in range(0, len(rows), 4096):
        at, i = rows[j:j + 4096], of[j:j + 4096]
        z, w = s["x"][at].double(), s["weight"].double()[i] + (0 if case["affine"] else 1)
        if kind == "norm" and case["residual"]:
            x_out[at] = z + s["gate"].double()[i] * s["r"][at].double()
            z = x_out[at].to(BF).double()                           # (the norm is that of the row as it is kept)
        mean = z.sum(-1, keepdim=True) / C
        std = torch.sqrt((z - mean).pow(2).sum(-1, keepdim=True) / C + EPS)
        h = (z - mean) / std
        if kind == "norm":
            out[at] = h * w + s["bias"].double()[i]
            continue
        dy = s["dy"][at].double()
        a = dy * w
        d = (a - a.sum(-1, keepdim=True) / C - h * ((a * h).sum(-1, keepdim=True) / C)) / std
        if case["residual"]:
            d += s["dz"][at].double()
            dr[at] = d * s["gate"].double()[i]
            sums[2].index_add_(0, i, d * s["r"][at].double())
        out[at] = d
        sums[0].index_add_(0, i, dy * h)
        sums[1].index_add_(0, i, dy)
    if kind == "norm":
        return (x_out, out) if case["residual"] else (out,)
    return (out, dr, *sums) if case["residual"] else (out, sums[0], sums[1])
