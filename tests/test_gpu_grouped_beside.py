"""Grouped products beside the attention, on streams of their own and in turn on one: both use tensor memory, and each gives what it gives
alone."""
import pytest

from gpu_util import dev_i32
from paper_2510_25590_b200 import binding

pytestmark = pytest.mark.gpu


def _attention(gen, D, rows, kept, H=4):
    import torch
    t = lambda n: torch.randn((1, n, H, D), device="cuda", generator=gen).to(torch.bfloat16)
    q, k, v, kc, vc = t(rows), t(rows), t(rows), t(kept), t(kept)
    n, c, out = dev_i32([rows]), dev_i32([kept]), torch.empty_like(q)
    ws = torch.empty(binding.region_attention_workspace(1, rows, rows, kept, H, D), dtype=torch.uint8, device="cuda")
    return out, lambda stream: binding.region_attention(q, k, v, kc, vc, n, n, c, out, workspace=ws, stream=stream)


def _products(gen, fp4, rows, K, N):
    import torch
    x, w = (torch.randn(s, device="cuda", generator=gen).to(torch.bfloat16) for s in ((1, rows, K), (1, N, K)))
    begin, end, out = dev_i32([0]), dev_i32([rows]), torch.empty((rows, N), dtype=torch.bfloat16, device="cuda")
    if not fp4:
        return out, lambda stream: binding.grouped_matmul(x[0], w, begin, end, out, stream=stream)
    u = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
    xq, xs, wq, ws = u(1, rows, K // 2), u(1, rows, K // 32), u(1, N, K // 2), u(1, N, K // 32)
    binding.mxfp4_quantize(w, wq, ws)

    def call(stream):
        binding.mxfp4_quantize(x, xq, xs, stream=stream)
        binding.mxfp4_grouped_matmul(xq[0], xs[0], wq, ws, begin, end, out, stream=stream)
    return out, call


@pytest.mark.parametrize("together", ["streams", "in turn"])
@pytest.mark.parametrize("D", [64, 128])
def test_beside_the_attention(D, together):
    import torch
    gen = torch.Generator("cuda").manual_seed(D)
    parts = [_attention(gen, D, 300, 1500), _products(gen, False, 5, 1024, 1536), _products(gen, True, 5, 1024, 1536),
             _attention(gen, D, 70, 200), _products(gen, False, 2000, 512, 2048), _products(gen, True, 2000, 512, 2048)]
    here = torch.cuda.current_stream()
    alone = []
    for out, call in parts:
        call(here)
        torch.cuda.synchronize()
        alone.append(out.clone())
        out.fill_(-7.0)
    streams = [torch.cuda.Stream() if together == "streams" else here for _ in parts]
    torch.cuda.synchronize()
    for _ in range(30):
        for stream, (out, call) in zip(streams, parts):
            call(stream)
    torch.cuda.synchronize()
    for (out, call), want in zip(parts, alone):
        assert torch.equal(out, want)
