"""What the CTAs of a pair hand each other: scales that one CTA brings are multiplied by products that the other issues, and accumulators
that one reads out are overwritten by them.  Whole numbers whose scales differ from block to block and from row to row: a scale or an
accumulator of another chunk, tile or CTA changes the sums, which are exact in fp32 in any order (at most 4096 * 48 * 24 < 2^23)."""
import pytest

from gpu_util import dev_i32
from paper_2510_25590_b200 import binding

pytestmark = pytest.mark.gpu

# many rounds of tiles a pair (both accumulators again and again); few tiles with many chunks; a last tile of few rows
CASES = [(5000, 512, 4096), (1700, 4096, 2048), (2309, 1152, 1000), (4111, 2048, 1544)]


def _whole(gen, shape):
    """E2M1 values times 1, 2, 4 or 8 by block and row: whole numbers up to 48, exact in the 4-bit format."""
    import torch
    table = torch.tensor([0., 1., 2., 3., 4., 6., -1., -2., -3., -4., -6.], device="cuda")
    x = table[torch.randint(0, 11, shape, device="cuda", generator=gen)].unflatten(-1, (-1, 32))
    x[..., 0] = 6.0                                                    # (every block's scale is the one drawn for it)
    x = x * torch.exp2(torch.randint(0, 4, x.shape[:-1] + (1,), device="cuda", generator=gen).float())
    return x.flatten(-2).to(torch.bfloat16)


def _codes(x):
    import torch
    shape = (1, x.numel() // x.shape[-1], x.shape[-1])
    c = torch.empty(shape[:2] + (shape[2] // 2,), dtype=torch.uint8, device="cuda")
    s = torch.empty(shape[:2] + (shape[2] // 32,), dtype=torch.uint8, device="cuda")
    binding.mxfp4_quantize(x.reshape(shape), c, s)
    return c.view(x.shape[:-1] + (-1,)), s.view(x.shape[:-1] + (-1,))


def _call(fp4, x, w, begin, end, out):
    if fp4:
        cx, cw = _codes(x), _codes(w)
        return lambda: binding.mxfp4_grouped_matmul(*cx, *cw, begin, end, out)
    return lambda: binding.grouped_matmul(x, w, begin, end, out)


@pytest.mark.parametrize("rows,K,N", CASES)
@pytest.mark.parametrize("fp4", [False, True], ids=["bf16", "mxfp4"])
def test_handed_over_whole(fp4, rows, K, N):
    import torch
    gen = torch.Generator("cuda").manual_seed(rows + K)
    x, w = _whole(gen, (rows, K)), _whole(gen, (2, N, K)) / 2           # (halves: sums below 2^23 keep them)
    mid = rows // 3
    begin, end = dev_i32([0, mid]), dev_i32([mid, rows])
    out = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda")
    call = _call(fp4, x, w, begin, end, out)
    want = torch.cat([x[:mid].double() @ w[0].double().T, x[mid:].double() @ w[1].double().T]).float().to(torch.bfloat16)
    for _ in range(30):
        out.fill_(-7.0)
        call()
        assert torch.equal(out, want)


@pytest.mark.parametrize("rows,K,N", [(1, 1024, 264), (17, 4096, 136), (300, 1920, 520), (1700, 4096, 2048), (5000, 512, 1000)])
@pytest.mark.parametrize("fp4", [False, True], ids=["bf16", "mxfp4"])
def test_calls_repeat_bit_for_bit(fp4, rows, K, N):
    """Numbers whose sums depend on the order of the additions: it is the same in every call."""
    import torch
    gen = torch.Generator("cuda").manual_seed(rows)
    x, w = (torch.randn(s, device="cuda", generator=gen).to(torch.bfloat16) for s in ((rows, K), (1, N, K)))
    out = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda")
    call = _call(fp4, x, w, dev_i32([0]), dev_i32([rows]), out)
    call()
    first = out.clone()
    for _ in range(20):
        out.fill_(-7.0)
        call()
        assert torch.equal(out, first)
