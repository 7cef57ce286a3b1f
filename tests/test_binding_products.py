"""What the binding refuses of the grouped products and the 4-bit format before it calls the library (CPU only: stand-ins for the
tensors and for the library)."""
import pytest
import torch

from paper_2510_25590_b200 import binding

BF, U8, I32 = torch.bfloat16, torch.uint8, torch.int32


class Tensor:
    """What the binding asks of a CUDA tensor."""
    is_cuda = True

    def __init__(self, shape, dtype, at=0):
        self.shape, self.dtype, self.at, self.device = torch.Size(shape), dtype, at, f"cuda:{at}"

    def get_device(self):
        return self.at

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def numel(self):
        return self.shape.numel()

    def stride(self, d=None):
        s = torch.empty(self.shape, device="meta").stride()
        return s if d is None else s[d]


class Stream:
    cuda_stream = 0


@pytest.fixture
def called(monkeypatch):
    """The library's calls, which succeed; device 0 is current."""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or binding.OK

    monkeypatch.setattr(binding, "load", lambda *a: Library())
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    return calls


B, R, CAP, K, N, H, D = 2, 9, 5, 128, 24, 3, 64
CALLS = {
    "mxfp4_quantize": dict(x=((B, R, K), BF), codes=((B, CAP, K // 2), U8), scales=((B, CAP, K // 32), U8), idx=((B, CAP), I32), n=((B,), I32)),
    "mxfp4_dequantize": dict(codes=((B, CAP, K // 2), U8), scales=((B, CAP, K // 32), U8), x=((B, CAP, K), BF), n=((B,), I32)),
    "rikv_store_mxfp4": dict(k_full=((B, R, H, D), BF), v_full=((B, R, H, D), BF), keep_rows=((B, CAP), I32), n_keep=((B,), I32),
                             k_q=((B, CAP, H, D // 2), U8), v_q=((B, CAP, H, D // 2), U8), k_scale=((B, CAP, H, D // 32), U8),
                             v_scale=((B, CAP, H, D // 32), U8)),
    "rikv_load_mxfp4": dict(k_q=((B, CAP, H, D // 2), U8), v_q=((B, CAP, H, D // 2), U8), k_scale=((B, CAP, H, D // 32), U8),
                            v_scale=((B, CAP, H, D // 32), U8), n_keep=((B,), I32), k_cache=((B, CAP, H, D), BF),
                            v_cache=((B, CAP, H, D), BF)),
    "grouped_matmul": dict(x=((R, K), BF), w=((2, N, K), BF), row_begin=((2,), I32), row_end=((2,), I32), out=((R, N), BF), bias=((2, N), BF)),
    "mxfp4_grouped_matmul": dict(x_q=((R, K // 2), U8), x_scale=((R, K // 32), U8), w_q=((2, N, K // 2), U8), w_scale=((2, N, K // 32), U8),
                                 row_begin=((2,), I32), row_end=((2,), I32), out=((R, N), BF), bias=((2, N), BF)),
}
EACH = [(name, arg) for name, args in CALLS.items() for arg in (*args, "dev_status")]


def _args(name, **other):
    args = {arg: Tensor(*spec) for arg, spec in CALLS[name].items()}
    return {**args, "dev_status": Tensor((1,), I32), "stream": Stream(), **other}


@pytest.mark.parametrize("name", CALLS)
def test_the_calls_as_they_are_meant(called, name):
    getattr(binding, name)(**_args(name))
    assert called == ["regione_" + name]


@pytest.mark.parametrize("name,arg", EACH)
def test_a_tensor_of_another_device_is_refused(called, name, arg):
    shape, dtype = CALLS[name].get(arg, ((1,), I32))
    with pytest.raises(binding.RegionEError, match=f"^{arg} is on cuda:1"):
        getattr(binding, name)(**_args(name, **{arg: Tensor(shape, dtype, at=1)}))
    assert not called


@pytest.mark.parametrize("name,arg", [(name, arg) for name, args in CALLS.items() for arg in args])
@pytest.mark.parametrize("other", ["fewer dimensions", "more dimensions", "no tensor"])
def test_other_dimensions_are_refused_by_name(called, name, arg, other):
    """By the library's own error, whatever is wrong with the argument."""
    shape, dtype = CALLS[name][arg]
    t = {"fewer dimensions": Tensor(shape[1:], dtype), "more dimensions": Tensor((1, *shape), dtype), "no tensor": list(range(3))}[other]
    with pytest.raises(binding.RegionEError, match=rf"^{arg} |row_end must have shape" if arg == "row_begin" else f"^{arg} "):
        getattr(binding, name)(**_args(name, **{arg: t}))
    assert not called
