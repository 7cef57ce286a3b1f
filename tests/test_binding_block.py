"""What the binding refuses of the layer norm, the rotary positions and the products with adapters before it calls the library (CPU only:
stand-ins for the tensors and for the library)."""
import pytest
import torch

from paper_2510_25590_b200 import binding
from test_binding_products import Stream, Tensor as Plain, called    # noqa: F401  (called: a fixture)

BF, U8, I32, F32 = torch.bfloat16, torch.uint8, torch.int32, torch.float32


class Tensor(Plain):
    @property
    def nbytes(self):
        return self.numel() * self.dtype.itemsize


R, C, G, B, CAP, P, D, K, N = 9, 64, 4, 2, 5, 7, 64, 128, 24
CALLS = {
    "layer_norm": dict(x=((R, C), BF), weight=((G, C), BF), bias=((G, C), BF), row_begin=((G,), I32), row_end=((G,), I32), out=((R, C), BF),
                       residual=((R, C), BF), gate=((G, C), BF), x_out=((R, C), BF), mean=((R,), F32), rstd=((R,), F32)),
    "layer_norm_backward": dict(x=((R, C), BF), mean=((R,), F32), rstd=((R,), F32), dy=((R, C), BF), weight=((G, C), BF), row_begin=((G,), I32),
                                row_end=((G,), I32), dx=((R, C), BF), dweight=((G, C), F32), dbias=((G, C), F32), workspace=((4096,), U8),
                                dx_out=((R, C), BF), residual=((R, C), BF), gate=((G, C), BF), dresidual=((R, C), BF), dgate=((G, C), F32)),
    "rotary_axes": dict(q=((B, P, 3, D), BF), k=((B, P, 2, D), BF), positions=((B, P, 3), F32), q_out=((B, CAP, 3, D), BF), k_out=((B, CAP, 2, D), BF),
                        idx=((B, CAP), I32), n=((B,), I32), q_weight=((D,), BF), k_weight=((D,), BF)),
    "adapter_matmul": dict(x=((R, K), BF), w=((2, N, K), BF), a=((3, 16, K), BF), b=((3, N, 16), BF), adapter=((G,), I32), row_begin=((G,), I32),
                           row_end=((G,), I32), out=((R, N), BF), workspace=((4096,), U8), scale=((3,), F32), bias=((2, N), BF)),
}
MORE = {"layer_norm": dict(eps=1e-6), "rotary_axes": dict(freq=[0.5] * (D // 2), axis=[0] * (D // 2), layout=binding.ROPE_HALF, eps=1e-6)}
EACH = [(name, arg) for name, args in CALLS.items() for arg in args]


def _args(name, **other):
    args = {arg: Tensor(*spec) for arg, spec in CALLS[name].items()}
    return {**args, **MORE.get(name, {}), "dev_status": Tensor((1,), I32), "stream": Stream(), **other}


@pytest.mark.parametrize("name", CALLS)
def test_the_calls_as_they_are_meant(called, name):
    getattr(binding, name)(**_args(name))
    assert called == ["regione_" + name]


@pytest.mark.parametrize("name,arg", EACH + [(name, "dev_status") for name in CALLS])
def test_a_tensor_of_another_device_is_refused(called, name, arg):
    shape, dtype = CALLS[name].get(arg, ((1,), I32))
    with pytest.raises(binding.RegionEError, match=f"^{arg} is on cuda:1"):
        getattr(binding, name)(**_args(name, **{arg: Tensor(shape, dtype, at=1)}))
    assert not called


@pytest.mark.parametrize("name,arg", EACH)
@pytest.mark.parametrize("other", ["fewer dimensions", "more dimensions", "one more", "no tensor"])
def test_other_shapes_are_refused(called, name, arg, other):
    shape, dtype = CALLS[name][arg]
    if arg == "workspace" and other != "no tensor" or arg == "positions" and other == "one more":
        return                                                         # (of any shape, of any number of axes: the library sees the size)
    t = {"fewer dimensions": Tensor(shape[1:], dtype), "more dimensions": Tensor((1, *shape), dtype),
         "one more": Tensor((*shape[:-1], shape[-1] + 8), dtype), "no tensor": list(range(3))}[other]
    with pytest.raises(binding.RegionEError):
        getattr(binding, name)(**_args(name, **{arg: t}))
    assert not called


@pytest.mark.parametrize("name,arg", [(n, a) for n, a in EACH if a != "workspace"])
def test_other_types_are_refused(called, name, arg):
    shape, dtype = CALLS[name][arg]
    other = torch.float16 if dtype != torch.float16 else BF
    with pytest.raises(binding.RegionEError):
        getattr(binding, name)(**_args(name, **{arg: Tensor(shape, other)}))
    assert not called


@pytest.mark.parametrize("name,kw", [("layer_norm", dict(residual=None)), ("layer_norm", dict(x_out=None)), ("layer_norm", dict(residual=None, x_out=None)),
                                     ("layer_norm_backward", dict(residual=None)), ("layer_norm_backward", dict(gate=None)),
                                     ("layer_norm_backward", dict(dresidual=None)),
                                     ("layer_norm_backward", dict(residual=None, gate=None, dresidual=None)),
                                     ("rotary_axes", dict(k=None)), ("rotary_axes", dict(k_out=None)), ("rotary_axes", dict(eps=None)),
                                     ("rotary_axes", dict(freq=[0.5])), ("rotary_axes", dict(axis=[0])), ("rotary_axes", dict(axis=[0.5] * (D // 2))),
                                     ("rotary_axes", dict(freq="x" * (D // 2))), ("rotary_axes", dict(src_compact=True))], ids=str)
def test_what_does_not_go_together(called, name, kw):
    with pytest.raises(binding.RegionEError):
        getattr(binding, name)(**_args(name, **kw))
    assert not called


def test_what_may_be_left_out(called):
    binding.layer_norm(**_args("layer_norm", residual=None, x_out=None, gate=None, weight=None, bias=None, mean=None, rstd=None))
    binding.layer_norm(**_args("layer_norm", gate=None))
    binding.layer_norm_backward(**_args("layer_norm_backward", dweight=None, dbias=None, dgate=None, dx_out=None))
    binding.layer_norm_backward(**_args("layer_norm_backward", residual=None, gate=None, dresidual=None, dgate=None, weight=None))
    binding.rotary_axes(**_args("rotary_axes", k=None, k_out=None, n=None, q_weight=None, k_weight=None, eps=None))
    binding.adapter_matmul(**_args("adapter_matmul", scale=None, bias=None))
    assert len(called) == 6


def test_frequencies():
    freq, axis = binding.rotary_frequencies((16, 56, 56))
    assert len(freq) == len(axis) == 64 and axis == [0] * 8 + [1] * 28 + [2] * 28
    assert freq[0] == freq[8] == freq[36] == 1.0 and abs(freq[7] - 10000.0 ** (-14 / 16)) < 1e-15
    with pytest.raises(binding.RegionEError):
        binding.rotary_frequencies((15, 49))
