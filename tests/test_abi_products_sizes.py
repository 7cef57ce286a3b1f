"""Sizes of the 4-bit format whose product passes 64 bits (CPU only: fake addresses, nothing may be launched)."""
import ctypes

from paper_2510_25590_b200 import binding

FAKE, NULL = ctypes.c_void_p(4096), None


def test_mxfp4_sizes_that_pass_64_bits():
    """Numbers of elements are counted in 64 bits: what does not fit is refused before anything is multiplied."""
    lib = binding.load()
    many, wide = (1 << 31) - 1, (1 << 31) - 32
    assert lib.regione_mxfp4_quantize(FAKE, NULL, NULL, 4, many, many, wide, FAKE, FAKE, NULL, NULL) == binding.UNSUPPORTED
    assert lib.regione_mxfp4_quantize(FAKE, FAKE, FAKE, many, many, many, wide, FAKE, FAKE, NULL, NULL) == binding.UNSUPPORTED
    assert lib.regione_mxfp4_dequantize(FAKE, FAKE, NULL, 8, many, wide, FAKE, NULL, NULL) == binding.UNSUPPORTED
    assert lib.regione_mxfp4_dequantize(FAKE, FAKE, FAKE, many, many, wide, FAKE, NULL, NULL) == binding.UNSUPPORTED
    assert lib.regione_rikv_store_mxfp4(FAKE, FAKE, FAKE, FAKE, many, 8, many, many, 128, FAKE, FAKE, FAKE, FAKE, NULL, NULL) == binding.UNSUPPORTED
    assert lib.regione_rikv_load_mxfp4(FAKE, FAKE, FAKE, FAKE, FAKE, many, many, many, 128, FAKE, FAKE, NULL, NULL) == binding.UNSUPPORTED
