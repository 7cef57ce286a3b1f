"""Refusals of the grouped products and of the 4-bit format, on the host (CPU only: fake addresses, nothing may be launched)."""
import ctypes

from paper_2510_25590_b200 import binding

FAKE, ODD, NULL = ctypes.c_void_p(4096), ctypes.c_void_p(4100), None


def _grouped(x=FAKE, xs=64, w=FAKE, bias=NULL, begin=FAKE, end=FAKE, rows=4, groups=1, sets=1, K=64, N=16, act=0, out=FAKE, os=16):
    return binding.load().regione_grouped_matmul(x, xs, w, bias, begin, end, rows, groups, sets, K, N, act, out, os, NULL, NULL)


def test_grouped_matmul():
    for kw in (dict(x=NULL), dict(w=NULL), dict(begin=NULL), dict(end=NULL), dict(out=NULL), dict(x=ODD), dict(w=ODD), dict(out=ODD),
               dict(bias=ODD), dict(rows=-1), dict(groups=-1), dict(sets=0), dict(K=0), dict(N=0), dict(act=2), dict(act=-1), dict(xs=56),
               dict(os=8)):
        assert _grouped(**kw) == binding.INVALID_ARG, kw
    for kw in (dict(K=60), dict(N=12), dict(xs=68), dict(os=20), dict(groups=513), dict(K=1 << 21, xs=1 << 21), dict(N=1 << 21, os=1 << 21),
               dict(rows=(1 << 24) + 1), dict(rows=1 << 24, N=1 << 20, os=1 << 20), dict(sets=65537),
               dict(K=1 << 20, xs=1 << 20, N=1 << 20, os=1 << 20)):
        assert _grouped(**kw) == binding.UNSUPPORTED, kw
    assert _grouped(rows=0, x=NULL, out=NULL) == binding.OK and _grouped(groups=0, begin=NULL, end=NULL) == binding.OK


def test_mxfp4_grouped_matmul():
    def call(x=FAKE, xs=FAKE, w=FAKE, ws=FAKE, K=128, rows=4):
        return binding.load().regione_mxfp4_grouped_matmul(x, xs, w, ws, NULL, FAKE, FAKE, rows, 1, 1, K, 16, 0, FAKE, 16, NULL, NULL)
    for kw in (dict(x=NULL), dict(xs=NULL), dict(w=NULL), dict(ws=NULL), dict(xs=ODD), dict(ws=ODD), dict(x=ODD)):
        assert call(**kw) == binding.INVALID_ARG, kw
    assert call(K=64) == binding.UNSUPPORTED and call(K=160) == binding.UNSUPPORTED
    assert call(rows=0) == binding.OK


def test_mxfp4_rows():
    lib = binding.load()
    q = lambda x=FAKE, B=1, src=4, cap=4, K=64, c=FAKE, s=FAKE, idx=NULL: lib.regione_mxfp4_quantize(x, idx, NULL, B, src, cap, K, c, s, NULL, NULL)
    for kw in (dict(x=NULL), dict(c=NULL), dict(s=NULL), dict(x=ODD), dict(c=ODD), dict(B=-1), dict(cap=-1), dict(K=0), dict(src=-1), dict(src=3)):
        assert q(**kw) == binding.INVALID_ARG, kw
    assert q(K=48) == binding.UNSUPPORTED and q(cap=1 << 31, src=1 << 31) == binding.UNSUPPORTED
    assert q(cap=0) == binding.OK and q(B=0, x=NULL) == binding.OK
    d = lambda c=FAKE, s=FAKE, x=FAKE, B=1, cap=4, K=64: lib.regione_mxfp4_dequantize(c, s, NULL, B, cap, K, x, NULL, NULL)
    assert d(c=NULL) == d(s=NULL) == d(x=NULL) == d(x=ODD) == d(B=-1) == binding.INVALID_ARG
    assert d(K=16) == binding.UNSUPPORTED and d(cap=0) == binding.OK


def test_mxfp4_cache():
    lib = binding.load()
    st = lambda k=FAKE, keep=FAKE, n=FAKE, B=1, N=8, cap=8, H=3, D=64, q=FAKE: lib.regione_rikv_store_mxfp4(
        k, FAKE, keep, n, B, N, cap, H, D, q, FAKE, FAKE, FAKE, NULL, NULL)
    for kw in (dict(k=NULL), dict(keep=NULL), dict(n=NULL), dict(q=ODD), dict(B=-1), dict(N=-1), dict(cap=-1), dict(H=0)):
        assert st(**kw) == binding.INVALID_ARG, kw
    assert st(D=96) == binding.UNSUPPORTED and st(cap=0) == binding.OK and st(B=0) == binding.OK
    ld = lambda D=64, n=FAKE, cap=8: lib.regione_rikv_load_mxfp4(FAKE, FAKE, FAKE, FAKE, n, 1, cap, 3, D, FAKE, FAKE, NULL, NULL)
    assert ld(D=32) == binding.UNSUPPORTED and ld(n=NULL) == binding.INVALID_ARG and ld(cap=0) == binding.OK
