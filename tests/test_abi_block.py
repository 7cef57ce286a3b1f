"""Refusals of the layer norm, the rotary positions with several axes and the products with adapters, on the host (CPU only: fake
addresses, nothing may be launched)."""
import ctypes

import pytest

from paper_2510_25590_b200 import binding

FAKE, ODD, NULL = ctypes.c_void_p(4096), ctypes.c_void_p(4100), None
INVALID, UNSUPPORTED, OK, SMALL = binding.INVALID_ARG, binding.UNSUPPORTED, binding.OK, binding.WORKSPACE_TOO_SMALL


def _norm(x=FAKE, xs=64, r=NULL, rs=0, gate=NULL, w=FAKE, b=FAKE, ss=64, mod=0, eps=1e-6, begin=FAKE, end=FAKE, rows=4, groups=1, sets=1, C=64,
          xo=NULL, xos=0, out=FAKE, os=64):
    return binding.load().regione_layer_norm(x, xs, r, rs, gate, w, b, ss, mod, eps, begin, end, rows, groups, sets, C, xo, xos, out, os, NULL, NULL,
                                             NULL, NULL)


BOTH = dict(r=FAKE, rs=64, xo=FAKE, xos=64)


@pytest.mark.parametrize("kw", [dict(x=NULL), dict(x=ODD), dict(out=NULL), dict(out=ODD), dict(w=ODD), dict(b=ODD), dict(begin=NULL), dict(end=NULL),
                                dict(rows=-1), dict(groups=-1), dict(sets=0), dict(C=0), dict(xs=56), dict(os=56), dict(ss=56), dict(eps=-1.0),
                                dict(eps=float("nan")), dict(gate=FAKE), dict(xo=FAKE, xos=64), dict(r=FAKE, rs=64), dict(BOTH, r=ODD), dict(BOTH, xo=ODD),
                                dict(BOTH, gate=ODD), dict(BOTH, rs=56), dict(BOTH, xos=56)], ids=str)
def test_layer_norm_refuses(kw):
    assert _norm(**kw) == INVALID


@pytest.mark.parametrize("kw", [dict(C=60), dict(C=8200, xs=8200, os=8200, ss=8200), dict(xs=68), dict(os=68), dict(ss=68), dict(groups=513),
                                dict(sets=65536), dict(rows=(1 << 24) + 1), dict(xs=1 << 33), dict(BOTH, rs=68), dict(BOTH, xos=68)], ids=str)
def test_layer_norm_does_not_support(kw):
    assert _norm(**kw) == UNSUPPORTED


def test_layer_norm_of_nothing():
    assert _norm(rows=0, x=NULL, out=NULL) == OK and _norm(groups=0, begin=NULL, end=NULL) == OK


def _back(x=FAKE, xs=64, m=FAKE, s=FAKE, dy=FAKE, ys=64, dz=NULL, zs=0, r=NULL, rs=0, gate=NULL, w=FAKE, ss=64, begin=FAKE, end=FAKE, rows=4, groups=1,
          sets=1, C=64, dx=FAKE, ds=64, dr=NULL, qs=0, dw=FAKE, db=FAKE, dg=NULL, ws=FAKE, bytes=1 << 30):
    return binding.load().regione_layer_norm_backward(x, xs, m, s, dy, ys, dz, zs, r, rs, gate, w, ss, 0, begin, end, rows, groups, sets, C, dx, ds, dr, qs,
                                                      dw, db, dg, ws, bytes, NULL, NULL)


GATED = dict(r=FAKE, rs=64, gate=FAKE, dr=FAKE, qs=64, dg=FAKE)


@pytest.mark.parametrize("kw", [dict(x=NULL), dict(x=ODD), dict(m=NULL), dict(s=NULL), dict(dy=NULL), dict(dx=NULL), dict(dx=ODD), dict(dz=ODD, zs=64),
                                dict(dz=FAKE, zs=56), dict(w=ODD), dict(dw=ODD), dict(db=ODD), dict(ws=ODD), dict(xs=56), dict(ys=56), dict(ds=56),
                                dict(rows=-1), dict(sets=0), dict(dg=FAKE), dict(gate=FAKE), dict(r=FAKE, rs=64), dict(dr=FAKE, qs=64),
                                dict(GATED, gate=NULL), dict(GATED, dr=NULL), dict(GATED, r=ODD), dict(GATED, dr=ODD), dict(GATED, dg=ODD),
                                dict(GATED, rs=56), dict(GATED, qs=56)], ids=str)
def test_layer_norm_backward_refuses(kw):
    assert _back(**kw) == INVALID


def test_layer_norm_backward_workspace():
    lib = binding.load()
    need = lib.regione_layer_norm_backward_workspace
    assert _back(ws=NULL) == _back(bytes=need(4, 1, 64) - 1) == SMALL
    assert _back(C=60) == _back(groups=513) == _back(ys=68) == UNSUPPORTED
    assert need(-1, 1, 64) == need(4, -1, 64) == need(4, 1, 60) == need(4, 1, 8200) == need(4, 513, 64) == 0
    sizes = [need(rows, groups, 512) for rows, groups in ((1, 1), (9, 1), (9, 3), (5000, 3), (1 << 24, 512))]
    assert sizes == sorted(sizes) and sizes[0] > 0


def _rotary(q=FAKE, qb=512, qr=128, k=FAKE, kb=512, kr=128, idx=NULL, n=NULL, pos=FAKE, pb=12, B=2, places=4, cap=4, Hq=2, Hk=2, D=64, axes=3, compact=1,
            freq=None, axis=None, layout=0, inverse=0, norm=0, qw=NULL, kw=NULL, eps=1e-6, qo=FAKE, qob=512, qor=128, ko=FAKE, kob=512, kor=128):
    freq = (ctypes.c_double * 128)(*([0.5] * 128)) if freq is None else (ctypes.c_double * 128)(*(freq * 128)[:128])
    axis = (ctypes.c_int32 * 128)(*([2] * 128)) if axis is None else (ctypes.c_int32 * 128)(*(axis * 128)[:128])
    return binding.load().regione_rotary_axes(q, qb, qr, k, kb, kr, idx, n, pos, pb, B, places, cap, Hq, Hk, D, axes, compact, freq, axis, layout, inverse,
                                              norm, qw, kw, eps, qo, qob, qor, ko, kob, kor, NULL, NULL)


@pytest.mark.parametrize("kw", [dict(q=NULL), dict(q=ODD), dict(qo=NULL), dict(qo=ODD), dict(k=ODD), dict(ko=ODD), dict(k=NULL), dict(ko=NULL), dict(Hk=0),
                                dict(pos=NULL), dict(B=-1), dict(cap=-1), dict(places=-1), dict(Hq=0), dict(Hk=-1), dict(D=0), dict(axes=0),
                                dict(layout=2), dict(layout=-1), dict(axis=[3]), dict(axis=[-1]), dict(freq=[float("nan")]), dict(freq=[float("inf")]), dict(freq=[-1.1e7]),
                                dict(qr=120), dict(kr=120), dict(qor=120), dict(kor=120), dict(qb=-8), dict(pb=-1), dict(cap=5), dict(qob=0), dict(kob=0),
                                dict(qw=FAKE), dict(kw=FAKE), dict(norm=1, qw=ODD), dict(norm=1, kw=ODD), dict(norm=1, eps=-1.0),
                                dict(norm=1, eps=float("nan"))], ids=str)
def test_rotary_axes_refuses(kw):
    assert _rotary(**kw) == INVALID


@pytest.mark.parametrize("kw", [dict(D=72), dict(D=272, qr=544, kr=544, qor=544, kor=544), dict(axes=5), dict(qr=132), dict(qb=516), dict(kor=132), dict(kob=516),
                                dict(B=65536), dict(cap=(1 << 24) + 1, places=1 << 25), dict(B=16, cap=1 << 23, places=1 << 23), dict(inverse=1, norm=1), dict(Hq=65537, qr=1 << 23, qor=1 << 23)], ids=str)
def test_rotary_axes_does_not_support(kw):
    assert _rotary(**kw) == UNSUPPORTED


def test_rotary_axes_of_nothing():
    assert _rotary(B=0, q=NULL) == OK and _rotary(cap=0, q=NULL, pos=NULL) == OK


def _adapt(x=FAKE, xs=64, w=FAKE, bias=NULL, a=FAKE, b=FAKE, scale=NULL, which=FAKE, n=2, rank=8, begin=FAKE, end=FAKE, rows=4, groups=1, sets=1, K=64, N=16,
           act=0, out=FAKE, os=16, ws=FAKE, bytes=1 << 30):
    return binding.load().regione_adapter_matmul(x, xs, w, bias, a, b, scale, which, n, rank, begin, end, rows, groups, sets, K, N, act, out, os, ws, bytes,
                                                 NULL, NULL)


def test_adapter_matmul():
    for kw in (dict(x=NULL), dict(w=NULL), dict(a=NULL), dict(b=NULL), dict(which=NULL), dict(begin=NULL), dict(end=NULL), dict(out=NULL), dict(x=ODD),
               dict(w=ODD), dict(a=ODD), dict(b=ODD), dict(bias=ODD), dict(out=ODD), dict(ws=ODD), dict(rows=-1), dict(groups=-1), dict(sets=0), dict(n=0),
               dict(rank=0), dict(rank=-8), dict(K=0), dict(N=0), dict(act=2), dict(xs=56), dict(os=8)):
        assert _adapt(**kw) == INVALID, kw
    for kw in (dict(K=60), dict(N=12), dict(xs=68), dict(os=20), dict(rank=12), dict(rank=264), dict(n=65537), dict(groups=513), dict(rows=(1 << 24) + 1),
               dict(sets=65537)):
        assert _adapt(**kw) == UNSUPPORTED, kw
    assert _adapt(rows=0, x=NULL, out=NULL, ws=NULL) == OK and _adapt(groups=0, begin=NULL, end=NULL, which=NULL, ws=NULL) == OK


def test_adapter_matmul_workspace():
    need = binding.load().regione_adapter_matmul_workspace
    assert _adapt(ws=NULL) == _adapt(bytes=need(4, 1, 64, 16, 8) - 1) == SMALL
    assert need(-1, 1, 64, 16, 8) == need(4, -1, 64, 16, 8) == need(4, 1, 64, 0, 8) == need(4, 1, 64, 16, 0) == need(4, 1, 64, 16, 264) == 0
    # it never takes more to do less: the number of rows, which decides about the form, among it
    rows = [need(r, 4, 64, 512, 16) for r in (1, 8, 31, 33, 128, 129, 500, 100000)]
    assert rows == sorted(rows)
    groups = [need(500, g, 64, 512, 16) for g in (1, 4, 15, 16, 63, 512)]
    assert groups == sorted(groups)
