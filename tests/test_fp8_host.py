"""8-bit linear layers: every argument error is reported before anything touches
a GPU (the calls run here without one), and the C structure has the layout that the
binding declares."""
import ctypes as C

import pytest

from paper_2511_22533_gb300 import f3dc

P = 1 << 20  # an aligned address that no call may use


@pytest.fixture(scope="module")
def L():
    return f3dc.lib()


def quantize(L, **kw):
    a = dict(x=P, x_type=0, ldx=256, q=P, ldq=256, scales=P, lds=4, rows=3, cols=200)
    a.update(kw)
    return L.f3dc_quantize_fp8(*a.values(), None)


@pytest.mark.parametrize("kw,needle", [
    (dict(x=None), b"null"), (dict(q=None), b"null"), (dict(scales=None), b"null"), (dict(x_type=2), b"x_type"),
    (dict(rows=-1), b"rows"), (dict(cols=0), b"cols"), (dict(ldx=199), b"leading"), (dict(ldq=199), b"leading"),
    (dict(lds=1), b"leading"), (dict(x=P + 1), b"aligned"), (dict(x=P + 2, x_type=1), b"aligned")])
def test_quantize_refusals(L, kw, needle):
    assert quantize(L, **kw) == 1
    assert needle in L.f3dc_last_error(None)


GEMM = dict(A=P, lda=1024, sa=P, ldas=8, B=P, ldb=1024, sb=P, ldbs=8, bias=P, gate=None, out=P, ldo=512, out_scales=None,
            ldos=0, M=5, N=512, K=1000, epi=0)


@pytest.mark.parametrize("kw,needle", [
    (dict(A=None), b"null"), (dict(sa=None), b"null"), (dict(B=None), b"null"), (dict(sb=None), b"null"),
    (dict(out=None), b"null"), (dict(M=-1), b"M"), (dict(N=0), b"N"), (dict(N=12, ldo=16), b"N"), (dict(K=0), b"K"),
    (dict(epi=3), b"epilogue"), (dict(epi=-1), b"epilogue"), (dict(lda=992), b"lda"), (dict(lda=1001), b"lda"),
    (dict(ldb=1000), b"ldb"), (dict(ldas=7), b"ldas"), (dict(ldas=4), b"ldas"), (dict(ldbs=10), b"ldbs"),
    (dict(ldo=504), b"ldo"), (dict(ldo=516), b"ldo"), (dict(gate=P), b"gate"),
    (dict(epi=2, gate=P + 8), b"aligned"), (dict(bias=P + 2), b"aligned"), (dict(A=P + 8), b"aligned"),
    (dict(out=P + 4), b"aligned"), (dict(sb=P + 2), b"aligned"), (dict(epi=2, out_scales=P, ldos=4), b"8-bit"),
    (dict(out_scales=P, ldos=3), b"ldos"), (dict(out_scales=P, ldos=4, N=504, ldo=512), b"multiple of 16"),
    (dict(out_scales=P, ldos=4, ldo=520), b"ldo"), (dict(M=2 ** 31 - 1), b"large"),
    (dict(N=2 ** 31 - 8, ldo=2 ** 31), b"large"), (dict(K=2 ** 26 + 1, lda=2 ** 27, ldb=2 ** 27, ldas=2 ** 20, ldbs=2 ** 20), b"large")])
def test_gemm_refusals(L, kw, needle):
    a = dict(GEMM)
    a.update(kw)
    assert L.f3dc_gemm_fp8(*a.values(), None) == 1
    assert needle in L.f3dc_last_error(None)


NORM = dict(x=P, ldx=256, x_out=P, ldxo=256, y=P, ldy=256, gate=P, scale=P, shift=P, ldmod=256, group=None, groups=1, h=P,
            ldh=256, hs=None, ldhs=0, rows=3)


@pytest.mark.parametrize("kw,needle", [
    (dict(x=None), b"null"), (dict(x_out=None, h=None), b"null"), (dict(h=None, hs=P, ldhs=4), b"h_scales"),
    (dict(y=None), b"gate"), (dict(rows=-1), b"rows"), (dict(groups=0), b"groups"), (dict(ldx=255), b"rows of x"),
    (dict(ldxo=250), b"rows of x"), (dict(ldy=260), b"rows of x"), (dict(ldh=252), b"ldh"), (dict(ldmod=128), b"ldmod"),
    (dict(ldmod=258), b"ldmod"), (dict(hs=P, ldhs=1), b"ldhs"), (dict(x=P + 4), b"aligned"), (dict(h=P + 8), b"aligned"),
    (dict(x_out=P, ldxo=260), b"in place"), (dict(scale=P + 4), b"aligned"), (dict(group=P + 2), b"group_of_row")])
def test_norm_refusals(L, kw, needle):
    a = dict(NORM)
    a.update(kw)
    layer = f3dc.NormLayer(256)
    assert L.f3dc_norm_residual(C.byref(layer), *a.values(), None) == 1
    assert needle in L.f3dc_last_error(None)


@pytest.mark.parametrize("field,value,needle", [
    ("width", 0, b"width"), ("width", 252, b"width"), ("width", 8200, b"width"), ("post", 3, b"kind"), ("pre", -1, b"kind"),
    ("eps", -1.0, b"eps"), ("eps", float("nan"), b"eps"), ("pre_g", P + 2, b"aligned")])
def test_norm_layer_refusals(L, field, value, needle):
    layer = f3dc.NormLayer(256)
    setattr(layer, field, value)
    assert L.f3dc_norm_residual(C.byref(layer), *NORM.values(), None) == 1
    assert needle in L.f3dc_last_error(None)
    assert L.f3dc_norm_residual(None, *NORM.values(), None) == 1


def test_no_rows_is_no_work(L):
    # nothing is launched, so no GPU is needed
    assert quantize(L, rows=0) == 0
    a = dict(GEMM, M=0)
    assert L.f3dc_gemm_fp8(*a.values(), None) == 0
    layer = f3dc.NormLayer(256)
    a = dict(NORM, rows=0)
    assert L.f3dc_norm_residual(C.byref(layer), *a.values(), None) == 0


def test_norm_layer_layout():
    assert [getattr(f3dc.NormLayer, n).offset for n, _ in f3dc.NormLayer._fields_] == [0, 4, 8, 12, 16, 24, 32, 40, 48]
    assert C.sizeof(f3dc.NormLayer) == 56
