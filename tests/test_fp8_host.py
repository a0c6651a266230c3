"""8-bit linear layers: every argument error is reported before anything touches
a GPU (the calls run here without one), and the C structure has the layout that the
binding declares."""
import ctypes as C

import pytest
import torch

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


# Element types: the calls take pointers, so a tensor of another type would be read as what it
# is not, and an output of narrower elements written past its end.  Tensors that say they are on
# a GPU and calls that only record stand in for both.

class Tensor:
    def __init__(self, dtype, is_cuda=True, width=256):
        self.dtype, self.is_cuda, self.shape, self.device = dtype, is_cuda, (width,), "cuda:0" if is_cuda else "cpu"

    def data_ptr(self):
        return P

    def get_device(self):
        return 0

    def numel(self):
        return self.shape[0]

    def is_contiguous(self):
        return True


@pytest.fixture
def made(monkeypatch):
    """The calls that reach the library."""
    made = []
    calls = tuple(lambda *a, n=n: made.append((n, a)) or 0 for n in ("quantize", "gemm", "norm"))
    monkeypatch.setattr(f3dc, "_fp8_state", (calls, f3dc._fp8_args(), None))
    return made


BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64
U8, E4M3, E8M0, E5M2, I32, I64 = torch.uint8, torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.float8_e5m2, torch.int32, torch.int64


def py_quantize(x=BF16, q=U8, scales=U8):
    f3dc.quantize_fp8(Tensor(x), 256, Tensor(q), 256, Tensor(scales), 4, 3, 200, stream=0)


def py_gemm(A=U8, sa=U8, B=U8, sb=U8, bias=BF16, gate=None, out=BF16, out_scales=None, epi=0):
    t = [None if d is None else Tensor(d) for d in (A, sa, B, sb, bias, gate, out, out_scales)]
    f3dc.gemm_fp8(t[0], 1024, t[1], 8, t[2], 1024, t[3], 8, t[4], t[5], t[6], 512, t[7], 4, 5, 512, 1000, epi, stream=0)


def py_norm(x=F32, x_out=F32, y=BF16, gate=F32, scale=F32, shift=F32, group=I32, h=BF16, hs=None):
    t = [None if d is None else Tensor(d) for d in (x, x_out, y, gate, scale, shift, group, h, hs)]
    f3dc.norm_residual(f3dc.NormLayer(256), t[0], 256, t[1], 256, t[2], 256, t[3], t[4], t[5], 256, t[6], 1, t[7], 256, t[8], 4, 3,
                       stream=0)


def each(call, base, wrong):
    return [(call, dict(base, **{k: d})) for k, ds in wrong.items() for d in ds]


RESID, OUT8 = dict(epi=2, gate=F32, out=F32), dict(out=U8, out_scales=U8)


@pytest.mark.parametrize("call,kw", [
    *each(py_quantize, {}, dict(x=[F16, F64, U8, I32], q=[BF16, F32, E5M2], scales=[F32, BF16, E4M3])),
    *each(py_gemm, {}, dict(A=[BF16, E5M2, F32], sa=[F32, I32], B=[F16, E5M2], sb=[F32, BF16], bias=[F32, F16], out=[F32, F16, U8])),
    *each(py_gemm, dict(epi=1), dict(bias=[F32], out=[F32, F16])),
    *each(py_gemm, RESID, dict(gate=[BF16, F16, F64], out=[BF16, F16, F64], bias=[F32])),
    *each(py_gemm, OUT8, dict(out=[BF16, F32, E5M2], out_scales=[F32, BF16])),
    *each(py_norm, {}, dict(x=[BF16, F16, F64], x_out=[BF16, F16, F64], y=[F32, F16], gate=[BF16, F16], scale=[BF16, F64], shift=[BF16],
                            group=[I64, F32], h=[F32, F16, U8])),
    *each(py_norm, dict(h=U8, hs=U8), dict(h=[BF16, E5M2], hs=[F32, I32]))])
def test_types_are_refused(made, call, kw):
    with pytest.raises(f3dc.F3dcError) as e:
        call(**kw)
    assert e.value.status == 1 and "need" in str(e.value) and not made


@pytest.mark.parametrize("call,kw", [
    (py_quantize, {}), (py_quantize, dict(x=F32, q=E4M3, scales=E8M0)), (py_quantize, dict(x=torch.int16)), (py_quantize, dict(x=torch.uint16)),
    (py_gemm, {}), (py_gemm, dict(A=E4M3, sa=E8M0, B=torch.int8, sb=torch.int8, bias=None, out=torch.int16)), (py_gemm, RESID),
    (py_gemm, OUT8), (py_gemm, dict(out=E4M3, out_scales=E8M0, epi=1)), (py_norm, {}), (py_norm, dict(h=E4M3, hs=E8M0, group=None)),
    (py_norm, dict(x_out=None, y=None, gate=None, scale=None, shift=None))])
def test_types_that_fit_reach_the_library(made, call, kw):
    call(**kw)
    assert len(made) == 1
    if call is py_quantize:
        assert made[0][1][1] == (1 if kw.get("x") is F32 else 0)


@pytest.mark.parametrize("dtype", [F16, F32, U8, torch.uint32])
def test_norm_layer_refuses_vectors_of_other_types(dtype):
    for name in ("post_g", "post_b", "pre_g", "pre_b"):
        with pytest.raises(f3dc.F3dcError) as e:
            f3dc.NormLayer(256, **{name: Tensor(dtype)})
        assert e.value.status == 1
    f3dc.NormLayer(256, post_g=Tensor(BF16), pre_b=Tensor(torch.int16))


def test_tensors_off_the_gpu_are_refused(made):
    with pytest.raises(f3dc.F3dcError) as e:
        f3dc.quantize_fp8(Tensor(BF16, is_cuda=False), 256, Tensor(U8), 256, Tensor(U8), 4, 3, 200, stream=0)
    assert e.value.status == 1 and "device" in str(e.value) and not made
