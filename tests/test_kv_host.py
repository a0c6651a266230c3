"""Attention over a paged 8-bit cache: every argument error is reported before anything touches a GPU
(the calls run here without one), the C structures have the layout that the binding declares, and
rotation frequencies become exact fractions of a turn."""
import ctypes as C
import decimal
import math
import random

import numpy as np
import pytest
import torch

from paper_2511_22533_gb300 import f3dc

P = 1 << 20  # an aligned address that no call may use


@pytest.fixture(scope="module")
def L():
    return f3dc.lib()


def struct(cls, values):
    s = cls.__new__(cls)
    C.Structure.__init__(s, *values.values())
    return s


CACHE = dict(pages=10, page_tokens=64, kv_heads=4, dh=64, k=P, v=P, k_scales=P, v_scales=P, page_stride=64 * 64 * 4, scale_stride=4)
BATCH = dict(row_start=P, lengths=P, page_table=P, table_stride=5, batch=2, rows=7, max_rows=4, max_length=300)
ROTARY = dict(dims=64, interleaved=0, axes=1, turns=P)
APPEND = dict(k=P, ldk=256, v=P, ldv=256, q=P, ldq=512, q_out=P, ldqo=512, heads=8, positions=None)
ATTEND = dict(q=P, ldq=512, out=P, ldo=512, lse=P, heads=8, scale=0.125, causal=1, ws=P, ws_bytes=1 << 20)


def ref(cls, base, kw):
    return None if kw is None else C.byref(struct(cls, dict(base, **kw)))


def append(L, cache={}, batch={}, rotary={}, **kw):
    return L.f3dc_kv_append_fp8(ref(f3dc.KVCache, CACHE, cache), ref(f3dc.KVBatch, BATCH, batch), ref(f3dc.Rotary, ROTARY, rotary),
                                *dict(APPEND, **kw).values(), None)


def attend(L, cache={}, batch={}, **kw):
    return L.f3dc_kv_attention_fp8(ref(f3dc.KVCache, CACHE, cache), ref(f3dc.KVBatch, BATCH, batch), *dict(ATTEND, **kw).values(), None)


BOTH = [
    (dict(cache=None), b"null cache"), (dict(batch=None), b"null batch"), (dict(cache=dict(pages=0)), b"pages"),
    (dict(cache=dict(page_tokens=48)), b"page_tokens"), (dict(cache=dict(page_tokens=256)), b"page_tokens"),
    (dict(cache=dict(kv_heads=0)), b"kv_heads"), (dict(cache=dict(kv_heads=1025)), b"kv_heads"), (dict(cache=dict(dh=96)), b"dh"),
    (dict(cache=dict(page_stride=64 * 64 * 4 - 16)), b"page_stride"), (dict(cache=dict(page_stride=64 * 64 * 4 + 8)), b"page_stride"),
    (dict(cache=dict(scale_stride=3)), b"scale_stride"), (dict(cache=dict(page_stride=1 << 60)), b"too large"),
    (dict(cache=dict(k=None)), b"null pointer"), (dict(cache=dict(v_scales=None)), b"null pointer"), (dict(cache=dict(k=P + 8)), b"aligned"),
    (dict(batch=dict(batch=-1)), b"negative"), (dict(batch=dict(rows=-1)), b"negative"), (dict(batch=dict(max_rows=-1)), b"negative"),
    (dict(batch=dict(max_length=-1)), b"negative"), (dict(batch=dict(table_stride=-1)), b"table_stride"),
    (dict(batch=dict(table_stride=2 ** 31)), b"table_stride"), (dict(batch=dict(row_start=None)), b"null pointer"),
    (dict(batch=dict(lengths=None)), b"null pointer"), (dict(batch=dict(page_table=None)), b"null pointer"),
    (dict(batch=dict(lengths=P + 2)), b"aligned"), (dict(q=P + 8), b"aligned"), (dict(ldq=511), b"ldq"), (dict(ldq=504), b"ldq"),
    (dict(batch=dict(batch=2 ** 31 - 1, max_rows=2 ** 31 - 1)), b"too large")]


@pytest.mark.parametrize("kw,needle", BOTH + [
    (dict(k=None), b"null"), (dict(v=None), b"null"), (dict(q_out=None), b"q_out"), (dict(ldk=252), b"ldk"), (dict(ldk=248), b"ldk"),
    (dict(ldv=260), b"ldv"), (dict(ldqo=500), b"ldq"), (dict(ldqo=520), b"in place"), (dict(heads=0), b"heads"), (dict(heads=65537), b"heads"),
    (dict(rotary=None), b"rotary"), (dict(rotary=dict(dims=0)), b"dims"), (dict(rotary=dict(dims=24)), b"dims"),
    (dict(rotary=dict(dims=80)), b"dims"), (dict(rotary=dict(interleaved=2)), b"interleaved"), (dict(rotary=dict(axes=0)), b"axes"),
    (dict(rotary=dict(axes=4)), b"axes"), (dict(rotary=dict(axes=2)), b"positions"), (dict(rotary=dict(turns=None)), b"turns"),
    (dict(rotary=dict(turns=P + 4)), b"turns"), (dict(positions=P + 1), b"positions"), (dict(rotary=None, q=None, positions=P), b"positions"),
    (dict(v=P + 2), b"aligned"), (dict(q_out=P + 2), b"aligned"), (dict(batch=dict(max_length=2 ** 31 - 1)), b"too large"),
    (dict(batch=dict(max_length=2 ** 31 - 1000)), b"too large")])
def test_append_refusals(L, kw, needle):
    assert append(L, **kw) == 1
    assert needle in L.f3dc_last_error(None)


@pytest.mark.parametrize("kw,needle", BOTH + [
    (dict(q=None), b"null"), (dict(out=None), b"null"), (dict(ldo=504), b"ldo"), (dict(ldo=514), b"ldo"), (dict(heads=0), b"heads"),
    (dict(heads=6), b"heads"), (dict(heads=65540), b"heads"), (dict(scale=0.0), b"scale"), (dict(scale=-1.0), b"scale"),
    (dict(scale=float("nan")), b"scale"), (dict(scale=float("inf")), b"scale"), (dict(causal=2), b"causal"), (dict(ws=P + 8), b"aligned"),
    (dict(lse=P + 2), b"lse"), (dict(out=P + 8), b"aligned"), (dict(batch=dict(max_length=2 ** 31 - 1)), b"too large")])
def test_attention_refusals(L, kw, needle):
    assert attend(L, **kw) == 1
    assert needle in L.f3dc_last_error(None)


def test_no_rows_is_no_work(L):
    # nothing is launched, so no GPU is needed
    for batch in (dict(batch=0), dict(rows=0), dict(max_rows=0)):
        assert append(L, batch=batch) == 0 and attend(L, batch=batch) == 0
        assert L.f3dc_kv_attention_workspace(ref(f3dc.KVCache, CACHE, {}), ref(f3dc.KVBatch, BATCH, batch), 8) == 0
    assert L.f3dc_kv_attention_workspace(None, None, 8) == 0


def test_layouts():
    assert [getattr(f3dc.KVCache, n).offset for n, _ in f3dc.KVCache._fields_] == [0, 4, 8, 12, 16, 24, 32, 40, 48, 56]
    assert [getattr(f3dc.KVBatch, n).offset for n, _ in f3dc.KVBatch._fields_] == [0, 8, 16, 24, 32, 36, 40, 44]
    assert [getattr(f3dc.Rotary, n).offset for n, _ in f3dc.Rotary._fields_] == [0, 4, 8, 16]
    assert (C.sizeof(f3dc.KVCache), C.sizeof(f3dc.KVBatch), C.sizeof(f3dc.Rotary)) == (64, 48, 24)


def test_turns_are_exact():
    # within one unit of 2^-64 turns of the frequency over 2 pi, of either sign and any size that matters
    rng = random.Random(5)
    freq = [1.0, 0.0, -1.0, 1e-30, -1e-30, 6.283185307179586, 123.456] + [10000.0 ** (-j / 32) for j in range(32)] + [
        rng.uniform(-20, 20) for _ in range(200)]
    with decimal.localcontext() as ctx:
        ctx.prec = 60
        tau = 2 * decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494")
        for f, t in zip(freq, f3dc.rotary_turns(freq)):
            off = (int(t) - decimal.Decimal(f) / tau * 2 ** 64) % 2 ** 64
            assert min(off, 2 ** 64 - off) <= 1
    for f in (math.nan, math.inf, -math.inf):
        with pytest.raises(f3dc.F3dcError):
            f3dc.rotary_turns([f])
    assert f3dc.rotary_turns([]).size == 0


def test_turns_of_large_frequencies():
    # exact to a unit of 2^-64 turns up to 2^40 radians, refused above
    rng = random.Random(6)
    freq = [s * f for f in [2.0 ** e for e in range(0, 41)] + [rng.uniform(1, 2) * 2.0 ** rng.randrange(40) for _ in range(500)] for s in (1, -1)]
    with decimal.localcontext() as ctx:
        ctx.prec = 80
        tau = 2 * decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798")
        for f, t in zip(freq, f3dc.rotary_turns(freq)):
            off = (int(t) - decimal.Decimal(f) / tau * 2 ** 64) % 2 ** 64
            assert min(off, 2 ** 64 - off) <= 1
    for f in (2.0 ** 40 * (1 + 2.0 ** -52), 1e13, -1e18, 1e300):
        with pytest.raises(f3dc.F3dcError) as e:
            f3dc.rotary_turns([1.0, f])
        assert e.value.status == 1


# Tensors that say they are on a GPU stand in for GPU tensors, and calls that only record.

class Tensor:
    def __init__(self, dtype, shape=(256,), stride=None, is_cuda=True, index=0):
        self.dtype, self.shape, self.is_cuda, self.index = dtype, tuple(shape), is_cuda, index
        self.device = f"cuda:{index}" if is_cuda else "cpu"
        self.strides = stride or tuple(int(np.prod(shape[i + 1:])) for i in range(len(shape)))

    def data_ptr(self):
        return P

    def get_device(self):
        return self.index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return int(np.prod(self.shape))

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def is_contiguous(self):
        return True


U8, E4M3, E8M0, I32, I64, BF16, F32 = (torch.uint8, torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.int32, torch.int64, torch.bfloat16,
                                       torch.float32)


def cache(k=U8, v=U8, ks=U8, vs=U8, shape=(10, 4, 64, 64), sshape=(10, 4), **kw):
    return f3dc.KVCache(kw.get("tk") or Tensor(k, shape), kw.get("tv") or Tensor(v, shape), Tensor(ks, sshape), kw.get("tvs") or Tensor(vs, sshape))


def batch(rs=I32, ln=I32, pt=I32, n=2, **kw):
    return f3dc.KVBatch(kw.get("trs") or Tensor(rs, (n + 1,)), kw.get("tln") or Tensor(ln, (n,)), kw.get("tpt") or Tensor(pt, (n, 5)), 7, 4, 300)


@pytest.mark.parametrize("make,kw", [
    (cache, dict(k=BF16)), (cache, dict(v=torch.float8_e5m2)), (cache, dict(ks=F32)), (cache, dict(vs=I32)), (cache, dict(shape=(10, 4, 64))),
    (cache, dict(sshape=(10, 5))), (cache, dict(tv=Tensor(U8, (10, 4, 32, 64)))), (cache, dict(tvs=Tensor(U8, (9, 4)))),
    (cache, dict(tk=Tensor(U8, (10, 4, 64, 64), (16384, 64, 256, 1)))), (cache, dict(tk=Tensor(U8, (10, 4, 64, 64), (32768, 4096, 64, 1)))),
    (cache, dict(tvs=Tensor(U8, (10, 4), (8, 2)))), (cache, dict(tv=Tensor(U8, (10, 4, 64, 64), is_cuda=False))),
    (cache, dict(tv=Tensor(U8, (10, 4, 64, 64), index=1))),
    (batch, dict(rs=I64)), (batch, dict(ln=F32)), (batch, dict(pt=I64)), (batch, dict(trs=Tensor(I32, (2,)))), (batch, dict(tpt=Tensor(I32, (3, 5)))),
    (batch, dict(tln=Tensor(I32, (2,), (2,)))), (batch, dict(tpt=Tensor(I32, (2, 5), (1, 5)))), (batch, dict(tpt=Tensor(I32, (2, 5), (0, 1)))),
    (batch, dict(tln=Tensor(I32, (2,), is_cuda=False)))])
def test_tensors_that_do_not_fit_are_refused(make, kw):
    with pytest.raises(f3dc.F3dcError) as e:
        make(**kw)
    assert e.value.status == 1


def test_views_of_larger_pools_fit():
    joint = (2 * 16384, 4096, 64, 1)
    c = f3dc.KVCache(*(Tensor(E4M3, (10, 4, 64, 64), joint) for _ in range(2)), *(Tensor(E8M0, (10, 4), (8, 1)) for _ in range(2)))
    assert (c.page_stride, c.scale_stride, c.pages, c.kv_heads, c.page_tokens, c.dh) == (32768, 8, 10, 4, 64, 64)
    assert batch(tpt=Tensor(I32, (2, 5), (9, 1))).table_stride == 9
    # dimensions of one may have any stride
    one = f3dc.KVCache(*(Tensor(U8, (1, 1, 64, 64), (7, 3, 64, 1)) for _ in range(2)), *(Tensor(U8, (1, 1), (5, 9)) for _ in range(2)))
    assert (one.page_stride, one.scale_stride) == (4096, 1)
    single = batch(n=1, trs=Tensor(I32, (2,)), tln=Tensor(I32, (1,), (3,)), tpt=Tensor(I32, (1, 1), (4, 8)))
    assert single.table_stride == 1


@pytest.fixture
def made(monkeypatch):
    """The calls that reach the library."""
    made = []
    calls = tuple(lambda *a, n=n: made.append((n, a)) or 0 for n in ("append", "attend"))
    monkeypatch.setattr(f3dc, "_kv_state", (calls, f3dc._kv_args(), None))
    return made


def py_append(k=BF16, v=BF16, q=None, q_out=None, positions=None):
    t = [None if d is None else Tensor(d, (7, 512)) for d in (k, v, q, q_out)]
    f3dc.kv_append_fp8(cache(), batch(), t[0], 256, t[1], 256, q=t[2], ldq=512, q_out=t[3], ldqo=512, heads=8,
                       positions=positions, stream=0)


def py_attend(q=BF16, out=BF16, lse=F32, ws=U8, lse_shape=(7, 8)):
    f3dc.kv_attention_fp8(cache(), batch(), Tensor(q, (7, 512)), 512, Tensor(out, (7, 512)), 512, 8, 0.125,
                          lse=None if lse is None else Tensor(lse, lse_shape), workspace=None if ws is None else Tensor(ws, (99,)), stream=0)


@pytest.mark.parametrize("call,kw", [
    (py_append, dict(k=F32)), (py_append, dict(v=torch.float16)), (py_append, dict(q=F32, q_out=BF16)), (py_append, dict(q=BF16, q_out=F32)),
    (py_append, dict(positions=Tensor(I64, (7, 1)))), (py_append, dict(positions=Tensor(I32, (6, 1)))), (py_attend, dict(q=F32)),
    (py_attend, dict(out=torch.float16)), (py_attend, dict(lse=BF16)), (py_attend, dict(ws=F32)), (py_attend, dict(lse_shape=(7, 7)))])
def test_wrong_tensors_do_not_reach_the_library(made, call, kw):
    with pytest.raises(f3dc.F3dcError) as e:
        call(**kw)
    assert e.value.status == 1 and not made


def test_calls_that_fit_reach_the_library(made):
    py_append()
    py_append(k=torch.int16, q=BF16, q_out=BF16, positions=Tensor(I32, (7, 1)))
    py_attend()
    py_attend(lse=None, ws=None)
    assert [n for n, _ in made] == ["append", "append", "attend", "attend"]
    assert made[2][1][-3:-1] == (P, 99) and made[3][1][-3:-1] == (None, 0)


def test_lengths_are_bounded_by_a_views_columns(made, monkeypatch):
    # to the library a row of a page table is as long as its stride: a narrower view bounds the lengths in every call
    t = [Tensor(BF16, (7, 512)) for _ in range(2)]

    class Library:
        @staticmethod
        def f3dc_kv_attention_workspace(*a):
            made.append(("workspace", a))
            return 5

    for view, tokens, want in ((Tensor(I32, (2, 4), (9, 1)), 64, 256), (Tensor(I32, (2, 5), (9, 1)), 64, 300), (Tensor(I32, (2, 4)), 64, 300),
                               (Tensor(I32, (2, 5), (9, 1)), 16, 80), (Tensor(I32, (2, 1), (2, 1)), 32, 32)):
        c, b = cache(shape=(10, 4, tokens, 64)), batch(tpt=view)
        f3dc.kv_append_fp8(c, b, t[0], 256, t[1], 256, stream=0)
        f3dc.kv_attention_fp8(c, b, t[0], 512, t[1], 512, 8, 0.125, stream=0)
        with monkeypatch.context() as m:
            m.setattr(f3dc, "lib", Library)
            assert f3dc.kv_attention_workspace(c, b, 8) == 5
        assert [n for n, _ in made] == ["append", "attend", "workspace"]
        for _, a in made:
            got = a[1].contents
            assert (got.max_length, got.table_stride, got.batch, got.rows, got.max_rows) == (want, view.strides[0], 2, 7, 4)
            assert (got.row_start, got.lengths, got.page_table) == (P, P, P)
        assert b.max_length == 300  # (a later call with another cache asks again)
        made.clear()


def test_a_page_table_without_columns():
    # as torch strides it; no sequence has a token then
    for n in (1, 2, 3):
        assert batch(n=n, trs=Tensor(I32, (n + 1,)), tln=Tensor(I32, (n,)), tpt=Tensor(I32, (n, 0), (1, 1))).table_stride == 0
