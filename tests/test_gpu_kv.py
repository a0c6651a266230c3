"""Attention over a paged 8-bit cache (f3dc_kv_append_fp8, f3dc_kv_attention_fp8) against a plain
64-bit evaluation: every size where a page, a chunk or a tile ends, empty rows and sequences, NaN
wherever nothing may be read, strides, streams, graphs, and the two together as a serving loop."""
import math

import pytest
import torch

import kv_ref as R
from paper_2511_22533_gb300 import f3dc

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN = float("nan")


def cache_of(c):
    return f3dc.KVCache(c.k, c.v, c.ks, c.vs)


def batch_of(c, max_rows=None, max_length=None, **kw):
    return f3dc.KVBatch(c.row_start, c.length, c.table, rows=c.n_rows, max_rows=max(c.rows + [0]) if max_rows is None else max_rows,
                        max_length=max(c.lengths + [0]) if max_length is None else max_length, **kw)


def attend(c, q, causal, scale=None, workspace=True, out=None, lse=True, cache=None, batch=None, **kw):
    cache, batch = cache or cache_of(c), batch or batch_of(c)
    scale = scale or 1.0 / math.sqrt(c.dh)
    if out is None:
        out = torch.full((c.n_rows, c.heads * c.dh), 7.0, dtype=torch.bfloat16, device=DEV)
    if lse is True:
        lse = torch.full((c.n_rows, c.heads), 7.0, device=DEV)
    n = f3dc.kv_attention_workspace(cache, batch, c.heads) if workspace else 0
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) if n else None
    f3dc.kv_attention_fp8(cache, batch, q, q.stride(0), out, out.stride(0), c.heads, scale, causal=causal, lse=lse, workspace=ws, **kw)
    return out, lse


def queries(c, part=40, scale=1.0):
    return c.randn(c.n_rows, c.heads * c.dh, part=part, scale=scale).to(torch.bfloat16)


def run_attend(c, causal, q=None, **kw):
    q = queries(c) if q is None else q
    out, lse = attend(c, q, causal, **kw)
    assert f3dc.gemm_status() == 0
    R.check_attend(c, out, lse, q, 1.0 / math.sqrt(c.dh), causal, stay=7.0)
    return out, lse


# ------------------------------------------------------------------ attention

FEW = [
    # held tokens, rows, heads, key heads, dh, page
    ([0], [1], 1, 1, 64, 16), ([1], [1], 16, 16, 64, 64), ([30], [1], 4, 4, 32, 16), ([31], [1], 4, 2, 128, 32),
    ([126], [1], 8, 1, 64, 128), ([127, 128, 129], [1, 1, 1], 6, 2, 64, 64), ([1000, 0, 5], [1, 1, 1], 12, 4, 128, 16),
    ([517], [5], 3, 1, 128, 32), ([63], [16], 2, 2, 32, 32), ([64], [17], 1, 1, 64, 16), ([99], [31], 4, 4, 32, 64),
    ([4097], [2], 8, 8, 64, 128), ([2500, 777], [3, 0], 10, 2, 128, 64), ([2047], [1], 40, 2, 128, 16),
    ([333, 40, 0, 12], [7, 1, 3, 9], 5, 1, 64, 32)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("held,rows,heads,kv_heads,dh,page", FEW)
def test_attention_of_few_rows(held, rows, heads, kv_heads, dh, page, causal):
    c = R.Case(held, rows, heads, kv_heads, dh, page, seed=len(held) + dh, spare_rows=2, before=1)
    c.fill()
    run_attend(c, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("held,rows,heads,kv_heads,dh,page", [
    ([0], [64], 1, 1, 64, 64), ([0], [128], 1, 1, 128, 16), ([5], [129], 2, 2, 64, 32), ([1], [257], 1, 1, 32, 128),
    ([200], [300], 6, 2, 64, 64), ([77, 0, 300], [130, 64, 255], 4, 4, 128, 32), ([700], [85], 3, 1, 32, 16),
    ([128], [511], 8, 2, 128, 128), ([0, 1300], [1, 400], 5, 1, 64, 16), ([1374], [333], 2, 2, 64, 64)])
def test_attention_of_many_rows(held, rows, heads, kv_heads, dh, page, causal):
    c = R.Case(held, rows, heads, kv_heads, dh, page, seed=len(held) + dh + 7, spare_rows=3, before=2)
    c.fill()
    run_attend(c, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("held,rows,heads,kv_heads,page", [
    ([300, 0, 33], [4, 3, 4], 8, 1, 16), ([5000], [32], 2, 2, 64), ([40, 700], [17, 2], 3, 3, 32), ([0], [33], 1, 1, 16),
    ([129, 2000, 64, 0], [8, 8, 0, 7], 8, 2, 128), ([90], [25], 1, 1, 64)])
def test_attention_of_some_rows(held, rows, heads, kv_heads, dh, page, causal):
    # 17 to 33 packed rows, as one part and as several; values and keys of NaN that some rows see
    c = R.Case(held, rows, heads, kv_heads, dh, page, seed=len(held) + dh + 31, spare_rows=2, before=1)
    c.fill()
    run_attend(c, causal)
    run_attend(c, causal, workspace=False)
    for b, n in enumerate(c.rows):
        if n > 2:
            at = c.lengths[b] - 1
            c.v[c.table_list[b][at // page], kv_heads - 1, at % page, 3] = R.STALE
            c.k[c.table_list[b][(at - 1) // page], 0, (at - 1) % page, dh - 1] = R.STALE
    run_attend(c, causal)
    run_attend(c, causal, q=queries(c, scale=6.0), workspace=False)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("rows,heads,dh,page", [(1537, 40, 64, 64), (1700, 40, 64, 16), (2048, 38, 32, 128), (1920, 40, 32, 32)])
def test_attention_of_many_rows_for_every_sm(rows, heads, dh, page, causal):
    # launches that fill the GPU with larger blocks of rows, the last of one row to a whole one; NaN beside them
    c = R.Case([70], [rows], heads, heads, dh, page, seed=rows)
    c.fill(spread=1.0, v_spread=2.0)
    last = 70 + rows - 1
    c.v[c.table_list[0][last // page], 3, last % page, 5] = R.STALE
    c.v[c.table_list[0][(last - 600) // page], 7, (last - 600) % page, dh - 2] = R.STALE
    c.k[c.table_list[0][(last - 300) // page], 11, (last - 300) % page, 0] = R.STALE
    run_attend(c, causal)
    if not causal:
        run_attend(c, False, q=queries(c, scale=4.0))


def cross(lengths, rows, heads, kv_heads, dh, page, **kw):
    """Queries over caches that do not hold their rows (shorter than them, too)."""
    c = R.Case(lengths, [0] * len(lengths), heads, kv_heads, dh, page, **kw)
    c.rows, c.starts = list(rows), [sum(rows[:b]) for b in range(len(rows) + 1)]
    c.n_rows = c.starts[-1]
    c.row_start = torch.tensor(c.starts, dtype=torch.int32, device=DEV)
    return c


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("lengths,rows", [([0], [3]), ([0, 5, 0], [1, 9, 40]), ([2], [300]), ([130, 0, 1], [200, 150, 129])])
def test_rows_that_see_no_token(lengths, rows, dh, causal):
    # empty caches, and causal rows ahead of the first token
    c = cross(lengths, rows, 4, 2, dh, 16)
    c.fill()
    out, lse = run_attend(c, causal)
    if causal:
        b = len(rows) - 1
        blind = max(0, rows[b] - lengths[b])
        assert torch.all(out[c.starts[b]:c.starts[b] + blind] == 0) and torch.all(torch.isinf(lse[c.starts[b]:c.starts[b] + blind]))


@pytest.mark.parametrize("rows", [4, 200])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_scales_from_page_to_page(dh, rows):
    # scales over many powers of two, and pages of zeros
    c = R.Case([900, 300], [rows, rows], 4, 2, dh, 16, seed=dh)
    c.fill(spread=1.5, v_spread=12.0)
    for j in (0, 5, 11):
        c.v[c.table_list[0][j]], c.vs[c.table_list[0][j]] = 0, 0
    c.k[c.table_list[1][2]], c.ks[c.table_list[1][2]] = 0, 0
    run_attend(c, True)
    run_attend(c, False)


@pytest.mark.parametrize("rows", [4, 200])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_scores_far_apart(dh, rows):
    # the largest scores late, early and in the middle, weights over the whole range
    c = R.Case([1500], [rows], 2, 1, dh, 32, seed=dh + 1)
    c.fill(spread=0.0)
    for j, e in ((3, 3), (20, 5), (40, 6), (len(c.table_list[0]) - 1, 4)):
        c.ks[c.table_list[0][j]] += e
    run_attend(c, False, q=queries(c, scale=3.0))
    run_attend(c, True, q=queries(c, scale=3.0))


@pytest.mark.parametrize("rows", [1, 150])
def test_a_token_that_takes_nearly_all(rows):
    # the first token's score far above thousands of others', its values zero: what the others give is left, each
    # 2^-14 of it or so, and with a second such token at the end the first's reference is no more
    c = R.Case([6000], [rows], 2, 1, 64, 64, seed=30)
    c.fill(spread=0.0, v_spread=0.0)
    q = torch.ones((c.n_rows, 128), dtype=torch.bfloat16, device=DEV)
    p0, p1 = c.table_list[0][0], c.table_list[0][len(c.table_list[0]) // 2]
    for t in c.table_list[0]:
        c.k[t] = torch.zeros_like(c.k[t])
    c.k[p0, 0, 0], c.v[p0, 0, 0] = 0x40, 0         # 2.0 in every element of the key
    c.ks[:] = 127                                  # score 16: 2^23 times the weights of the others
    run_attend(c, True, q=q)
    c.k[p1, 0, 5] = 0x48                           # 4.0: score 32
    run_attend(c, False, q=q)


@pytest.mark.parametrize("rows", [3, 150])
def test_queries_of_all_sizes(rows):
    # bf16 queries from 2^-100 to 2^60 against keys that bring their scores back, zeros among them
    c = R.Case([200], [rows], 2, 1, 64, 64, seed=3)
    c.fill(spread=0.0)
    q = queries(c).view(c.n_rows, 2, 64)
    q[0] = 0.0
    for e in (-100, 60):
        c.ks[:] = 127 - 6 - e - 3
        run_attend(c, True, q=(q * 2.0 ** e).view(c.n_rows, -1))
    q[1, 0, ::2] *= 2.0 ** -30
    c.ks[:] = 121
    run_attend(c, True, q=q.reshape(c.n_rows, -1))


@pytest.mark.parametrize("rows", [1, 6, 140])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_nan_in_the_cache(dh, rows):
    # what a row does not see counts for nothing; a NaN value shows in its element alone, a NaN key or scale in all
    c = R.Case([150, 150], [rows, rows], 4, 2, dh, 16, seed=dh)
    c.fill()

    def put(b, token, head, which, e):
        (c.v if which == "v" else c.k)[c.table_list[b][token // 16], head, token % 16, e] = R.STALE

    last = 150 + rows - 1
    put(0, last, 0, "v", 3)            # seen by the last row alone
    put(0, last - rows // 2, 1, "v", dh - 1)
    put(0, last, 1, "k", 0)
    put(1, 40, 0, "v", 7)              # seen by every row
    c.vs[c.table_list[1][-1], 1] = 255
    run_attend(c, True)
    run_attend(c, False)


def test_nan_queries_stay_in_their_rows():
    for rows in (5, 200):
        c = R.Case([90], [rows], 2, 1, 64, 64, seed=4)
        c.fill()
        q = queries(c)
        q[1, 5], q[2, 64 + 9] = NAN, NAN
        run_attend(c, True, q=q)


@pytest.mark.parametrize("rows", [2, 190])
def test_attention_strides(rows):
    # queries and outputs among other columns, keys and values of a page in one pool
    c = R.Case([100, 17], [rows, 1], 4, 2, 64, 32, joint=True, seed=5)
    c.fill()
    wide, q = torch.full((c.n_rows, 1024), NAN, dtype=torch.bfloat16, device=DEV), queries(c)
    wide[:, 512:768] = q
    big = torch.full((c.n_rows, 600), 7.0, dtype=torch.bfloat16, device=DEV)
    out, lse = attend(c, wide[:, 512:768], True, out=big[:, 24:280])
    R.check_attend(c, out.contiguous(), lse, q, 0.125, True)
    assert torch.all(big[:, :24] == 7) and torch.all(big[:, 280:] == 7)
    without, none = attend(c, wide[:, 512:768], True, lse=None)
    assert none is None and torch.equal(without, out)


@pytest.mark.parametrize("rows", [1, 20, 150])
def test_with_and_without_workspace(rows):
    c = R.Case([5000, 100], [rows, rows], 4, 2, 64, 64, seed=6)
    c.fill()
    run_attend(c, True)
    run_attend(c, True, workspace=False)
    # a part of what would be used
    cache, batch, q = cache_of(c), batch_of(c), queries(c)
    n = f3dc.kv_attention_workspace(cache, batch, 4)
    out = torch.full((c.n_rows, 256), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((c.n_rows, 4), device=DEV)
    ws = torch.zeros(max(16, n // 2 + 5), dtype=torch.uint8, device=DEV)
    f3dc.kv_attention_fp8(cache, batch, q, 256, out, 256, 4, 0.125, causal=True, lse=lse, workspace=ws)
    R.check_attend(c, out, lse, q, 0.125, True)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("held,rows,heads,kv_heads,page", [
    ([1500], [1], 16, 16, 64), ([700, 2500, 0, 31], [1, 5, 8, 2], 4, 4, 16), ([3000] * 4, [2, 0, 1, 2], 32, 16, 32), ([2600], [11], 2, 1, 128),
    ([30000, 1], [1, 1], 3, 3, 64)])
def test_sums_joined_in_a_cluster(held, rows, heads, kv_heads, dh, page):
    # shares of a sequence that need no workspace, some of no tokens; NaN in one share alone
    c = R.Case(held, rows, heads, kv_heads, dh, page, seed=dh + 41, spare_rows=1, before=1)
    c.fill()
    one, _ = run_attend(c, True, workspace=False)
    two, _ = run_attend(c, True, workspace=False)
    assert torch.equal(one, two)
    c.v[c.table_list[0][3], 0, 7, dh - 1] = R.STALE
    c.k[c.table_list[0][5], kv_heads - 1, 2, 0] = R.STALE
    run_attend(c, True, workspace=False)
    run_attend(c, False)


@pytest.mark.parametrize("rows", [1, 130])
def test_same_call_same_bits(rows):
    c = R.Case([3000, 500, 77], [rows] * 3, 8, 2, 128, 16, seed=8)
    c.fill()
    q = queries(c)
    first, lse = attend(c, q, True)
    for _ in range(3):
        again, l2 = attend(c, q, True)
        assert torch.equal(first, again) and torch.equal(lse, l2)


@pytest.mark.parametrize("rows", [1, 135])
def test_offsets_past_32_bits(rows):
    # a pool of more than 4 GiB whose pages lie far apart
    page, dh, stride = 16, 64, 3 << 28
    pool = torch.empty(7 * stride + 2 * page * dh, dtype=torch.uint8, device=DEV)
    c = R.Case([85], [rows], 2, 2, dh, page, seed=9, spare_pages=0) if rows == 1 else R.Case([0], [rows - 32], 2, 2, dh, page, seed=9,
                                                                                          spare_pages=0)
    c.fill()
    assert c.pages <= 7
    k, v = (pool.as_strided((c.pages, 2, page, dh), (stride, page * dh, dh, 1), o) for o in (0, stride // 2))
    k.copy_(c.k), v.copy_(c.v)
    q = queries(c)
    out, lse = attend(c, q, True, cache=f3dc.KVCache(k, v, c.ks, c.vs))
    R.check_attend(c, out, lse, q, 0.125, True)
    del pool


def test_sequences_may_share_pages():
    # a common prefix, and the same sequence twice
    c = R.Case([640, 640, 640], [1, 4, 4], 4, 1, 64, 64, seed=10)
    for b in (1, 2):
        c.table_list[b][:10] = c.table_list[0][:10]
    c.table_list[2] = list(c.table_list[1])
    for b in range(3):
        c.table[b, :11] = torch.tensor(c.table_list[b], dtype=torch.int32, device=DEV)
    c.fill()
    out, _ = run_attend(c, True)


def test_many_sequences():
    n = 700
    held, rows = [(37 * b) % 210 for b in range(n)], [b % 3 for b in range(n)]
    c = R.Case(held, rows, 2, 1, 32, 16, seed=11)
    c.fill()
    run_attend(c, True)


def test_bad_sequences_are_left_out():
    # what the device finds wrong is reported, and the other sequences are answered
    def fresh():
        c = R.Case([100, 200, 50], [2, 2, 2], 4, 2, 64, 16, seed=12)
        c.fill()
        return c

    def check(c, broken, zeros=False):
        q = queries(c)
        out, lse = attend(c, q, True, batch=batch_of(c, max_rows=2, max_length=202))
        assert f3dc.gemm_status() == 2 and f3dc.gemm_status() == 0
        good = fresh()
        ref, _, err, _ = R.attend(good, q, 0.125, True)
        for b in range(3):
            at = slice(2 * b, 2 * b + 2)
            if b != broken:
                assert torch.all((out.double().view(6, 4, 64)[at] - ref[at]).abs() <= err[at] + 2.0 ** -8 * (ref[at].abs() + err[at]))
            elif not zeros:
                assert torch.all(out[at] == 7.0) and torch.all(lse[at] == 7.0)

    c = fresh()
    c.length[1] = 203               # longer than the bound
    check(c, 1)
    c.length[1] = -1
    check(c, 1)
    c.length[1] = 202
    c.table[1, 3] = c.pages         # a page outside the pool: zeros
    check(c, 1, zeros=True)
    c.table[1, 3] = -1
    check(c, 1, zeros=True)
    c = fresh()
    c.row_start[3] = 7              # more rows than there are
    check(c, 2)
    c.row_start[3] = 3              # and fewer than none
    check(c, 2)


# ------------------------------------------------------------------ append

def rows_of(c, part, heads):
    return c.randn(c.n_rows, heads * c.dh, part=part) * torch.exp2(c.randn(c.n_rows, 1, part=part + 1, scale=2.0))


def run_append(c, dims=0, interleaved=False, axes=1, positions=None, with_q=True, k=None, v=None, base=10000.0, spread=0.3, **kw):
    kv = torch.cat([rows_of(c, 50, c.kv_heads), rows_of(c, 52, c.kv_heads)], 1).to(torch.bfloat16)
    W = c.kv_heads * c.dh
    k = kv[:, :W] if k is None else k
    v = kv[:, W:] if v is None else v
    q = rows_of(c, 54, c.heads).to(torch.bfloat16) if with_q and dims else None
    q_out = torch.full_like(q, 7.0) if q is not None else None
    c.fill(c.held, spread=spread, v_spread=spread)
    before = [t.clone() for t in (c.k, c.ks, c.v, c.vs)]
    rot = None
    if dims:
        per = dims // 2 // axes
        freq = [base ** (-(j % per) / per) if j < per * axes else 0.0 for j in range(dims // 2)]
        rot = f3dc.Rotary(dims, freq, interleaved=interleaved, axes=axes)
    f3dc.kv_append_fp8(cache_of(c), batch_of(c), k, k.stride(0), v, v.stride(0), q=q, ldq=q.stride(0) if dims and with_q else 0, q_out=q_out,
                       ldqo=q_out.stride(0) if q_out is not None else 0, heads=c.heads if q is not None else 0, rotary=rot,
                       positions=positions, **kw)
    assert f3dc.gemm_status() == 0
    k64, v64 = (x.double().reshape(c.n_rows, c.kv_heads, c.dh) for x in (k, v))
    k_err = torch.zeros_like(k64)
    if dims:
        place = torch.zeros((c.n_rows, dims // 2), dtype=torch.float64, device=DEV)
        for b in range(c.batch):
            at = slice(c.starts[b], c.starts[b + 1])
            place[at] = torch.arange(c.held[b], c.lengths[b], device=DEV).double()[:, None]
        angle = place * torch.tensor(freq, dtype=torch.float64, device=DEV)
        if positions is not None:
            at = positions.tolist()
            angle = R.angles([[row[min(j // per, axes - 1)] for j in range(dims // 2)] for row in at], freq).to(DEV)
        k_err = R.rotate_err(k64, dims, interleaved)
        k64 = R.rotate(k64, angle, dims, interleaved)
        if q is not None:
            q64 = q.double().view(c.n_rows, c.heads, c.dh)
            err = R.rotate_err(q64, dims, interleaved)
            ref = R.rotate(q64, angle, dims, interleaved)
            got = q_out.double().view(c.n_rows, c.heads, c.dh)
            mine = slice(c.starts[0], c.starts[-1])
            bound = R.U_BF16 * (ref.abs() + err) + err
            assert torch.all((got - ref).abs()[mine] <= bound[mine])
            out = torch.ones(c.n_rows, dtype=torch.bool, device=DEV)
            out[mine] = False
            assert torch.all(q_out[out] == 7.0)
    R.check_append(c, "k", k64, k_err, before[0], before[1])
    R.check_append(c, "v", v64, torch.zeros_like(v64), before[2], before[3])
    return q_out


APPEND = [
    ([0], [1], 1, 1, 64, 64), ([5], [1], 16, 16, 64, 16), ([16], [1], 8, 2, 128, 16), ([31, 32, 33], [1, 1, 1], 4, 2, 32, 32),
    ([0], [16], 2, 1, 64, 16), ([0], [17], 2, 2, 32, 16), ([15], [34], 6, 3, 128, 16), ([100, 0, 7], [0, 129, 64], 5, 5, 64, 64),
    ([127], [258], 12, 4, 128, 128), ([3], [500], 1, 1, 32, 128), ([1, 2, 3, 4], [33, 1, 95, 2], 16, 8, 64, 32), ([64], [128], 40, 20, 128, 128)]


@pytest.mark.parametrize("dims,interleaved", [(0, False), ("all", False), ("half", True)])
@pytest.mark.parametrize("held,rows,heads,kv_heads,dh,page", APPEND)
def test_append(held, rows, heads, kv_heads, dh, page, dims, interleaved):
    c = R.Case(held, rows, heads, kv_heads, dh, page, seed=dh + page, spare_rows=2, before=1)
    run_append(c, dims={"all": dh, "half": dh // 2}.get(dims, 0), interleaved=interleaved)


@pytest.mark.parametrize("held,rows,heads,kv_heads,dh,page", [
    ([0, 100], [0, 9000], 3, 3, 64, 32), ([20] * 70, [i % 7 for i in range(70)], 16, 16, 64, 16), ([1000, 5], [4100, 70], 8, 2, 128, 128)])
def test_append_many_pages(held, rows, heads, kv_heads, dh, page):
    # more pages than CTAs fit the GPU, sequences without rows
    run_append(R.Case(held, rows, heads, kv_heads, dh, page, seed=dh + page, spare_rows=2, before=1), dims=dh)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axes,dims", [(1, 64), (2, 64), (3, 64), (3, 16), (2, 48)])
def test_append_positions(axes, dims, interleaved):
    # given positions, some negative and far; pairs that are left over stay
    c = R.Case([10, 0], [40, 9], 4, 2, 64, 32, seed=axes)
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (c.n_rows, axes), generator=c.gen(60), device=DEV).to(torch.int32)
    pos[::2] %= 64
    run_append(c, dims=dims, interleaved=interleaved, axes=axes, positions=pos)


def test_append_far_positions():
    # tokens two million places in: the angle's whole turns are dropped exactly
    c = R.Case([30], [3], 2, 1, 64, 16, seed=2)
    for base in (10000.0, 5e5):
        pos = torch.tensor([[2 ** 21 + 1], [2 ** 31 - 1], [1999999]], dtype=torch.int32, device=DEV)
        run_append(c, dims=64, positions=pos, base=base)


def test_append_in_place_and_strides():
    # keys, values and queries of one wide matrix, queries rotated in place; a joint pool
    c = R.Case([21, 3], [50, 4], 6, 2, 64, 16, joint=True, seed=13)
    wide = torch.cat([rows_of(c, 50 + 2 * i, n) for i, n in enumerate((6, 2, 2))], 1).to(torch.bfloat16)
    k, v, keep = wide[:, 384:512], wide[:, 512:], wide.clone()
    run_append(c, dims=32, with_q=False, k=k, v=v)
    want = torch.empty((c.n_rows, 384), dtype=torch.bfloat16, device=DEV)
    rot, cache, batch = f3dc.Rotary(32), cache_of(c), batch_of(c)
    f3dc.kv_append_fp8(cache, batch, k, 640, v, 640, q=wide, ldq=640, q_out=want, ldqo=384, heads=6, rotary=rot)
    assert torch.equal(wide, keep)
    f3dc.kv_append_fp8(cache, batch, k, 640, v, 640, q=wide, ldq=640, q_out=wide, ldqo=640, heads=6, rotary=rot)
    assert torch.equal(wide[:, :384], want) and torch.equal(wide[:, 384:], keep[:, 384:])


def test_append_larger_scales_round_the_page_anew():
    # new tokens up to 2^40 larger than those there, and far smaller ones
    for up in (1, 3, 9, 20, 40, -30):
        c = R.Case([20, 40], [3, 30], 2, 2, 64, 64, seed=up + 50)
        v = (rows_of(c, 52, 2) * 2.0 ** up).to(torch.bfloat16)
        run_append(c, v=v, k=(rows_of(c, 56, 2) * 2.0 ** -up).to(torch.bfloat16))


def test_append_range_ends_and_non_finite():
    c = R.Case([5, 0, 16], [6, 40, 1], 2, 2, 32, 16, seed=14)
    v = rows_of(c, 52, 2)
    v[0, 3], v[1, 4], v[2, 40] = NAN, math.inf, -math.inf
    v[7:23] = 0.0
    v[25] = torch.finfo(torch.bfloat16).max
    v[40] = 2.0 ** -130
    v[46] = NAN
    run_append(c, v=v.to(torch.bfloat16), spread=0.0)


def test_append_into_a_page_whose_scale_is_nan():
    c = R.Case([5], [2], 1, 1, 32, 16, seed=15)
    c.fill(c.held)
    p = c.table_list[0][0]
    c.vs[p] = 255
    x = rows_of(c, 50, 1).to(torch.bfloat16)
    f3dc.kv_append_fp8(cache_of(c), batch_of(c), x, 32, x, 32)
    assert c.vs[p].item() == 255 and c.ks[p].item() != 255 and f3dc.gemm_status() == 0


def test_append_starts_a_page_anew():
    # a page used before: nothing of its scale or bytes counts
    c = R.Case([32], [16], 2, 1, 64, 16, seed=16)
    c.fill(c.lengths)
    c.ks[:], c.vs[:] = 255, 200
    c.ks[c.table_list[0][0]], c.ks[c.table_list[0][1]] = 121, 121
    x = rows_of(c, 50, 1).to(torch.bfloat16)
    f3dc.kv_append_fp8(cache_of(c), batch_of(c), x, 64, x, 64)
    p = c.table_list[0][2]
    assert c.ks[p].item() == c.vs[p].item() < 200
    assert torch.equal(c.k[p], c.v[p])


def test_append_bad_sequences_are_left_out():
    c = R.Case([20, 5, 9], [2, 2, 2], 2, 1, 64, 16, seed=17)
    c.fill(c.held)
    x = rows_of(c, 50, 1).to(torch.bfloat16)
    before = [t.clone() for t in (c.k, c.ks)]
    batch = batch_of(c, max_rows=2, max_length=100)

    def run(changed):
        f3dc.kv_append_fp8(cache_of(c), batch, x, 64, x, 64)
        assert f3dc.gemm_status() == 2
        for b in range(3):
            p = c.table_list[b][c.held[b] // 16]
            assert torch.equal(c.k[p], before[0][p]) == (b not in changed)
        c.k.copy_(before[0]), c.ks.copy_(before[1])

    c.length[1] = 1                 # shorter than its rows
    run((0, 2))
    c.length[1] = 101
    run((0, 2))
    c.length[1] = 7
    c.table[0, 1] = c.pages
    run((1, 2))
    c.table[0, 1] = c.table_list[0][1]
    c.row_start[3] = 9
    run((0, 1))


def test_append_offsets_past_32_bits():
    page, dh, stride = 16, 32, 3 << 29
    c = R.Case([30], [5], 1, 1, dh, page, seed=18, spare_pages=0)
    c.fill(c.held)
    pool = torch.zeros(2 * stride + page * dh + stride // 2, dtype=torch.uint8, device=DEV)
    k, v = (pool.as_strided((c.pages, 1, page, dh), (stride, page * dh, dh, 1), o) for o in (0, stride // 2))
    k.copy_(c.k), v.copy_(c.v)
    x = rows_of(c, 50, 1).to(torch.bfloat16)
    ks, vs = c.ks.clone(), c.vs.clone()
    f3dc.kv_append_fp8(f3dc.KVCache(k, v, ks, vs), batch_of(c), x, dh, x, dh)
    f3dc.kv_append_fp8(cache_of(c), batch_of(c), x, dh, x, dh)
    assert torch.equal(k, c.k) and torch.equal(v, c.v) and torch.equal(ks, c.ks)


# ------------------------------------------------------------------ together

def dense(q, k, v, scale, n):
    """Causal attention of the last n rows over dense fp64 keys and values [tokens, heads, dh]."""
    L = k.shape[0]
    g = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    x = torch.einsum("nhd,lhd->hnl", q, k) * scale
    x = torch.where(torch.arange(L, device=DEV) <= torch.arange(n, device=DEV)[:, None] + (L - n), x, -math.inf)
    return torch.einsum("hnl,lhd->nhd", torch.softmax(x, 2), v)


@pytest.mark.parametrize("dh,page,heads,kv_heads", [(64, 16, 4, 4), (128, 64, 8, 2), (32, 32, 3, 1)])
def test_a_serving_loop(dh, page, heads, kv_heads):
    # two prompts come in chunks, then tokens one at a time in a captured graph that follows the lengths
    # on the device; against dense attention over the unrounded keys and values
    g = torch.Generator(device=DEV).manual_seed(dh)
    B, total, chunks = 2, [150, 97], [[70, 1], [50, 66]]
    W = kv_heads * dh
    qkv = torch.randn((B, 200, heads * dh + 2 * W), generator=g, device=DEV).to(torch.bfloat16)
    width = 200 // page + 1
    table = torch.randperm(B * width, generator=g, device=DEV).to(torch.int32).view(B, width)
    shape = (B * width, kv_heads, page, dh)
    k8, v8 = (torch.full(shape, R.STALE, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.full(shape[:2], 255, dtype=torch.uint8, device=DEV) for _ in range(2))
    cache, rot = f3dc.KVCache(k8, v8, ks, vs), f3dc.Rotary(dh)
    lengths = torch.zeros(B, dtype=torch.int32, device=DEV)
    freq = torch.tensor([10000.0 ** (-j / (dh // 2)) for j in range(dh // 2)], dtype=torch.float64, device=DEV)
    angle = torch.arange(200, device=DEV).double()[:, None] * freq
    q64, k64, v64 = [], [], []
    for b in range(B):
        x = qkv[b].double()
        q64.append(R.rotate(x[:, :heads * dh].reshape(200, heads, dh), angle, dh, False))
        k64.append(R.rotate(x[:, heads * dh:heads * dh + W].reshape(200, kv_heads, dh), angle, dh, False))
        v64.append(x[:, heads * dh + W:].reshape(200, kv_heads, dh))

    def step(batch, rows, out, ws):
        qk, ld = rows, rows.stride(0)
        f3dc.kv_append_fp8(cache, batch, qk[:, heads * dh:], ld, qk[:, heads * dh + W:], ld, q=qk, ldq=ld, q_out=qk, ldqo=ld, heads=heads,
                           rotary=rot)
        f3dc.kv_attention_fp8(cache, batch, qk, ld, out, heads * dh, heads, 1 / math.sqrt(dh), causal=True, workspace=ws)

    def check(b, lo, hi, got):
        # e4m3 keys: 2^-4 relative, scores off by about 2^-4 |q| |k| / sqrt(dh) of random signs: what is looked for
        # is a token, a page or a rotation gone wrong, which costs the whole norm
        ref = dense(q64[b][lo:hi], k64[b][:hi], v64[b][:hi], 1 / math.sqrt(dh), hi - lo)
        assert (got.double().view(hi - lo, heads, dh) - ref).norm() <= 0.15 * ref.norm()

    done = [0, 0]
    for chunk in chunks:
        starts = torch.tensor([0, chunk[0], sum(chunk)], dtype=torch.int32, device=DEV)
        rows = torch.cat([qkv[b, done[b]:done[b] + chunk[b]] for b in range(B)])
        lengths += torch.tensor(chunk, dtype=torch.int32, device=DEV)
        batch = f3dc.KVBatch(starts, lengths, table, rows=sum(chunk), max_rows=max(chunk), max_length=200)
        ws = torch.empty(max(16, f3dc.kv_attention_workspace(cache, batch, heads)), dtype=torch.uint8, device=DEV)
        out = torch.empty((sum(chunk), heads * dh), dtype=torch.bfloat16, device=DEV)
        step(batch, rows, out, ws)
        for b in range(B):
            check(b, done[b], done[b] + chunk[b], out[starts[b]:starts[b + 1]])
            done[b] += chunk[b]
    starts = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    batch = f3dc.KVBatch(starts, lengths, table, rows=B, max_rows=1, max_length=200)
    ws = torch.empty(max(16, f3dc.kv_attention_workspace(cache, batch, heads)), dtype=torch.uint8, device=DEV)
    rows, out = torch.zeros((B, qkv.shape[2]), dtype=torch.bfloat16, device=DEV), torch.empty((B, heads * dh), dtype=torch.bfloat16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(batch, rows, out, ws)
    for _ in range(40):
        rows.copy_(torch.stack([qkv[b, done[b]] for b in range(B)]))
        lengths += 1
        graph.replay()
        for b in range(B):
            check(b, done[b], done[b] + 1, out[b:b + 1])
            done[b] += 1
    assert f3dc.gemm_status() == 0


@pytest.mark.parametrize("rows", [1, 140])
def test_streams_and_graphs(rows):
    # the same work on two streams at once, each with a workspace of its own, and captured twice
    cases = [R.Case([3000 + 64 * i], [rows], 4, 2, 64, 64, seed=20 + i) for i in range(2)]
    want, keep = [], []
    for c in cases:
        c.fill()
        q = queries(c)
        want.append(attend(c, q, True))
        cache, batch = cache_of(c), batch_of(c)
        n = f3dc.kv_attention_workspace(cache, batch, 4)
        keep.append((c, q, cache, batch, torch.empty(max(16, n), dtype=torch.uint8, device=DEV),
                     torch.empty((c.n_rows, 256), dtype=torch.bfloat16, device=DEV), torch.empty((c.n_rows, 4), device=DEV)))

    def call(i, stream=None):
        c, q, cache, batch, ws, out, lse = keep[i]
        f3dc.kv_attention_fp8(cache, batch, q, 256, out, 256, 4, 0.125, causal=True, lse=lse, workspace=ws, stream=stream)

    def same():
        for (_, _, _, _, _, out, lse), (o, l) in zip(keep, want):
            assert torch.equal(out, o) and torch.equal(lse, l)
            out.zero_(), lse.zero_()

    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, s in enumerate(streams):
            call(i, s.cuda_stream)
    torch.cuda.synchronize()
    same()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            call(i)
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    same()


@pytest.mark.parametrize("call", ["append", "few", "many"])
def test_first_call_in_a_capture(call):
    # a process whose first call of the library is captured, and replayed
    import os
    import subprocess
    import sys
    code = f"""
import sys
sys.path.insert(0, {os.path.dirname(os.path.abspath(__file__))!r})
sys.path.insert(0, {os.path.dirname(os.path.dirname(os.path.abspath(__file__)))!r})
import torch, kv_ref as R
from paper_2511_22533_gb300 import f3dc
c = R.Case([100], [{1 if call == "few" else 140}], 2, 1, 64, 64, seed=3)
c.fill(c.held if {call == "append"} else None)
q = c.randn(c.n_rows, 128, part=40).to(torch.bfloat16)
cache, batch = f3dc.KVCache(c.k, c.v, c.ks, c.vs), f3dc.KVBatch(c.row_start, c.length, c.table, c.n_rows, max(c.rows), max(c.lengths))
before = [t.clone() for t in (c.v, c.vs)]
out, lse = torch.zeros_like(q), torch.zeros((c.n_rows, 2), device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    if {call == "append"}:
        f3dc.kv_append_fp8(cache, batch, q, 128, q[:, 64:], 128)
    else:
        f3dc.kv_attention_fp8(cache, batch, q, 128, out, 128, 2, 0.125, causal=True, lse=lse)
g.replay()
torch.cuda.synchronize()
assert f3dc.gemm_status() == 0
if {call == "append"}:
    new = q[:, 64:].double().view(-1, 1, 64)
    R.check_append(c, "v", new, torch.zeros_like(new), *before)
else:
    R.check_attend(c, out, lse, q, 0.125, True)
print("fine")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]


def test_append_on_streams_and_in_graphs():
    # two appends at once on two streams, and captured and replayed: the same pages as one after the other
    cases = [R.Case([40, 7], [3, 60], 4, 2, 64, 32, seed=40 + i) for i in range(2)]
    rot, want, args = f3dc.Rotary(64), [], []
    for c in cases:
        c.fill(c.held)
        x, q = c.randn(c.n_rows, 256, part=50).to(torch.bfloat16), queries(c)
        start = [t.clone() for t in (c.k, c.v, c.ks, c.vs)]
        out = torch.zeros_like(q)
        args.append((c, cache_of(c), batch_of(c), x, q, out, start))
    torch.cuda.synchronize()

    def call(i, stream=None):
        c, cache, batch, x, q, out, _ = args[i]
        f3dc.kv_append_fp8(cache, batch, x, 256, x[:, 128:], 256, q=q, ldq=256, q_out=out, ldqo=256, heads=4, rotary=rot, stream=stream)

    def state(i):
        c, _, _, _, _, out, _ = args[i]
        return [t.clone() for t in (c.k, c.v, c.ks, c.vs, out)]

    def reset():
        for c, _, _, _, _, out, start in args:
            for t, b in zip((c.k, c.v, c.ks, c.vs), start):
                t.copy_(b)
            out.zero_()
        torch.cuda.synchronize()

    for i in range(2):
        call(i)
        want.append(state(i))
    reset()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, s in enumerate(streams):
        call(i, s.cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(state(i), want[i]))
    reset()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            call(i)
    reset()
    for g, s in zip(graphs, streams):
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(state(i), want[i]))
    assert f3dc.gemm_status() == 0


# exponents of the value scales of a sequence's pages, as shares of its length: far apart, pages of zeros (-127) among them
FAR = [(-127, 74), (90, -127, 90), (-20, 113, -60), (0, -127, 100, 5, 113, -64), (113,), (-127, 6, -64, 7)]


@pytest.mark.parametrize("rows,held", [(1, [1500]), (1, [9000, 40]), (4, [700, 300]), (20, [1300]), (150, [900, 100]), (150, [6000])])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_value_scales_far_apart(dh, rows, held):
    # every token counts in the sum of weights, however small its values are beside others'.  The reference's bounds take
    # value scales of 2^64 at most: the three roundings of the affine step, the reference and the shift (kv_ref.attend) are of
    # numbers larger by up to 2 * (113 - 64) here, 3 U32 98 = 294 2^-24 = 2^-15.8 in a score: twice that in a weight and its sum
    # is 2^-14.8 of the sum of magnitudes, of which err holds 2^-11.
    for spread in FAR:
        c = R.Case(held, [rows] * len(held), 4, 2, dh, 16, seed=dh + rows)
        c.fill(spread=0.0)
        for pages in c.table_list:
            for j, p in enumerate(pages):
                e = spread[min(j * len(spread) // len(pages), len(spread) - 1)]
                c.vs[p] = e + 127
                if e == -127:
                    c.v[p] = 0
        for causal in (False, True):
            for workspace in (True, False):
                q = queries(c)
                out, lse = attend(c, q, causal, workspace=workspace)
                assert f3dc.gemm_status() == 0
                ref, ref_lse, err, lse_err = R.attend(c, q, 1.0 / math.sqrt(dh), causal)
                err, lse_err = err * (1 + 2.0 ** -3.8), lse_err + 2.0 ** -15.8
                got = out.double().view(ref.shape)
                bound = err + R.U_BF16 * (ref.abs() + err) + 2.0 ** -133
                assert torch.all((got - ref).abs() <= bound), f"{spread} {causal} {workspace}"
                assert torch.all((lse.double() - ref_lse).abs() <= lse_err), f"{spread} {causal} {workspace}"


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("rows,held", [(2, 3000), (2, 40000), (150, 3000)])
def test_sequences_beside_broken_ones(rows, held, workspace):
    # a bound that is broken in the middle leaves out the two sequences that share it and no other, in one part or in many
    for broken in (10 ** 6, 4 * rows + 1, -5):
        c = R.Case([held, 300, held, 2500, 17], [rows] * 5, 2, 1, 64, 64, seed=rows, spare_rows=1, before=1)
        c.fill()
        q = queries(c)
        c.row_start[2] = broken
        out, lse = attend(c, q, True, workspace=workspace, batch=batch_of(c, max_rows=rows))
        assert f3dc.gemm_status() == 2
        ref, ref_lse, err, lse_err = R.attend(c, q, 0.125, True)
        got = out.double().view(ref.shape)
        for b in range(5):
            at = slice(c.starts[b], c.starts[b + 1])
            if b in (1, 2):
                assert torch.all(out[at] == 7.0) and torch.all(lse[at] == 7.0)
            else:
                assert torch.all((got[at] - ref[at]).abs() <= err[at] + R.U_BF16 * (ref[at].abs() + err[at]) + 2.0 ** -133)
                assert torch.all((lse[at].double() - ref_lse[at]).abs() <= lse_err[at])
        assert torch.all(out[0] == 7.0) and torch.all(out[-1] == 7.0)


def test_workspace_of_calls_that_are_too_large():
    # nothing for what the attention itself refuses: more rows and heads than it counts, and bounds whose products leave 64 bits
    pool = torch.zeros((1, 1, 64, 64), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((1, 1), dtype=torch.uint8, device=DEV)
    cache, zeros = f3dc.KVCache(pool, pool, scales, scales), torch.zeros(2, dtype=torch.int32, device=DEV)
    for heads, kw in ((32, dict(rows=1 << 27, max_rows=1, max_length=1 << 20)), (65536, dict(rows=1 << 20, max_rows=1, max_length=1 << 20)),
                      (1, dict(rows=1, max_rows=1, max_length=2 ** 31 - 1)), (65536, dict(rows=2 ** 31 - 1, max_rows=1 << 30, max_length=1 << 20))):
        batch = f3dc.KVBatch(zeros, zeros[:1], zeros[None], **kw)
        assert f3dc.kv_attention_workspace(cache, batch, heads) == 0
        batch.batch = 1 << 26
        assert f3dc.kv_attention_workspace(cache, batch, heads) == 0


@pytest.mark.parametrize("held,rows", [([0], [1]), ([100, 0, 7], [5, 70, 0])])
@pytest.mark.parametrize("page", [16, 128])
def test_loose_bounds(held, rows, page):
    # bounds far above what the sequences have: as with close ones
    top = dict(max_rows=2 ** 31 - 1, max_length=2 ** 31 - 1025)
    cases = [R.Case(held, rows, 4, 2, 64, page, seed=page) for _ in range(2)]
    x = rows_of(cases[0], 50, 2).to(torch.bfloat16)
    for c, kw in zip(cases, ({}, top)):
        c.fill(c.held)
        f3dc.kv_append_fp8(cache_of(c), batch_of(c, **kw), x, 128, x, 128)
    assert all(torch.equal(getattr(cases[0], n), getattr(cases[1], n)) for n in ("k", "v", "ks", "vs"))
    c = cases[1]
    run_attend(c, True, batch=batch_of(c, **top))
    run_attend(c, False, batch=batch_of(c, **top), workspace=False)


@pytest.mark.parametrize("rows", [2, 150])
def test_page_tables_that_are_views(rows):
    # columns among others of a wider table: what does not fit them is out of bounds, though the wider table goes on
    for side in ("left", "right"):
        c = R.Case([300, 500, 60], [rows] * 3, 4, 2, 64, 64, seed=rows)
        c.fill()
        q = queries(c)
        width = -(-(300 + rows) // 64)
        wide = torch.zeros((3, width + 4), dtype=torch.int32, device=DEV)
        view = wide[:, :width] if side == "left" else wide[:, 4:]
        view[:, :width] = c.table[:, :width]
        cache, kw = cache_of(c), dict(rows=c.n_rows, max_rows=rows, max_length=max(c.lengths))
        for workspace in (True, False):
            out, lse = attend(c, q, True, cache=cache, batch=f3dc.KVBatch(c.row_start, c.length, view, **kw), workspace=workspace)
            assert f3dc.gemm_status() == 2
            ref, _, err, _ = R.attend(c, q, 0.125, True)
            got = out.double().view(ref.shape)
            for b in (0, 2):
                at = slice(c.starts[b], c.starts[b + 1])
                assert torch.all((got[at] - ref[at]).abs() <= err[at] + R.U_BF16 * (ref[at].abs() + err[at]) + 2.0 ** -133)
            at = slice(c.starts[1], c.starts[2])
            assert torch.all(out[at] == 7.0) and torch.all(lse[at] == 7.0)
        before = [t.clone() for t in (c.k, c.ks)]
        f3dc.kv_append_fp8(cache, f3dc.KVBatch(c.row_start, c.length, view, **kw), q, 256, q, 256)
        assert f3dc.gemm_status() == 2
        for p in c.table_list[1]:
            assert torch.equal(c.k[p], before[0][p]) and torch.equal(c.ks[p], before[1][p])
        assert not torch.equal(c.k[c.table_list[0][-1]], before[0][c.table_list[0][-1]])


def test_sequences_without_pages():
    # a page table of no columns: no sequence has a token, and every row sees none
    for rows in (1, 200):
        c = cross([0, 0], [rows, rows], 4, 2, 64, 16)
        out, lse = attend(c, queries(c), False, batch=f3dc.KVBatch(c.row_start, c.length, c.table[:, :0].contiguous(), rows=c.n_rows, max_rows=rows,
                                                                   max_length=0))
        assert f3dc.gemm_status() == 0 and torch.all(out == 0) and torch.all(lse == -math.inf)


@pytest.mark.parametrize("page", [16, 32])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("rows,held", [(60, 4500), (200, 8800)])
def test_many_small_pages_in_one_part(rows, held, dh, page):
    # one CTA walks through the ring of page-table entries twice and more, the last group not whole, every page with scales of
    # its own; one tile of queries and two
    c = R.Case([held], [rows], 2, 1, dh, page, seed=held + dh + page)
    c.fill(v_spread=3.0)
    run_attend(c, True, workspace=False)
    run_attend(c, False, workspace=False)


@pytest.mark.parametrize("rows", [1, 20, 150])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_nan_beside_value_scales_far_apart(dh, rows):
    # NaN values, keys and scales where the sums take their own exponentials: in their elements and rows alone
    for page in (16, 64):
        c = R.Case([700, 300], [rows, rows], 4, 2, dh, page, seed=dh + rows + page)
        c.fill(spread=0.0)
        for pages in c.table_list:
            for j, p in enumerate(pages):
                c.vs[p] = 127 + (90, -40, 0)[j % 3]
        last = 700 + rows - 1
        c.v[c.table_list[0][last // page], 0, last % page, 3] = R.STALE
        c.v[c.table_list[0][2], 1, 7, dh - 1] = R.STALE
        c.k[c.table_list[0][last // page], 1, last % page, 0] = R.STALE
        c.ks[c.table_list[1][1], 0] = 255
        c.vs[c.table_list[1][3], 1] = 255
        for causal in (False, True):
            q = queries(c)
            if rows > 1:
                q[1, 2] = NAN
            out, lse = attend(c, q, causal)
            assert f3dc.gemm_status() == 0
            ref, ref_lse, err, lse_err = R.attend(c, q, 1.0 / math.sqrt(dh), causal)
            got = out.double().view(ref.shape)
            assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(torch.isnan(lse), torch.isnan(ref_lse))
            # (bounds as in test_value_scales_far_apart)
            err, lse_err = err * (1 + 2.0 ** -3.8), lse_err + 2.0 ** -15.8
            fine = (got - ref).abs() <= err + R.U_BF16 * (ref.abs() + err) + 2.0 ** -133
            assert torch.all(fine | torch.isnan(ref)) and torch.all(((lse.double() - ref_lse).abs() <= lse_err) | torch.isnan(ref_lse))
