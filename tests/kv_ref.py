"""Plain 64-bit reference of attention over a paged 8-bit cache, sequence by sequence,
and the tolerances of its tests (test helper; shares no code with the library)."""
import decimal
import math

import torch

from fp8_ref import E4M3_MIN, TOP, U32, U_BF16, U_E4M3, pow2

STALE = 0x7F  # what unused places of a cache hold: NaN


class Case:
    """Sequences with `held` tokens in their pages and `rows` new ones, on shuffled pages of a pool
    whose every other byte is NaN."""

    def __init__(self, held, rows, heads, kv_heads, dh, page, seed=0, device="cuda", spare_rows=0, spare_pages=3, joint=False,
                 before=0):
        self.held, self.rows, self.heads, self.kv_heads, self.dh, self.page = list(held), list(rows), heads, kv_heads, dh, page
        self.batch = len(self.held)
        self.lengths = [h + n for h, n in zip(self.held, self.rows)]
        self.before = before  # rows of no sequence ahead of the first
        self.starts = [before + sum(self.rows[:b]) for b in range(self.batch + 1)]
        self.n_rows = self.starts[-1] + spare_rows
        self.device, self.seed = device, seed
        need = [-(-n // page) for n in self.lengths]
        self.pages = sum(need) + spare_pages
        order = torch.randperm(self.pages, generator=self.gen(1), device=device).tolist()
        self.table_list = [[order.pop() for _ in range(n)] for n in need]
        width = max([1] + need)
        self.table = torch.full((self.batch, width + 1), -7, dtype=torch.int32, device=device)  # (unused entries: no page)
        for b, pages in enumerate(self.table_list):
            if pages:
                self.table[b, :len(pages)] = torch.tensor(pages, dtype=torch.int32, device=device)
        self.row_start = torch.tensor(self.starts, dtype=torch.int32, device=device)
        self.length = torch.tensor(self.lengths, dtype=torch.int32, device=device)
        shape = (self.pages, kv_heads, page, dh)
        if joint:  # a page's keys and values side by side in one pool, scales likewise
            pool = torch.full((self.pages, 2, kv_heads, page, dh), STALE, dtype=torch.uint8, device=device)
            scales = torch.full((self.pages, 2, kv_heads), 0xFF, dtype=torch.uint8, device=device)
            self.k, self.v, self.ks, self.vs = pool[:, 0], pool[:, 1], scales[:, 0], scales[:, 1]
        else:
            self.k, self.v = (torch.full(shape, STALE, dtype=torch.uint8, device=device) for _ in range(2))
            self.ks, self.vs = (torch.full(shape[:2], 0xFF, dtype=torch.uint8, device=device) for _ in range(2))

    def gen(self, part):
        return torch.Generator(device=self.device).manual_seed(self.seed * 64 + part)

    def randn(self, *shape, part, scale=1.0):
        return torch.randn(shape, generator=self.gen(part), device=self.device) * scale

    def fill(self, lengths=None, spread=1.0, v_spread=1.0, part=2):
        """Random tokens in the first `lengths` places of every sequence, each page and head with a scale of its own."""
        for q8, s8, sp, p in ((self.k, self.ks, spread, part), (self.v, self.vs, v_spread, part + 1)):
            q = self.randn(self.pages, self.kv_heads, self.page, self.dh, part=p, scale=100.0).clamp(-TOP, TOP)
            q = q.to(torch.float8_e4m3fn).view(torch.uint8)
            e = torch.round(self.randn(self.pages, self.kv_heads, part=p + 20, scale=sp)) - 6.0
            for b, n in enumerate(self.lengths if lengths is None else lengths):
                for j in range(-(-n // self.page)):
                    at, used = self.table_list[b][j], min(self.page, n - j * self.page)
                    q8[at, :, :used] = q[at, :, :used]
                    s8[at] = (e[at] + 127).to(torch.uint8)

    def token_values(self, which, b):
        """[kv_heads, length, dh] of sequence b in 64 bits."""
        q8, s8 = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        pages = torch.tensor(self.table_list[b], dtype=torch.long, device=self.device)
        x = q8[pages].contiguous().view(torch.float8_e4m3fn).float().double() * pow2(s8[pages])[:, :, None, None]
        return x.transpose(0, 1).reshape(self.kv_heads, -1, self.dh)[:, :self.lengths[b]]


def attend(c, q, scale, causal):
    """(out [rows, heads, dh], lse [rows, heads], error bound of out before its rounding, of lse), rows of
    no sequence NaN.

    The scores: the queries' fp16 form is exact (bf16 values at least 2^-28 of the row's largest; smaller
    ones off by 2^-39 of it), products are exact, the tensor core drops up to 2^-23 of the magnitudes at
    every 16 of dh; the affine step to log2, the reference and the shift are three fp32 roundings of numbers no larger than
    |s| + |m| + 80 (a value scale of at most 2^64 either way).  A weight: the exponential's 2^-22,
    the rounding to fp16 2^-11 relative, below fp16's normal range 2^-25 of a weight of 1, which the row's
    largest is at least (its reference is taken so that it is 2^3 or more, or, from the sum of 64 weights, 2^6 / 64).  The sums: 2^-23
    at each step of 16 tokens, 2^-24 at each step of a sum of weights."""
    R, H, dh = c.n_rows, c.heads, c.dh
    g = H // c.kv_heads
    out = torch.full((R, H, dh), math.nan, dtype=torch.float64, device=c.device)
    lse, err, lse_err = out[:, :, 0].clone(), out.clone(), out[:, :, 0].clone()
    q = q.double().view(R, H, dh)
    for b in range(c.batch):
        n, L = c.rows[b], c.lengths[b]
        at = slice(c.starts[b], c.starts[b + 1])
        if n == 0:
            continue
        k, v = c.token_values("k", b), c.token_values("v", b)
        pages = torch.tensor(c.table_list[b], dtype=torch.long, device=c.device)
        scales = pow2(c.vs[pages]).T.repeat_interleave(c.page, 1)[:, :L]  # of a token's values
        for h in range(H):
            kh, vh = k[h // g], v[h // g]
            seen = torch.ones((n, L), dtype=torch.bool, device=c.device)
            if causal:
                seen = torch.arange(L, device=c.device) <= torch.arange(n, device=c.device)[:, None] + (L - n)
            x = torch.where(seen, q[at, h] @ kh.T * scale, -math.inf) if L else q.new_zeros((n, 0))
            # (a masked NaN counts for nothing)
            x = torch.where(seen, x, -math.inf)
            lse[at, h] = torch.logsumexp(x, 1) if L else -math.inf
            p = torch.exp(x - torch.where(torch.isinf(lse[at, h]), 0.0, lse[at, h])[:, None])
            p = torch.where(seen, p, 0.0)
            o = torch.zeros((n, dh), dtype=torch.float64, device=c.device)
            mag = torch.zeros_like(o)
            nan = torch.isnan(vh).double()
            vz = torch.nan_to_num(vh)
            if L:
                o, mag = p @ vz, p @ vz.abs()
                o = torch.where(seen.double() @ nan > 0, math.nan, o)
            out[at, h] = o
            if L:
                xa = torch.where(seen, q[at, h].abs() @ torch.nan_to_num(kh).abs().T * scale, 0.0).amax(1)
                xs = torch.where(seen, x.abs(), 0.0).amax(1)
            else:
                xa = xs = o.new_zeros(n)
            ds = xa * (dh // 16 + 2) * 2.0 ** -23 + 3 * U32 * (2 * xs + 80)
            steps = (L / 16 + 64) * 2.0 ** -23
            err[at, h] = mag * (2.0 ** -11 + 2 * ds + steps + 2.0 ** -20)[:, None]
            if L:
                most = torch.where(seen, p * (TOP * scales[h // g].nan_to_num()), 0.0).amax(1, keepdim=True)
                err[at, h] += L * 2.0 ** -25 * most + 2.0 ** -39 * mag
            lse_err[at, h] = ds + steps + 2.0 ** -20 + 4 * U32 * lse[at, h].abs().nan_to_num(posinf=0.0, neginf=0.0)
    return out, lse, err, lse_err


def check_attend(c, out, lse, q, scale, causal, stay=None):
    """stay: what rows of no sequence held before."""
    ref, ref_lse, err, lse_err = attend(c, q, scale, causal)
    o = out.double().view(c.n_rows, c.heads, c.dh)
    mine = torch.zeros(c.n_rows, dtype=torch.bool, device=c.device)
    mine[c.starts[0]:c.starts[-1]] = True
    if stay is not None:
        assert torch.all(out[~mine] == stay)
    assert torch.equal(torch.isnan(o[mine]), torch.isnan(ref[mine])), "NaN where none belongs, or none"
    bound = err + U_BF16 * (ref.abs() + err) + 2.0 ** -133
    bad = ((o - ref).abs() > bound)[mine]
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {((o - ref).abs() / bound)[mine].nan_to_num().max().item():.2f}"
    if lse is not None:
        l = lse.double().view(c.n_rows, c.heads)[mine]
        r = ref_lse[mine]
        inf = torch.isinf(r)
        assert torch.equal(torch.isinf(l) & (l < 0), inf) and torch.equal(torch.isnan(l), torch.isnan(r))
        assert torch.all(((l - r).abs() <= lse_err[mine]) | inf | torch.isnan(r))


def angles(place, freq):
    """Angles place[r][j] * freq[j] modulo a turn, of any size, exactly but for the last rounding."""
    with decimal.localcontext() as ctx:
        ctx.prec = 60
        turn = 2 * decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494")
        f = [decimal.Decimal(x) for x in freq]
        return torch.tensor([[float(decimal.Decimal(int(p)) * x % turn) for p, x in zip(row, f)] for row in place], dtype=torch.float64)


def rotate(x, a, dims, interleaved):
    """x [rows, heads, dh] in 64 bits turned by angles a [rows, dims / 2]."""
    y = x.clone()
    one = slice(0, dims, 2) if interleaved else slice(0, dims // 2)
    two = slice(1, dims, 2) if interleaved else slice(dims // 2, dims)
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    y[:, :, one], y[:, :, two] = x[:, :, one] * c - x[:, :, two] * s, x[:, :, two] * c + x[:, :, one] * s
    return y


# A rotated element: the angle is off by 2^-24 of a half turn at most, the fraction's last bit times the
# position next to nothing; cosine and sine by two steps of fp32; two products and a sum.
def rotate_err(x, dims, interleaved):
    y = torch.zeros_like(x)
    one = slice(0, dims, 2) if interleaved else slice(0, dims // 2)
    two = slice(1, dims, 2) if interleaved else slice(dims // 2, dims)
    y[:, :, one] = y[:, :, two] = (x[:, :, one].abs() + x[:, :, two].abs()) * 2.0 ** -21
    return y


def exponent(top):
    """Smallest e >= -127 with top <= 448 2^e, by trying every e."""
    e = torch.full(top.shape, -127, dtype=torch.int64, device=top.device)
    for i in range(-127, 121):
        e += (top > TOP * 2.0 ** i).long()
    return e


def check_append(c, which, new, err, before_q, before_s):
    """The cache after rows `new` [rows, kv_heads, dh] (64 bits, known to err) came in, against the bytes before:
    every page that was not written as it was, every scale the block's for values within err, every value
    within half a step of a value within err; with err = 0 exactly the rounded values."""
    q8, s8 = (c.k, c.ks) if which == "k" else (c.v, c.vs)
    want_same = torch.ones_like(before_q, dtype=torch.bool)
    scale_same = torch.ones_like(before_s, dtype=torch.bool)
    for b in range(c.batch):
        n, L = c.rows[b], c.lengths[b]
        if n == 0:
            continue
        for j in range((L - n) // c.page, (L - 1) // c.page + 1):
            p = c.table_list[b][j]
            lo, hi = max(L - n, j * c.page), min(L, (j + 1) * c.page)
            r = slice(c.starts[b] + lo - (L - n), c.starts[b] + hi - (L - n))
            x, e = new[r].transpose(0, 1), err[r].transpose(0, 1)          # [heads, tokens, dh]
            fin = torch.where(torch.isfinite(x), x.abs(), 0.0)
            top, slack = fin.amax((1, 2)), e.nan_to_num().amax((1, 2))
            floor = torch.full(top.shape, -127, dtype=torch.int64, device=top.device)
            if lo > j * c.page:
                floor = before_s[p].long() - 127
            got = s8[p].long() - 127
            assert torch.all(got >= torch.maximum(exponent(top - slack), floor)), "a scale is too small"
            assert torch.all(got <= torch.maximum(exponent(top + slack), floor)), "a scale is too large"
            scale = torch.exp2(got.double())[:, None, None]
            now = q8[p].contiguous().view(torch.float8_e4m3fn).float().double()
            a = slice(lo - j * c.page, hi - j * c.page)
            x = torch.where(torch.isinf(x), math.nan, x)
            assert torch.equal(torch.isnan(now[:, a]), torch.isnan(x))
            step = U_E4M3 * (x.abs() + e) + 0.5 * E4M3_MIN * scale + e
            assert torch.all(((now[:, a] * scale - x).abs() <= step) | torch.isnan(x)), "a value is off"
            if not err.any():
                assert torch.equal(q8[p][:, a], (x / scale).float().to(torch.float8_e4m3fn).view(torch.uint8))
            if lo > j * c.page:  # the tokens that were there
                old = before_q[p][:, :a.start].contiguous().view(torch.float8_e4m3fn).float().double()
                moved = old * torch.exp2((before_s[p].long() - 127).double())[:, None, None] / scale
                want = moved.float().to(torch.float8_e4m3fn).view(torch.uint8)
                assert torch.equal(q8[p][:, :a.start], want)
            want_same[p, :, :hi - j * c.page] = False
            scale_same[p] = False
    assert torch.equal(q8[want_same], before_q[want_same]), "bytes that belong to no token changed"
    assert torch.equal(s8[scale_same], before_s[scale_same])
