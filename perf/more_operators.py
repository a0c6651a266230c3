"""Operators of attention over a paged 8-bit cache: their performance cases and
plain forms.

Two operators of a transformer block that keeps its keys and values between
calls, in pages of P tokens, as e4m3 values with one power-of-two scale for
each page and head:

* ``append``  f3dc.kv_append_fp8: the keys and values of new tokens into the
              pages of their sequences, the keys (and the queries) rotated by
              their positions on the way.
* ``attend``  f3dc.kv_attention_fp8: attention of packed query rows over the
              cache, from single tokens over long caches to whole prompts,
              also with several query heads to a key head and causal.

``own`` selects the library's calls; otherwise ``run`` computes the operators
from elementary torch operations in 32 bits.  Sizes are those of the library's
configurations (16 heads of 64, 1374 condition tokens, 16^3 and 32^3 grids,
eight samples with up to 955 active tokens) or generic ones around them.
"""
import math

import torch

own = False

DEV = "cuda"
TOP = 448.0      # largest e4m3 value
BASE = 10000.0   # of the rotation's frequencies

_f3dc = None


def _lib():
    """The library's binding, imported only where its calls are made."""
    global _f3dc
    if _f3dc is None:
        from paper_2511_22533_gb300 import f3dc
        _f3dc = f3dc
    return _f3dc


# ---------------------------------------------------------------- the cases

def _append(batch, rows, ctx, heads, kv_heads, dh, page, ragged=False, dims=None, interleaved=False, axes=1, **kw):
    return dict(op="append", batch=batch, rows=rows, ctx=ctx, ragged=ragged, heads=heads, kv_heads=kv_heads, dh=dh, page=page,
                dims=dims or dh, interleaved=interleaved, axes=axes, **kw)


def _attend(batch, rows, ctx, heads, kv_heads, dh, page, causal, cross=False, ragged=False, **kw):
    return dict(op="attend", batch=batch, rows=rows, ctx=ctx, ragged=ragged, heads=heads, kv_heads=kv_heads, dh=dh, page=page,
                causal=causal, cross=cross, **kw)


def listed():
    return [
        # one sequence's next token: latency
        _append(1, 1, 1000, 16, 16, 64, 64, name="append_token"),
        # the next tokens of 64 sequences of different lengths, four query heads to a key head
        _append(64, 1, 5000, 32, 8, 128, 64, ragged=True, name="append_decode_b64"),
        # the active tokens of eight samples, rotated by their places in the grid, odd lengths before and after
        _append(8, 955, 333, 16, 16, 64, 32, ragged=True, dims=64, axes=3, name="append_ragged_b8"),
        # every token of a 32^3 grid, neighbouring elements rotated
        _append(1, 32768, 0, 16, 16, 64, 64, interleaved=True, name="append_grid_32768"),
        # one token over the condition tokens: latency
        _attend(1, 1, 1374, 16, 16, 64, 64, False, cross=True, name="attend_token_1374"),
        # a decoding step of 64 sequences of different lengths
        _attend(64, 1, 8191, 32, 8, 128, 64, True, ragged=True, name="attend_decode_b64"),
        # one sequence's next token over a very long cache, small pages
        _attend(1, 1, 524287, 32, 8, 128, 16, True, name="attend_decode_524288"),
        # a few tokens at once of four sequences, an odd number of query heads to a key head
        _attend(4, 5, 30000, 12, 4, 64, 32, True, ragged=True, name="attend_draft_b4"),
        # active tokens of a cached step over the condition tokens
        _attend(1, 1229, 1374, 16, 16, 64, 128, False, cross=True, name="attend_cross_1229"),
        # chunks of eight prompts behind what their caches hold
        _attend(8, 955, 6000, 32, 8, 128, 64, True, ragged=True, name="attend_chunks_b8"),
        # a whole prompt
        _attend(1, 8192, 0, 32, 8, 128, 64, True, name="attend_prompt_8192"),
        # every token of a 32^3 grid over all of them
        _attend(1, 32768, 0, 16, 16, 64, 64, False, name="attend_grid_32768"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most_flops, most_bytes = 4.0 * 64 * 16 * 32768 ** 2, 524288 * 8 * 128 * 2
    while True:
        kv_heads, group = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 1, 2, 3, 4, 8])
        shape = (kv_heads * group, kv_heads, rng.choice([32, 64, 128]), rng.choice([16, 32, 64, 128]))
        batch, ragged = _log_int(rng, 1, 128), rng.random() < 0.6
        if rng.random() < 0.35:
            rows = 1 if rng.random() < 0.3 else _log_int(rng, 1, 32768 // batch)
            ctx = 0 if rng.random() < 0.2 else _log_int(rng, 1, 8192)
            dims = rng.choice([shape[2], shape[2] // 2])
            c = _append(batch, rows, ctx, *shape, ragged=ragged, dims=dims, interleaved=rng.random() < 0.4,
                        axes=rng.choice([1, 1, 2, 3]))
            if batch * rows * (shape[0] + shape[1]) * shape[2] <= 32768 * 32 * 64 * 2 and work(c)["bytes"] <= most_bytes:
                return c
            continue
        # single tokens, a few, many
        rows = rng.choice([1, _log_int(rng, 2, 64), _log_int(rng, 64, 32768)])
        cross = rng.random() < 0.3
        ctx = _log_int(rng, 1, 524288) if cross or rng.random() < 0.8 else 0
        c = _attend(batch, rows, ctx, *shape, causal=not cross and rng.random() < 0.7, cross=cross, ragged=ragged)
        w = work(c)
        if w["flops"] <= most_flops and w["bytes"] <= most_bytes and batch * rows * shape[0] * shape[2] <= 2 ** 27:
            return c


def _lengths(c):
    """Rows of each sequence and the tokens that its cache holds with them."""
    def spread(n, b):  # from half of n (rounded) to n
        return n if not c["ragged"] else int(round(n * (0.5 + 0.5 * (b * 5 % c["batch"] + 1) / c["batch"])))

    rows = [max(1, spread(c["rows"], b)) for b in range(c["batch"])]
    held = [spread(c["ctx"], c["batch"] - 1 - b) for b in range(c["batch"])]
    if c["op"] == "attend" and c["cross"]:
        return rows, held
    return rows, [h + n for h, n in zip(held, rows)]


# ------------------------------------------------------------------ inputs

def _gen(seed, part):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 64 + part)


def _randn(shape, seed, part, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=_gen(seed, part), device=DEV) * scale).to(dtype)


def _heads(rows, heads, dh, seed, part):
    """Normal rows whose size differs, with a few channels of each head that are
    larger than the others, as keys have."""
    x = _randn((rows, heads, dh), seed, part)
    x *= torch.exp(0.3 * _randn((rows, 1, 1), seed, part + 1))
    big = torch.rand((heads, dh), generator=_gen(seed, part + 2), device=DEV) < 0.03
    return (x * torch.where(big, 8.0, 1.0)).reshape(rows, heads * dh)


def _exponent(top):
    """The smallest e >= -127 with top <= 448 2^e."""
    m, p = torch.frexp(top)                             # top = m 2^p, m in [1/2, 1)
    e = (p - 9 + (m > 0.875).int()).clamp(-127, 127)    # 448 = 0.875 2^9
    return torch.where(m == 0, torch.full_like(e, -127), e)


def _e4m3(x, e):
    return torch.ldexp(x, -e).clamp(-TOP, TOP).to(torch.float8_e4m3fn)


def _pool(pages, kv_heads, page, dh, seed, part):
    """Pages that hold tokens: e4m3 bytes [pages, heads, tokens, dh] and scale
    bytes [pages, heads]."""
    q = torch.empty((pages, kv_heads, page, dh), dtype=torch.uint8, device=DEV)
    s = torch.empty((pages, kv_heads), dtype=torch.uint8, device=DEV)
    some = max(1, 2 ** 26 // (kv_heads * page * dh))
    for i, lo in enumerate(range(0, pages, some)):
        n = min(some, pages - lo)
        x = _heads(n * page, kv_heads, dh, seed * 4096 + i, part).view(n, page, kv_heads, dh).transpose(1, 2)
        e = _exponent(x.abs().amax((2, 3)))
        q[lo:lo + n] = _e4m3(x, e[:, :, None, None]).view(torch.uint8)
        s[lo:lo + n] = (e + 127).to(torch.uint8)
    return q, s


def _inputs(c, seed):
    rows, lengths = _lengths(c)
    H, Hk, dh, P, B = c["heads"], c["kv_heads"], c["dh"], c["page"], c["batch"]
    need = [-(-n // P) for n in lengths]
    pages = max(1, sum(need))
    order = torch.randperm(pages, generator=_gen(seed, 0), device=DEV).to(torch.int32)
    table = torch.zeros((B, max(1, max(need))), dtype=torch.int32, device=DEV)
    first = [sum(need[:b]) for b in range(B)]
    for b in range(B):
        table[b, :need[b]] = order[first[b]:first[b] + need[b]]
    starts = [sum(rows[:b]) for b in range(B + 1)]
    t = dict(n=rows, lengths=lengths, starts=starts, table=table,
             row_start_dev=torch.tensor(starts, dtype=torch.int32, device=DEV),
             lengths_dev=torch.tensor(lengths, dtype=torch.int32, device=DEV))
    t["k8"], t["ks"] = _pool(pages, Hk, P, dh, seed, 1)
    t["v8"], t["vs"] = _pool(pages, Hk, P, dh, seed, 5)
    R = starts[-1]
    t["q"] = _heads(R, H, dh, seed, 9).to(torch.bfloat16)
    if c["op"] == "append":
        # keys and values side by side, as one projection writes them; some pages' tokens larger than before
        kv = torch.cat([_heads(R, Hk, dh, seed, 12), _heads(R, Hk, dh, seed, 15)], 1)
        t["kv"] = (kv * torch.exp(0.5 * _randn((R, 1), seed, 18))).to(torch.bfloat16)
        t["q_out"] = torch.zeros_like(t["q"])
        pairs = c["dims"] // 2 // c["axes"]  # of an axis
        t["freq"] = [BASE ** (-(j % pairs) / pairs) if j < pairs * c["axes"] else 0.0 for j in range(c["dims"] // 2)]
        t["positions"] = None
        if c["axes"] > 1:  # places in a grid
            t["positions"] = torch.randint(0, 64, (R, c["axes"]), generator=_gen(seed, 19), device=DEV).to(torch.int32)
    return t


def prepare(case, seed):
    c = dict(case)
    t = _inputs(c, seed)
    s = dict(c=c, t=t)
    if c["op"] == "attend":
        s["out"] = torch.zeros_like(t["q"])
        s["lse"] = torch.zeros((t["starts"][-1], c["heads"]), dtype=torch.float32, device=DEV)
    if own:
        f = _lib()
        s["cache"] = f.KVCache(t["k8"], t["v8"], t["ks"], t["vs"])
        s["batch"] = f.KVBatch(t["row_start_dev"], t["lengths_dev"], t["table"], rows=t["starts"][-1], max_rows=max(t["n"]),
                               max_length=max(t["lengths"]))
        if c["op"] == "append":
            s["rotary"] = f.Rotary(c["dims"], t["freq"], interleaved=c["interleaved"], axes=c["axes"])
        else:
            n = f.kv_attention_workspace(s["cache"], s["batch"], c["heads"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    if c["op"] == "append":
        s["out"] = {"q": t["q_out"], "k": t["k8"].view(torch.float8_e4m3fn), "k_scales": t["ks"].view(torch.float8_e8m0fnu),
                    "v": t["v8"].view(torch.float8_e4m3fn), "v_scales": t["vs"].view(torch.float8_e8m0fnu)}
    return s


# --------------------------------------------------------------------- run

def _plain_rotated(x, cos, sin, interleaved):
    """x [rows, heads, dh] with its first dims rotated by cos, sin [rows, 1, dims / 2]."""
    half = cos.shape[2]
    if interleaved:
        a, b = x[:, :, 0:2 * half:2], x[:, :, 1:2 * half:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], 3).flatten(2)
    else:
        a, b = x[:, :, :half], x[:, :, half:2 * half]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], 2)
    return torch.cat([y, x[:, :, 2 * half:]], 2)


def _plain_store(c, new, page, slot, first, held, q8, scales):
    """New rows [rows, heads, dh] into (page, slot); first: the page that each
    sequence goes on in, held: the tokens there that stay."""
    top = torch.zeros(scales.shape, dtype=torch.float32, device=DEV)
    top.index_reduce_(0, page, new.abs().amax(2), "amax")
    e = _exponent(top) + 127
    some = held > 0
    first, held = first[some], held[some]
    old = scales[first].int()
    e[first] = torch.maximum(e[first], old)
    rows = q8[first].view(torch.float8_e4m3fn).float()
    moved = _e4m3(rows, (e[first] - old)[:, :, None, None]).view(torch.uint8)
    stay = torch.arange(c["page"], device=DEV) < held[:, None]
    q8[first] = torch.where(stay[:, None, :, None], moved, q8[first])
    q8[page, :, slot] = _e4m3(new, e[page][:, :, None] - 127).view(torch.uint8)
    scales[page] = e[page].to(torch.uint8)


def _plain_append(s):
    c, t = s["c"], s["t"]
    R, H, Hk, dh, P = t["starts"][-1], c["heads"], c["kv_heads"], c["dh"], c["page"]
    counts = t["row_start_dev"][1:] - t["row_start_dev"][:-1]
    held = (t["lengths_dev"] - counts).long()
    seq = torch.repeat_interleave(torch.arange(c["batch"], device=DEV), counts, output_size=R)
    token = torch.arange(R, device=DEV) - t["row_start_dev"][:-1].long()[seq] + held[seq]
    at = t["positions"] if t["positions"] is not None else token[:, None]
    pairs = c["dims"] // 2 // c["axes"]
    axis = torch.arange(c["dims"] // 2, device=DEV).div(pairs, rounding_mode="floor").clamp(max=c["axes"] - 1)
    angle = at.double()[:, axis] * torch.tensor(t["freq"], dtype=torch.float64, device=DEV)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q = _plain_rotated(t["q"].float().view(R, H, dh), cos, sin, c["interleaved"])
    k, v = t["kv"].float().view(R, 2, Hk, dh).unbind(1)
    page = t["table"][seq, token // P].long()
    first = t["table"][torch.arange(c["batch"], device=DEV), (held // P).clamp(max=t["table"].shape[1] - 1)].long()
    k = _plain_rotated(k, cos, sin, c["interleaved"])
    _plain_store(c, k, page, token % P, first, held % P, t["k8"], t["ks"])
    _plain_store(c, v, page, token % P, first, held % P, t["v8"], t["vs"])
    t["q_out"].copy_(q.view(R, H * dh))
    return s["out"]


def _plain_attend(s):
    c, t = s["c"], s["t"]
    H, Hk, dh, P = c["heads"], c["kv_heads"], c["dh"], c["page"]
    g, scale = H // Hk, 1.0 / math.sqrt(dh)

    def values(q8, e):  # [pages, heads, P, dh] -> [heads, tokens, dh]
        v = torch.ldexp(q8.view(torch.float8_e4m3fn).float(), (e.int() - 127)[:, :, None, None])
        return v.transpose(0, 1).reshape(v.shape[1], -1, dh)

    for b, (n, L) in enumerate(zip(t["n"], t["lengths"])):
        lo = t["starts"][b]
        if L == 0:
            s["out"][lo:lo + n] = 0.0
            s["lse"][lo:lo + n] = -math.inf
            continue
        pages = t["table"][b, :-(-L // P)].long()
        q = t["q"][lo:lo + n].float().view(n, Hk, g, dh)
        heads = max(1, min(Hk, 2 ** 29 // (L * n * g)))          # at once, and rows
        rows = max(1, min(n, 2 ** 29 // (L * heads * g)))
        for h in range(0, Hk, heads):
            k = values(t["k8"][pages, h:h + heads], t["ks"][pages, h:h + heads])[:, :L]
            v = values(t["v8"][pages, h:h + heads], t["vs"][pages, h:h + heads])[:, :L]
            m = k.shape[0]
            for r in range(0, n, rows):
                qr = q[r:r + rows, h:h + heads].permute(1, 0, 2, 3)      # [heads, rows, g, dh]
                x = torch.matmul(qr.reshape(m, -1, dh), k.transpose(1, 2)).mul_(scale)
                if c["causal"]:
                    place = torch.arange(r, r + qr.shape[1], device=DEV) + (L - n)
                    hidden = torch.arange(L, device=DEV) > place.repeat_interleave(g)[:, None]
                    x.masked_fill_(hidden, -math.inf)
                top = x.amax(2, keepdim=True)
                x = torch.exp_(x.sub_(top.clamp(min=-3.0e38)))
                total = x.sum(2, keepdim=True)
                o = torch.matmul(x, v) / total
                o, total, top = (torch.where(total > 0, o, 0.0), total.log() + top, None)
                at = slice(lo + r, lo + r + qr.shape[1])
                s["out"][at].view(-1, Hk, g, dh)[:, h:h + heads] = o.view(m, -1, g, dh).permute(1, 0, 2, 3).to(torch.bfloat16)
                s["lse"][at].view(-1, Hk, g)[:, h:h + heads] = total.view(m, -1, g).permute(1, 0, 2)
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    s, c, t = state, state["c"], state["t"]
    if c["op"] == "append":
        if not own:
            return _plain_append(s)
        W, kv, q = c["kv_heads"] * c["dh"], t["kv"], t["q"]
        _lib().kv_append_fp8(s["cache"], s["batch"], kv, kv.stride(0), kv[:, W:], kv.stride(0), q=q, ldq=q.stride(0),
                             q_out=t["q_out"], ldqo=t["q_out"].stride(0), heads=c["heads"], rotary=s["rotary"],
                             positions=t["positions"])
        return s["out"]
    if not own:
        return _plain_attend(s)
    q, o = t["q"], s["out"]
    _lib().kv_attention_fp8(s["cache"], s["batch"], q, q.stride(0), o, o.stride(0), c["heads"], 1.0 / math.sqrt(c["dh"]),
                            causal=c["causal"], lse=s["lse"], workspace=s["workspace"])
    return {"out": o, "lse": s["lse"]}


# -------------------------------------------------------------------- work

def _visible(c):
    """Keys that some row sees and (row, key) pairs, over all sequences."""
    keys = pairs = 0
    for n, L in zip(*_lengths(c)):
        keys += L
        pairs += n * L - (n * (n - 1) // 2 if c["causal"] else 0)
    return keys, pairs


def work(case):
    c = case
    rows, _ = _lengths(c)
    R, H, Hk, dh = sum(rows), c["heads"], c["kv_heads"], c["dh"]
    if c["op"] == "append":
        pages = sum(-(-n // c["page"]) for n in rows)
        return {"bytes": R * dh * (4 * H + 6 * Hk) + 2 * Hk * pages + 4 * pages + (4 * c["axes"] * R if c["axes"] > 1 else 0),
                "flops": 3.0 * R * (H + Hk) * c["dims"] + 4.0 * R * Hk * dh}
    keys, pairs = _visible(c)
    pages = -(-keys // c["page"])
    return {"bytes": 2 * Hk * (keys * dh + pages) + 4 * pages + R * H * (4 * dh + 4), "flops": 4.0 * dh * H * pairs}


# ------------------------------------------------------------------- exact

def _exact_stored(c, t, new, q8, scales):
    """Unrounded quotients and scales of the whole cache in 64 bits after the
    rows `new` [rows, heads, dh] came in, sequence by sequence, page by page."""
    P = c["page"]
    q = q8.contiguous().view(torch.float8_e4m3fn).double()
    scale = torch.exp2(scales.double() - 127.0)
    for b, (n, L) in enumerate(zip(t["n"], t["lengths"])):
        table = t["table"][b].tolist()
        for j in range((L - n) // P, (L - 1) // P + 1):
            lo, hi = max(L - n, j * P), min(L, (j + 1) * P)          # tokens of this page
            x = new[t["starts"][b] + lo - (L - n):t["starts"][b] + hi - (L - n)].transpose(0, 1)
            top = x.abs().amax((1, 2))
            e = torch.ceil(torch.log2(top / TOP)).clamp(-127, 127)
            # log2 may be off next to a power of two
            e = torch.where(top <= TOP * torch.exp2(e - 1), e - 1, e)
            e = torch.where(top > TOP * torch.exp2(e), e + 1, e).clamp(-127, 127)
            f, p = torch.exp2(e), table[j]
            if lo > j * P:
                f = torch.maximum(f, scale[p])
                q[p, :, :lo - j * P] *= (scale[p] / f)[:, None, None]
            q[p, :, lo - j * P:hi - j * P] = x / f[:, None, None]
            scale[p] = f
    return q, scale


def exact(case, seed):
    c = dict(case)
    t = _inputs(c, seed)
    R, H, Hk, dh, P = t["starts"][-1], c["heads"], c["kv_heads"], c["dh"], c["page"]
    if c["op"] == "append":
        half, pairs = c["dims"] // 2, c["dims"] // 2 // c["axes"]
        place = torch.empty((R, half), dtype=torch.float64, device=DEV)
        for b, (n, L) in enumerate(zip(t["n"], t["lengths"])):
            at = slice(t["starts"][b], t["starts"][b + 1])
            place[at] = torch.arange(L - n, L, dtype=torch.float64, device=DEV)[:, None]
        if t["positions"] is not None:
            for a in range(c["axes"]):
                place[:, a * pairs:(a + 1) * pairs] = t["positions"][:, a:a + 1].double()
        turn = torch.polar(torch.ones_like(place), place * torch.tensor(t["freq"], dtype=torch.float64, device=DEV))

        def rotated(x):
            y = x.double().view(R, -1, dh).clone()
            one, two = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["interleaved"] else (slice(0, half), slice(half, 2 * half))
            z = torch.complex(y[:, :, one].contiguous(), y[:, :, two].contiguous()) * turn[:, None]
            y[:, :, one], y[:, :, two] = z.real, z.imag
            return y

        k, ks = _exact_stored(c, t, rotated(t["kv"][:, :Hk * dh]), t["k8"], t["ks"])
        v, vs = _exact_stored(c, t, t["kv"][:, Hk * dh:].double().view(R, Hk, dh), t["v8"], t["vs"])
        return {"q": rotated(t["q"]).view(R, H * dh), "k": k, "k_scales": ks, "v": v, "v_scales": vs}
    out = torch.zeros((R, H * dh), dtype=torch.float64, device=DEV)
    lse = torch.full((R, H), -math.inf, dtype=torch.float64, device=DEV)
    g = H // Hk
    for b, (n, L) in enumerate(zip(t["n"], t["lengths"])):
        if L == 0:
            continue
        pages = t["table"][b, :-(-L // P)].long()
        for h in range(Hk):
            k, v = ((q8[pages, h].view(torch.float8_e4m3fn).double() * torch.exp2(e[pages, h].double() - 127.0)[:, None, None])
                    .reshape(-1, dh)[:L] for q8, e in ((t["k8"], t["ks"]), (t["v8"], t["vs"])))
            for i in range(g):
                col = slice((h * g + i) * dh, (h * g + i + 1) * dh)
                for r in range(0, n, 4096):
                    at = slice(t["starts"][b] + r, t["starts"][b] + min(r + 4096, n))
                    x = t["q"][at, col].double() @ k.T / math.sqrt(dh)
                    if c["causal"]:
                        last = torch.arange(r, r + x.shape[0], device=DEV) + (L - n)
                        x = torch.where(torch.arange(L, device=DEV) <= last[:, None], x, -math.inf)
                    lse[at, h * g + i] = torch.logsumexp(x, 1)
                    out[at, col] = torch.softmax(x, 1) @ v
    return {"out": out, "lse": lse}
