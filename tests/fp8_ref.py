"""Plain 64-bit reference of the 8-bit linear layers and the tolerances of their
tests (test helper; shares no code with the library)."""
import torch

BLOCK, TOP = 128, 448.0
U32 = 2.0 ** -24      # half a step of fp32, relative
U_BF16 = 2.0 ** -8    # of bf16
U_E4M3 = 2.0 ** -4    # of e4m3 (normal values)
E4M3_MIN = 2.0 ** -9  # smallest e4m3 step


def nblocks(cols):
    return -(-cols // BLOCK)


def storage(rows, cols, device="cuda", pad=0):
    """e4m3 bytes and scale bytes filled with a value that shows when it is changed."""
    q = torch.full((rows, -(-cols // 16) * 16 + 16 * pad), 0x55, dtype=torch.uint8, device=device)
    s = torch.full((rows, -(-nblocks(cols) // 4) * 4 + 4 * pad), 0x33, dtype=torch.uint8, device=device)
    return q, s


def pow2(byte):
    """2^(byte - 127) in 64 bits (NaN for 255)."""
    v = torch.exp2(byte.to(torch.float64) - 127.0)
    return torch.where(byte.to(torch.int32) == 255, float("nan"), v)


def values(q, s, cols):
    """What e4m3 bytes and scale bytes stand for, in 64 bits."""
    v = q[:, :cols].contiguous().view(torch.float8_e4m3fn).to(torch.float32).double()
    return v * pow2(s[:, :nblocks(cols)]).repeat_interleave(BLOCK, 1)[:, :cols]


def block_scales(x):
    """The scale byte of every block of x (64 bits): smallest e >= -127 with
    max |finite| <= 448 2^e, by trying every e."""
    rows, cols = x.shape
    a = torch.zeros((rows, nblocks(cols) * BLOCK), dtype=torch.float64, device=x.device)
    a[:, :cols] = torch.where(torch.isfinite(x), x.abs(), 0.0)
    top = a.view(rows, -1, BLOCK).amax(2)
    byte = torch.zeros(top.shape, dtype=torch.int64, device=x.device)
    for e in range(-127, 121):
        byte += (top > TOP * 2.0 ** e).long()
    return byte.to(torch.uint8), top


def quantized(x):
    """(bytes, scale bytes) of x in 64 bits; the quotients are exact, so the
    only rounding is the one to e4m3."""
    byte, _ = block_scales(x)
    quo = x / pow2(byte).repeat_interleave(BLOCK, 1)[:, :x.shape[1]]
    quo = torch.where(torch.isinf(quo), float("nan"), quo)
    return quo.to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8), byte


def check_out8(q, s, ref, err):
    """An 8-bit output against 64-bit values known to `err` (before rounding):
    each scale the one of some values within err of ref, each value within half
    an e4m3 step of such a value."""
    rows, cols = ref.shape
    byte, top = block_scales(ref)
    e = torch.zeros((rows, nblocks(cols) * BLOCK), dtype=torch.float64, device=ref.device)
    e[:, :cols] = err
    slack = e.view(rows, -1, BLOCK).amax(2)
    got = s[:, :nblocks(cols)]
    lo, hi = block_scales_of_top(top - slack), block_scales_of_top(top + slack)
    assert torch.all((got.int() >= lo) & (got.int() <= hi)), "a scale is not the block's"
    assert (got != byte).double().mean().item() < 0.01  # only at a border
    step = pow2(got).repeat_interleave(BLOCK, 1)[:, :cols]
    bound = U_E4M3 * ref.abs() + 0.5 * E4M3_MIN * step + (1 + U_E4M3) * err
    assert torch.all((values(q, s, cols) - ref).abs() <= bound)


def block_scales_of_top(top):
    byte = torch.zeros(top.shape, dtype=torch.int32, device=top.device)
    for e in range(-127, 121):
        byte += (top > TOP * 2.0 ** e).int()
    return byte


def gelu(x):
    return torch.nn.functional.gelu(x, approximate="tanh")


def gemm(A, sa, B, sb, K, bias=None):
    """(acc + bias, bound on an fp32 evaluation's error).  The tensor core adds 32
    products at a time to an fp32 sum and may drop up to 2^-23 of what the sum's
    magnitudes can reach at each step; the bias adds one rounding."""
    a, b = values(A, sa, K), values(B, sb, K)
    y, mag = a @ b.T, a.abs() @ b.abs().T
    err = mag * (2.0 ** -23 * -(-K // 32))
    if bias is not None:
        y, mag = y + bias.double(), mag + bias.double().abs()
    return y, err + U32 * mag


def gelu_bound(y, err):
    """Error of the GELU of y: slope at most 1.13; tanh.approx is within 2^-10.9
    relative, times |y| / 2; a few fp32 roundings."""
    return 1.13 * err + 0.5 * y.abs() * 2.0 ** -10.9 + 8 * U32 * y.abs()


def norm(v, err, kind, g, b, eps):
    """(norm of v times g plus b, error bound) for v known to err.  A row sum of
    W <= 8192 fp32 values in strands of at most 64 and a tree of depth <= 8 is off
    by at most C U32 of the sum of magnitudes, C = 72."""
    c = 72 * U32
    if kind != 0:
        if kind == 1:
            m = v.mean(1, keepdim=True)
            err = err + (err + c * v.abs()).mean(1, keepdim=True) + U32 * (v.abs() + m.abs())
            v = v - m
        r = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
        hat = v * r
        # the mean square's relative error: the values' and the sum's; the root halves it
        rel = (hat.abs() * err * r).mean(1, keepdim=True) + c + 4 * U32
        # (quadratic terms of err: the mean square is known to rel, never better than err itself)
        rel = rel + 2 * (err * r).square().mean(1, keepdim=True)
        v, err = hat, err * r + hat.abs() * (rel + 2 * U32)
    if g is not None:
        err = err * g.double().abs() + U32 * (v * g.double()).abs()
        v = v * g.double()
    if b is not None:
        v = v + b.double()
        err = err + U32 * (v.abs() + err)
    return v, err
