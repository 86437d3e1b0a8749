"""Plain 64-bit forms of the 8-bit projections, and what their results are held against.  Everything here runs on whatever device its tensors are on."""
import torch

F64 = torch.float64
TOP = 448.0


def power(e):
    """2^e for whole e, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(F64)


def rows_of(x):
    """[B, H, N, d] as [B N, H d]."""
    return x if x.dim() == 2 else x.permute(0, 2, 1, 3).reshape(x.shape[0] * x.shape[2], -1)


def heads_of(y, B, d):
    return y.reshape(B, y.shape[0] // B, y.shape[1] // d, d).permute(0, 2, 1, 3)


def norm64(x, weight=None, residual=None, eps=1e-6):
    t = rows_of(x).to(F64)
    if residual is not None:
        t = t + rows_of(residual).to(F64)
    y = t / torch.sqrt(t.square().sum(1, keepdim=True) / t.shape[1] + eps)
    return (y if weight is None else y * weight.to(F64)), t


def exponents64(y, block_rows=1):
    """Per row and block of 128 columns: the smallest e >= -127 with max |y| <= 448 * 2^e."""
    rows, cols = y.shape
    out = torch.empty((rows, (cols + 127) // 128), dtype=torch.int64, device=y.device)
    for k in range(out.shape[1]):
        top = y[:, 128 * k:128 * k + 128].abs().amax(1)
        if block_rows > 1:
            top = torch.cat([top[r:r + block_rows].max().expand(min(block_rows, rows - r)) for r in range(0, rows, block_rows)])
        e = torch.floor(torch.log2(torch.clamp(top, min=1e-300) / TOP)) - 1
        for _ in range(3):
            e = torch.where(top > TOP * power(e), e + 1, e)
        out[:, k] = torch.clamp(e, min=-127).to(torch.int64)
    return out


def table(scales, cols):
    """The bytes [rows, blocks] of the scales as they are kept, and those behind the last block."""
    b = scales.permute(1, 0, 2).reshape(scales.shape[1], -1).to(torch.int64)
    n = (cols + 127) // 128
    return b[:, :n], b[:, n:]


def value64(pair):
    """The matrix that a pair stands for; NaN where the scale is."""
    data, scales = pair
    e, _ = table(scales, data.shape[1])
    factor = torch.where(e == 255, torch.full_like(e, 0).to(F64) + float("nan"), power(e - 127))
    return data.to(F64) * factor.repeat_interleave(128, 1)[:, :data.shape[1]]


def check_form(pair, y, block_rows=1, slack=0.0):
    """`pair` is the 8-bit form of `y` (64 bits), of which the kernel saw a value up to `slack` (relative) away: scales are exact but where y's largest value
    is that close to a scale's bound; values are within half a spacing of e4m3 (2^-4 relative, 2^-10 of the scale below the normal ones) and the slack."""
    data, scales = pair
    e, behind = table(scales, y.shape[1])
    assert bool((behind == 0).all())
    low, high = exponents64(y * (1 - slack), block_rows), exponents64(y * (1 + slack), block_rows)
    assert bool(((e - 127 >= low) & (e - 127 <= high)).all())
    step = power(e - 127).repeat_interleave(128, 1)[:, :y.shape[1]]
    off = (value64(pair) - y).abs()
    assert bool((off <= torch.maximum(y.abs() * 2.0 ** -4, step * 2.0 ** -10) + y.abs() * slack).all())


def check_matmul(out, a, w, bias=None):
    """`out` (bf16, rows or heads) against the product in 64 bits.  Error: half a spacing of bf16 (2^-8 relative), and for the sums in fp32 one rounding or truncation
    (2^-23) of at most the sum of all |products| for every 32 columns, twice, and one for the bias."""
    av, wv = value64(a), value64(w)
    ref = av @ wv.T
    size = av.abs() @ wv.abs().T
    if bias is not None:
        ref, size = ref + bias.to(F64), size + bias.to(F64).abs()
    tol = ref.abs() * 2.0 ** -8 + size * 2.0 ** -23 * 2 * (av.shape[1] / 32 + 2)
    got = rows_of(out).to(F64)
    bad = ~((got - ref).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), float((got - ref).abs().max()))


def pair_of(x, block_rows=1):
    """The 8-bit form of x (64 bits) as tensors, made here."""
    rows, cols = x.shape
    e = exponents64(x, block_rows)
    q = x / power(e).repeat_interleave(128, 1)[:, :cols]
    data = torch.zeros((rows, (cols + 15) // 16 * 16), dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn)
    data[:, :cols] = q.to(torch.float32).to(torch.float8_e4m3fn)
    groups = (cols + 511) // 512
    full = torch.zeros((rows, 4 * groups), dtype=torch.uint8, device=x.device)
    full[:, :e.shape[1]] = (e + 127).to(torch.uint8)
    return data[:, :cols], full.reshape(rows, groups, 4).permute(1, 0, 2).contiguous()
