"""Plain 64-bit forms of the bf16 steps around the attention, and what their results are held against.  Everything here runs on whatever device its tensors are on."""
import math

import torch

F64 = torch.float64
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of a type, relative to the value


def rows_of(x):
    """[B, H, N, d] as [B N, H d]."""
    return x if x.dim() == 2 else x.permute(0, 2, 1, 3).reshape(x.shape[0] * x.shape[2], -1)


def heads_of(y, B, d):
    return y.reshape(B, y.shape[0] // B, y.shape[1] // d, d).permute(0, 2, 1, 3)


def within(got, ref, tol, what=""):
    got = got.to(F64)
    off = (got - ref).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), off.numel(), float((off / tol.clamp(min=1e-300))[bad].max()), got[bad][:4].tolist(), ref[bad][:4].tolist())


# ------------------------------------------------------------------------------------------------ rotation
def frequencies64(n, base=10000.0, scaling=None, factor=1.0, original=0.0):
    """(angle of one position for each of n pairs, amplitude)"""
    if scaling == "ntk":
        return [(base * factor ** (n / (n - 1))) ** (-i / n) if n > 1 else 1.0 for i in range(n)], 1.0
    f = [base ** (-i / n) for i in range(n)]
    if scaling == "linear":
        return [v / factor for v in f], 1.0
    if scaling == "yarn":
        g = [min(1.0, max(0.0, (original * v / math.tau - 1) / 31)) for v in f]
        return [v * a + v / factor * (1 - a) for v, a in zip(f, g)], 0.1 * math.log(factor) + 1
    return f, 1.0


def table64(sizes, pairs, **how):
    out = torch.zeros(sum(sizes), sum(pairs), 2, dtype=F64)
    row = col = 0
    for size, n in zip(sizes, pairs):
        f, amplitude = frequencies64(n, **how)
        angle = torch.arange(size, dtype=F64)[:, None] * torch.tensor(f, dtype=F64)
        out[row:row + size, col:col + n, 0] = amplitude * angle.cos()
        out[row:row + size, col:col + n, 1] = amplitude * angle.sin()
        row, col = row + size, col + n
    return out


def factors64(table, B, N, positions=None, first=0):
    """(cos, sin) [B, 1, N, P] of a table (factors, sizes, pairs); NaN for positions that are not there."""
    factors, sizes, pairs = table
    f = factors.to(F64)
    if positions is None:
        i, at = torch.arange(first, first + N, device=f.device), []
        for size in reversed(sizes):
            at.insert(0, (i % size).expand(B, N))
            i = i // size
    else:
        p = positions.reshape(positions.shape + (1,)) if len(sizes) == 1 and positions.dim() < 3 else positions
        at = [p[..., a].expand(B, N) for a in range(len(sizes))]
    out, row, col = [], 0, 0
    for a, (size, n) in enumerate(zip(sizes, pairs)):
        ok = (at[a] >= 0) & (at[a] < size)
        v = f[row + at[a].clamp(0, size - 1).long(), col:col + n]
        out.append(torch.where(ok[..., None, None], v, torch.full_like(v, float("nan"))))
        row, col = row + size, col + n
    cs = torch.cat(out, 2)[:, None]
    return cs[..., 0], cs[..., 1]


def turn64(x, cs, layout, inverse=False):
    c, s = cs
    s = -s if inverse else s
    p = c.shape[-1]
    y = x.to(F64).clone()
    ia, ib = (slice(0, 2 * p, 2), slice(1, 2 * p, 2)) if layout == "interleaved" else (slice(0, p), slice(p, 2 * p))
    a, b = y[..., ia].clone(), y[..., ib].clone()
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    return y


def size_of_turn(x, cs, layout):
    """For each element the sum of the absolute products that it is made of."""
    c, s = (v.abs().nan_to_num() for v in cs)
    p = c.shape[-1]
    y = x.to(F64).abs()
    ia, ib = (slice(0, 2 * p, 2), slice(1, 2 * p, 2)) if layout == "interleaved" else (slice(0, p), slice(p, 2 * p))
    a, b = y[..., ia].clone(), y[..., ib].clone()
    y[..., ia], y[..., ib] = a * c + b * s, a * s + b * c
    return y


def normed64(x, w, norm, eps):
    """(n = x r, r, weights laid out like x)"""
    B, H, N, d = x.shape
    x = x.to(F64)
    dims = (3,) if norm == "head" else (1, 3)
    r = 1 / torch.sqrt(x.square().mean(dims, keepdim=True) + eps)
    if w is None:
        w = torch.ones(d if norm == "head" else H * d, dtype=F64, device=x.device)
    return x * r, r, w.to(F64) if norm == "head" else w.to(F64).reshape(1, H, 1, d)


# fp32: x r w is three roundings and rsqrt's 2 ulp, the sum of squares up to 64 roundings one behind another (48 of a lane, the exchanges, the warps), halved by the root: 2^-18; with the turn's
# two roundings of either product still below 2^-17.
SLACK = 2.0 ** -17


def check_forward(got, x, w, cs, norm, eps, layout, what="", inverse=False):
    if norm is None:
        n = x.to(F64)
    else:
        n, _, scale = normed64(x, w, norm, eps)
        n = n * scale
    ref, size = (n, n.abs()) if cs is None else (turn64(n, cs, layout, inverse), size_of_turn(n, cs, layout))
    bad = ref.isnan()
    assert bool((got.isnan() == bad).all()), what
    within(got[~bad], ref[~bad], ref[~bad].abs() * HALF[x.dtype] + size[~bad] * SLACK + 1e-38, what)


def check_backward(got, dy, x, w, cs, norm, eps, layout, got_w=None, what=""):
    n, r, scale = normed64(x, w, norm, eps)
    d = dy.to(F64) if cs is None else turn64(dy, cs, layout, inverse=True)
    size = dy.to(F64).abs() if cs is None else size_of_turn(dy, cs, layout)
    dims = (3,) if norm == "head" else (1, 3)
    g = d * scale
    ref = r * (g - n * (g * n).mean(dims, keepdim=True))
    # every term's products, each off by the slack (sums over a row: up to 2^-18 of the absolute terms)
    reach = r * (size * scale.abs() + n.abs() * (size * scale.abs() * n.abs()).mean(dims, keepdim=True)) * 2 * SLACK
    within(got, ref, ref.abs() * HALF[x.dtype] + reach + 1e-38, what)
    if got_w is not None:
        dw, over = d * n, size * n.abs()
        dw, over = (v.sum((0, 1, 2)) if norm == "head" else v.sum((0, 2)).reshape(-1) for v in (dw, over))
        # sums over tokens (and heads) in runs: fewer than 256 additions one behind another
        within(got_w, dw, dw.abs() * HALF[got_w.dtype] + over * (SLACK + 2.0 ** -16) + 1e-38, what + " weight")


# ------------------------------------------------------------------------------------------------ linear layers
def act64(z, act):
    """(value, derivative)"""
    if act is None:
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(F64)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * torch.sigmoid(-z))
    if act == "gelu":
        c = torch.special.erfc(-z / math.sqrt(2)) / 2
        return z * c, c + z * torch.exp(-z * z / 2) / math.sqrt(math.tau)
    k = math.sqrt(2 / math.pi)
    s = torch.sigmoid(2 * k * (z + 0.044715 * z ** 3))
    t = torch.sigmoid(-2 * k * (z + 0.044715 * z ** 3))
    return z * s, s + 2 * k * z * s * t * (1 + 3 * 0.044715 * z * z)


def product_tol(size, k):
    """Of a sum of k products in fp32: one rounding or truncation (2^-23) of at most the sum of all |products| for every 16 of them, twice, and one for the bias; of parts that are added up, 32 more."""
    return size * 2.0 ** -23 * 2 * (k / 16 + 34)


# Activations: exponentials of arguments up to 90, whose rounding (three of 2^-24) is relative to the argument: below 2^-15 of the value; their slopes are bounded by 1.13.
ACT = 2.0 ** -14


def spread(gate, rows):
    return None if gate is None else gate.to(F64).reshape(-1, gate.shape[-1]).repeat_interleave(rows // (gate.shape[0] if gate.dim() == 2 else 1), 0)


def check_linear(y, x, w, bias=None, act=None, gate=None, residual=None, pre=None):
    xv, wv = rows_of(x).to(F64), w.to(F64)
    z, size = xv @ wv.T, xv.abs() @ wv.abs().T
    if bias is not None:
        z, size = z + bias.to(F64), size + bias.to(F64).abs()
    tol = product_tol(size, xv.shape[1])
    if pre is not None:
        within(rows_of(pre), z, z.abs() * 2.0 ** -8 + tol + 1e-38, "pre")
    u, _ = act64(z, act)
    tol = 1.13 * tol + u.abs() * ACT if act else tol
    g = spread(gate, xv.shape[0])
    if g is not None:
        u, tol = u * g, tol * g.abs() + (u * g).abs() * 2.0 ** -23
    ref = u if residual is None else u + rows_of(residual).to(F64)
    tol = tol + (0 if residual is None else ref.abs() * 2.0 ** -24)
    within(rows_of(y), ref, ref.abs() * HALF[y.dtype] + tol + 1e-38, "y")


def check_linear_backward(got, dy, x, w, pre=None, act=None, gate=None, bias=None):
    dyv, xv, wv = rows_of(dy).to(F64), rows_of(x).to(F64), w.to(F64)
    z = torch.zeros_like(dyv) if pre is None else rows_of(pre).to(F64)
    u, slope = act64(z, act)
    g = spread(gate, dyv.shape[0])
    e = dyv if g is None else dyv * g
    dz = e * slope
    rounded = act is not None or gate is not None or dy.dtype != torch.bfloat16
    off = e.abs() * ACT * (act is not None) + dz.abs() * (2.0 ** -8 + 2.0 ** -22 if rounded else 0)     # of an operand: its rounding to bf16
    for name, grad, ref, tol, k in (("x", got.x, lambda: dz @ wv, lambda: (off @ wv.abs(), dz.abs() @ wv.abs()), dz.shape[1]),
                                    ("w", got.w, lambda: dz.T @ xv, lambda: (off.T @ xv.abs(), dz.abs().T @ xv.abs()), dz.shape[0])):
        if grad is None:
            continue
        ref, (t, size) = ref(), tol()
        within(rows_of(grad), ref, ref.abs() * 2.0 ** -8 + t + product_tol(size, k) + 1e-38, "d" + name)
        # roundings of single operands and of the result, each at most 2^-8 relative and independent: together below 2^-7 of the whole
        assert float((rows_of(grad).to(F64) - ref).norm()) <= 2.0 ** -7 * float(ref.norm()) + 1e-30, name
    if got.bias is not None:
        ref = dz.sum(0)
        within(got.bias, ref, ref.abs() * HALF[got.bias.dtype] + (e.abs() * ACT).sum(0) + 1e-38, "dbias")
    if got.gate is not None:
        v, over = (t.reshape(-1, dyv.shape[0] // (gate.shape[0] if gate.dim() == 2 else 1), dyv.shape[1]).sum(1) for t in (dyv * u, (dyv * u).abs()))
        v, over = v.reshape(gate.shape), over.reshape(gate.shape)
        within(got.gate, v, v.abs() * HALF[got.gate.dtype] + over * ACT + 1e-38, "dgate")
