"""What the speed of the 8-bit projections around the attention is measured on, over the range of layers that they are called for.

A case names one call of one operator:

  norm     `rms_norm`: a row's root-mean-square norm, with the residual's addition in front of it, its output in bf16 (rows, or the
           attention's layout of heads) or in e4m3 with a power-of-two scale for every 128 columns
  quant    `quantize_fp8`: the same 8-bit form of what is there already: an attention's output (a scale for each row and 128 columns),
           or a weight matrix (a scale for each 128 rows and 128 columns)
  matmul   `matmul_fp8`: the product of two matrices in that form, with a bias, as rows or in the attention's layout of heads

Scales are kept as bytes e that stand for 2^(e - 127), in an array [groups of four blocks of 128 columns][rows][4]; bytes of blocks
behind the last column are 0.  Where `own` is false, `run` computes the operators in elementary torch operations in 32 bits.
"""
import math
from types import SimpleNamespace

import torch

own = False

EPS = 1e-6
TOP = 448.0                                                  # the largest e4m3 value


def _case(op, rows, cols, n=0, residual="", x="bf16", out="fp8", layout="rows", batch=1, head=128, block=1, bias=False, pad=0, **name):
    """`rows` x `cols`: the input's (and, for `matmul`, `n` output columns); `pad`: columns that lie between two rows of x."""
    return dict(name, op=op, rows=rows, cols=cols, n=n, residual=residual, x=x, out=out, layout=layout, batch=batch, head=head, block=block,
                bias=bias, pad=pad)


def listed():
    # 12 heads of 128: 1536 columns; 7800 tokens are 17 frames of 480p, 32760 are 81, 63960 are 161
    return [
        # the norm ahead of the projections of one timestep's modulation, a batch of two: a call whose time is its launch
        _case("norm", 2, 1536, name="norm 2 rows"),
        # the norm between attention and feed-forward layer of a 17-frame clip, on a residual stream in bf16
        _case("norm", 7800, 1536, residual="bf16", name="norm 17 frames residual"),
        # the same of an 81-frame clip on a residual stream in fp32
        _case("norm", 32760, 1536, residual="fp32", name="norm 81 frames residual fp32"),
        # the norm of the queries: from a third of the fused projection's rows into the attention's layout, in bf16
        _case("norm", 32760, 1536, out="bf16", layout="heads", pad=2 * 1536, name="norm 81 frames queries"),
        # a width that 128 does not divide, on a stream in fp32 that nothing is added to
        _case("norm", 1001, 1160, x="fp32", name="norm odd"),
        # the 8-bit form of the attention's output, ahead of the output projection
        _case("quant", 32760, 1536, layout="heads", name="quant 81 frames attention"),
        # a projection's weights, when a model is loaded
        _case("quant", 4608, 1536, block=128, name="quant weights"),
        # the modulation of a layer: six vectors from a timestep's embedding, a batch of two
        _case("matmul", 2, 1536, 9216, bias=True, name="matmul 2 rows"),
        # keys of the text that a clip is made from
        _case("matmul", 512, 1536, 1536, bias=True, name="matmul 512 rows"),
        # sizes that no tile divides
        _case("matmul", 1001, 1160, 1000, bias=True, name="matmul odd"),
        # queries, keys and values of an 81-frame clip in one product
        _case("matmul", 32760, 1536, 4608, bias=True, name="matmul 81 frames fused"),
        # values of 161 frames with both branches of classifier-free guidance in the batch, into the attention's layout
        _case("matmul", 2 * 63960, 1536, 1536, layout="heads", batch=2, name="matmul 161 frames cfg values"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


BLOCKS = (1, 2, 3, 4, 5, 6, 8, 9, 10, 12, 13, 16, 20, 22, 27, 32, 40, 45, 48, 56, 64, 72)


def _width(rng, lo, hi):
    """Columns: whole blocks of 128 half of the time, an odd multiple of 8 a third of it, any odd number for the rest."""
    u = rng.random()
    if u < 0.5:
        return 128 * rng.choice([k for k in BLOCKS if lo <= 128 * k <= hi])
    n = _log_int(rng, lo, hi - 16)
    return n // 16 * 16 + 8 if u < 0.83 else n | 1


def draw(rng):
    op = rng.choice(("norm", "norm", "quant", "matmul", "matmul", "matmul"))
    heads = rng.random() < 0.3
    batch, head = rng.choice((1, 1, 2)), rng.choice((64, 128))
    cols = rng.randint(2, 20) * head if heads and op != "matmul" else _width(rng, 128, 6144)
    rows = batch * _log_int(rng, 1, min(65536, 50331648 // cols))
    if op == "norm":
        out = "bf16" if heads else rng.choice(("fp8", "fp8", "bf16"))
        x, residual = rng.choice((("bf16", ""), ("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "")))
        return _case("norm", rows, cols, residual=residual, x=x, out=out, layout="heads" if heads else "rows", batch=batch, head=head,
                     pad=rng.choice((0, 0, 2 * cols)))
    if op == "quant":
        if rng.random() < 0.3:
            return _case("quant", _log_int(rng, 64, 6144), _width(rng, 128, 6144), block=128)
        return _case("quant", rows, cols, layout="heads" if heads else "rows", batch=batch, head=head)
    n = rng.randint(2, 20) * head if heads else _width(rng, 64, 9216)
    most = 6.0e11 / (2 * cols * n)
    rows = batch * _log_int(rng, 1, min(65536, 268435456 // n, most))
    return _case("matmul", rows, cols, n, layout="heads" if heads else "rows", batch=batch, head=head, bias=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ 8-bit form, plainly
def _exponents(amax):
    """The smallest e with amax <= 448 * 2^e, as whole numbers (amax = f * 2^x with f in [1/2, 1), and 448 = 7/8 * 2^9); -127 where all is 0."""
    f, x = torch.frexp(amax)
    return torch.where(amax > 0, x - torch.where(f > 0.875, 8, 9), -127).clamp(-127, 127)


def _scaled(y, block):
    """(quotients, exponents [rows, blocks of 128 columns]) of y [rows, cols], one scale for `block` rows and 128 columns."""
    rows, cols = y.shape
    kb, rb = -(-cols // 128), -(-rows // block)
    full = torch.zeros((rb * block, kb * 128), dtype=y.dtype, device=y.device)
    full[:rows, :cols] = y
    amax = full.reshape(rb, block, kb, 128).abs().amax((1, 3))
    e = _exponents(amax)
    inv = ((127 - e).to(torch.int32) << 23).view(torch.float32)   # 2^-e
    q = full.reshape(rb, block, kb, 128) * inv[:, None, :, None]
    return q.reshape(rb * block, kb * 128)[:rows, :cols], e.repeat_interleave(block, 0)[:rows]


def _packed(e):
    """The bytes of the exponents [rows, blocks] as they are kept: [groups of four blocks][rows][4]."""
    rows, kb = e.shape
    full = torch.zeros((rows, -(-kb // 4) * 4), dtype=torch.uint8, device=e.device)
    full[:, :kb] = (e + 127).to(torch.uint8)
    return full.reshape(rows, -1, 4).permute(1, 0, 2).contiguous()


def _values(q, scales):
    """The matrix that a pair stands for."""
    rows, cols = q.shape
    e = scales.permute(1, 0, 2).reshape(rows, -1)[:, :-(-cols // 128)]
    factor = (e.to(torch.int32) << 23).view(torch.float32)
    return q.float() * factor.repeat_interleave(128, 1)[:, :cols]


def _pitched(q):
    """q as e4m3 whose rows begin on multiples of 16 bytes."""
    rows, cols = q.shape
    t = torch.zeros((rows, -(-cols // 16) * 16), dtype=torch.uint8, device=q.device).view(torch.float8_e4m3fn)
    t[:, :cols] = q.to(torch.float8_e4m3fn)
    return t[:, :cols]


def _rows_of(x):
    """[batch, heads, tokens, head] as rows [batch * tokens, heads * head]; rows as they are."""
    return x if x.dim() == 2 else x.permute(0, 2, 1, 3).reshape(x.shape[0] * x.shape[2], -1)


def _heads_of(y, c):
    return y.reshape(c["batch"], c["rows"] // c["batch"], -1, c["head"]).permute(0, 2, 1, 3).contiguous()


# ------------------------------------------------------------------------------------------------ inputs
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def prepare(case, seed):
    """Activations are N(0, 1) with channels of their own spread, as behind a trained layer; the residual stream is twice as wide; weights are
    Glorot-uniform and the norm's are spread around 1."""
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)
    s = SimpleNamespace(c=c)
    rows, cols = c["rows"], c["cols"]

    def activations(width, spread):
        x = torch.randn((rows, width), generator=g, device="cuda")
        return x * torch.exp(0.5 * torch.randn((width,), generator=g, device="cuda")) * spread

    if c["op"] == "norm":
        x = torch.zeros((rows, cols + c["pad"]), dtype=TYPES[c["x"]], device="cuda")
        s.x = x[:, :cols]
        s.x.copy_(activations(cols, 1.0))
        s.residual = activations(cols, 2.0).to(TYPES[c["residual"]]) if c["residual"] else None
        s.weight = (1.0 + 0.2 * torch.randn((cols,), generator=g, device="cuda")).to(torch.bfloat16)
    elif c["op"] == "quant" and c["block"] == 1:
        x = activations(cols, 1.0).to(torch.bfloat16)
        s.x = _heads_of(x, c) if c["layout"] == "heads" else x
    elif c["op"] == "quant":
        a = math.sqrt(6.0 / (rows + cols))
        s.x = ((2 * torch.rand((rows, cols), generator=g, device="cuda") - 1) * a).to(torch.bfloat16)
    else:
        a = math.sqrt(6.0 / (c["n"] + cols))
        q, e = _scaled(activations(cols, 1.0), 1)
        s.a = (_pitched(q), _packed(e))
        q, e = _scaled((2 * torch.rand((c["n"], cols), generator=g, device="cuda") - 1) * a, 128)
        s.w = (_pitched(q), _packed(e))
        s.bias = (0.1 * torch.randn((c["n"],), generator=g, device="cuda")).to(torch.bfloat16) if c["bias"] else None
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _pair(data, scales):
    return {"data": data, "scales": scales.view(torch.float8_e8m0fnu)}


def _run_own(s):
    from paper_2509_24899_b200 import matmul_fp8, quantize_fp8, rms_norm
    c = s.c
    heads = c["layout"] == "heads"
    if c["op"] == "matmul":
        out = torch.empty((c["batch"], c["n"] // c["head"], c["rows"] // c["batch"], c["head"]), dtype=torch.bfloat16, device="cuda") if heads else None
        return matmul_fp8(s.a, s.w, bias=s.bias, out=out)
    if c["op"] == "quant":
        return _pair(*quantize_fp8(s.x, block_rows=c["block"]))
    out = torch.empty((c["batch"], c["cols"] // c["head"], c["rows"] // c["batch"], c["head"]), dtype=torch.bfloat16, device="cuda") if heads else None
    got = rms_norm(s.x, s.weight, residual=s.residual, eps=EPS, fp8=c["out"] == "fp8", out=out)
    y, total = got if s.residual is not None else (got, None)
    y = _pair(*y) if c["out"] == "fp8" else {"y": y}
    return y if total is None else dict(y, residual=total)


def run(s):
    if own:
        return _run_own(s)
    c = s.c
    heads = c["layout"] == "heads"
    if c["op"] == "matmul":
        y = _values(*s.a) @ _values(*s.w).T
        if s.bias is not None:
            y = y + s.bias.float()
        y = y.to(torch.bfloat16)
        return _heads_of(y, c) if heads else y
    if c["op"] == "quant":
        q, e = _scaled(_rows_of(s.x).float(), c["block"])
        return _pair(q.to(torch.float8_e4m3fn), _packed(e))
    t = s.x.float() if s.residual is None else s.x.float() + s.residual.float()
    y = t * torch.rsqrt((t * t).mean(1, keepdim=True) + EPS) * s.weight.float()
    if c["out"] == "fp8":
        q, e = _scaled(y, 1)
        got = _pair(q.to(torch.float8_e4m3fn), _packed(e))
    else:
        got = {"y": _heads_of(y.to(torch.bfloat16), c) if heads else y.to(torch.bfloat16)}
    return got if s.residual is None else dict(got, residual=t.to(s.residual.dtype))


def work(case):
    """Bytes of the inputs and outputs and operations of the formulas (multiply and add counted as two)."""
    c = case
    rows, cols, size = c["rows"], c["cols"], {"": 0, "bf16": 2, "fp32": 4, "fp8": 1}
    if c["op"] == "matmul":
        table = lambda m: m * cols + m * -(-cols // 128)     # noqa: E731
        return {"bytes": table(rows) + table(c["n"]) + 2 * rows * c["n"] + (2 * c["n"] if c["bias"] else 0), "flops": 2 * rows * cols * c["n"]}
    scales = rows * -(-cols // 128) if c["out"] == "fp8" else 0
    if c["op"] == "quant":
        return {"bytes": rows * cols * 3 + scales, "flops": 2 * rows * cols}
    per = size[c["x"]] + 2 * size[c["residual"]] + size[c["out"]]
    return {"bytes": rows * cols * per + 2 * cols + scales, "flops": (6 if c["residual"] else 5) * rows * cols}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """Each output from its formula in 64 bits, unrounded: an 8-bit value as the quotient that it is the nearest of, a scale as the power of two."""
    c, s, f64 = case, prepare(case, seed), torch.float64
    rows, cols = c["rows"], c["cols"]
    kb = -(-cols // 128)

    def power(e):
        return ((e.to(torch.int64) + 1023) << 52).view(f64)  # 2^e without a rounding

    def blocks(y, height):
        """y over its blocks' scales, and the scales, laid out as `run` returns them."""
        q = torch.empty_like(y)
        scale = torch.zeros((-(-kb // 4), rows, 4), dtype=f64, device="cuda") + 2.0 ** -127
        for k in range(kb):
            part = y[:, 128 * k:128 * k + 128]
            top = part.abs().amax(1)
            if height > 1:
                for r in range(0, rows, height):
                    top[r:r + height] = top[r:r + height].max()
            e = torch.round(torch.log2(top.clamp(min=1e-300) / TOP))
            e = torch.where(top > TOP * power(e), e + 1, e).clamp(min=-127)          # a quotient near a power of two may round to either side of it
            q[:, 128 * k:128 * k + 128] = part / power(e)[:, None]
            scale[k // 4, :, k % 4] = power(e)
        return {"data": q, "scales": scale}

    if c["op"] == "matmul":
        def value(pair):
            v = pair[0].to(f64)
            for k in range(kb):
                v[:, 128 * k:128 * k + 128] *= power(pair[1][k // 4, :, k % 4].to(f64) - 127)[:, None]
            return v

        w = value(s.w)
        y = torch.cat([value((s.a[0][r:r + 16384], s.a[1][:, r:r + 16384])) @ w.T for r in range(0, rows, 16384)])
        if s.bias is not None:
            y += s.bias.to(f64)
    else:
        x = s.x.to(f64)
        if x.dim() == 4:
            x = torch.cat([torch.cat([x[b, h] for h in range(x.shape[1])], 1) for b in range(x.shape[0])])
        if c["op"] == "quant":
            return blocks(x, c["block"])
        t = x if s.residual is None else x + s.residual.to(f64)
        y = t / torch.sqrt(t.square().sum(1, keepdim=True) / cols + EPS) * s.weight.to(f64)
        if c["out"] == "fp8":
            got = blocks(y, 1)
            return got if s.residual is None else dict(got, residual=t)
    if c["layout"] == "heads":
        n, h, per = y.shape[1], c["head"], rows // c["batch"]
        y = torch.stack([torch.stack([y[b * per:(b + 1) * per, i:i + h] for i in range(0, n, h)]) for b in range(c["batch"])])
    if c["op"] == "matmul":
        return y
    return {"y": y} if s.residual is None else {"y": y, "residual": t}
