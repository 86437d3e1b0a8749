"""What the speed of the bf16 half of a layer is measured on: the steps between the attention's products and the attention itself.

A case names one call of one operator:

  rotary       `rotary`: heads turned by their tokens' positions (one axis, or a latent grid's three), from a table of cos and sin that the program keeps, or
               (`build`) that it builds for this clip or context first
  qk           `qk_norm_rotary`: root-mean-square norms of queries and keys, for each head or over a token's heads, and the rotation in the same pass
  qk_grad      `qk_norm_rotary_backward`: the gradients of both inputs and both weights
  linear       `linear`: y = residual + gate * act(x W^T + b), with x W^T + b kept for the backward pass where a program trains
  linear_grad  `linear_backward`: gradients of x, W, b and gate

A pair i of a head of d elements is (2 i, 2 i + 1) (interleaved) or (i, i + P) (half), for i below P; what lies behind 2 P is copied.  Pairs belong to axes in turn: the
table has a row of P pairs (cos, sin) for every position of every axis, the axes' rows below each other, of which a row is filled at its own axis's pairs.
Where `own` is false, `run` computes the operators in elementary torch operations in 32 bits.
"""
import math
from types import SimpleNamespace

import torch

own = False

EPS = 1e-6
BASE = 10000.0
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _turn(op, b, n, h, hk=0, d=128, sizes="21,30,52", pairs="22,21,21", layout="interleaved", x="bf16", norm="", memory="rows", given=False, weight="bf16",
          build=False, scaling="", factor=1.0, original=0, **name):
    """`b` entries of `n` tokens, `h` heads of queries and `hk` of keys (0: of x alone), of `d` elements.  `memory`: "rows" [b, n, heads, d] of the fused projection, "heads"
    [b, heads, n, d].  `given`: positions come as a tensor (random ones below the axis's size) instead of the grid's order."""
    return dict(name, b=b, n=n, h=h, hk=hk, d=d, sizes=sizes, pairs=pairs, layout=layout, x=x, norm=norm, memory=memory, given=given, weight=weight, build=build,
                scaling=scaling, factor=factor, original=original)


def _linear(op, rows, k, n, act="", bias=True, gate=False, residual="", pre=False, batch=1, x="rows", out="rows", head=128, dy="bf16", **name):
    """x [rows, k] (or heads of `head` columns each) by w [n, k]; gate: a vector for each of `batch` entries."""
    return dict(name, op=op, rows=rows, k=k, n=n, act=act, bias=bias, gate=gate, residual=residual, pre=pre, batch=batch, x_layout=x, out_layout=out, head=head, dy=dy)


def _case(op, *args, **kw):
    return _linear(op, *args, **kw) if op.startswith("linear") else dict(_turn(op, *args, **kw), op=op)


def listed():
    # 12 heads of 128: 1536 columns; 7800 tokens are 17 frames of 480p (5 x 30 x 52), 32760 are 81 (21 x 30 x 52)
    return [
        # one new token of each of 16 sequences at its own position: a call whose time is its launch
        _case("rotary", 16, 1, 12, sizes="8192", pairs="64", layout="half", memory="heads", given=True, name="rotary single tokens"),
        # a long sequence behind a context scaled by 8, half of each head turned: the table of its positions, and its queries
        _case("rotary", 1, 65536, 12, sizes="65536", pairs="32", layout="half", build=True, scaling="yarn", factor=8.0, original=8192, name="rotary long scaled"),
        # queries and keys of a 17-frame clip, normed over all heads of a token, from the fused projection into the attention's layout
        _case("qk", 1, 7800, 12, 12, sizes="5,30,52", norm="row", name="qk 17 frames rows"),
        # of an 81-frame clip, normed for each head
        _case("qk", 1, 32760, 12, 12, norm="head", name="qk 81 frames heads"),
        # the same two in training
        _case("qk_grad", 1, 7800, 12, 12, sizes="5,30,52", norm="row", weight="fp32", name="qk gradient 17 frames rows"),
        _case("qk_grad", 1, 32760, 12, 12, norm="head", name="qk gradient 81 frames heads"),
        # the embedding of a timestep for both branches of classifier-free guidance, through its activation
        _case("linear", 2, 1536, 9216, act="silu", name="linear 2 rows"),
        # sizes that no tile divides
        _case("linear", 1001, 1160, 1000, act="gelu", pre=True, name="linear odd"),
        # the first layer of an 81-frame clip's feed-forward half
        _case("linear", 32760, 1536, 6144, act="gelu_tanh", name="linear 81 frames up"),
        # its second layer, gated onto the residual stream
        _case("linear", 32760, 6144, 1536, gate=True, residual="fp32", name="linear 81 frames down"),
        # the first layer's gradients for a 17-frame clip
        _case("linear_grad", 7800, 1536, 6144, act="gelu_tanh", name="linear gradient 17 frames up"),
        # the output projection's, from the attention's layout, two clips with a gate each
        _case("linear_grad", 2 * 7800, 1536, 1536, gate=True, batch=2, x="heads", dy="fp32", name="linear gradient 17 frames out"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


BLOCKS = (1, 2, 3, 4, 5, 6, 8, 9, 10, 12, 13, 16, 20, 22, 27, 32, 40, 45, 48)


def _width(rng, lo, hi):
    """Columns: whole blocks of 128 half of the time, an odd multiple of 8 a third of it, any odd number for the rest."""
    u = rng.random()
    if u < 0.5:
        return 128 * rng.choice([k for k in BLOCKS if lo <= 128 * k <= hi])
    n = _log_int(rng, lo, hi - 16)
    return n // 16 * 16 + 8 if u < 0.83 else n | 1


def _draw_turn(op, rng):
    d = rng.choice((64, 128, 128, 128, 96, 40))
    h = rng.randint(1, 24)
    hk = 0 if op == "rotary" else rng.choice((h, h, max(1, h // 4)))
    b = rng.choice((1, 1, 2, 4))
    n = _log_int(rng, 1, min(65536, 50331648 // (d * (h + hk) * b)))
    kind = rng.choice(("grid", "grid", "line", "part"))
    given = build = False
    scaling, factor, original = "", 1.0, 0
    if kind == "grid":
        t = rng.choice((21, 22, 24)) if d == 128 else d // 6
        rest = d // 2 - t
        pairs, w = "%d,%d,%d" % (t, rest // 2, rest - rest // 2), rng.randint(2, 60)
        hh = rng.randint(1, 34)
        frames = -(-n // (w * hh))
        sizes = "%d,%d,%d" % (frames, hh, w)
    else:
        p = d // 2 if kind == "line" else d // 4
        given = rng.random() < 0.4
        sizes, pairs = str(max(n, 4096) if given else n), str(p)
        build = rng.random() < 0.4 and op == "rotary"
        if build:
            scaling = rng.choice(("", "linear", "ntk", "yarn"))
            factor, original = rng.choice((2.0, 4.0, 16.0)), 4096
    return _case(op, b, n, h, hk, d=d, sizes=sizes, pairs=pairs, layout=rng.choice(("interleaved", "half")), x=rng.choice(("bf16", "bf16", "bf16", "fp32")),
                 norm="" if op == "rotary" else rng.choice(("head", "row")), memory=rng.choice(("rows", "heads")), given=given, weight=rng.choice(("bf16", "fp32")),
                 build=build, scaling=scaling, factor=factor, original=original)


def _draw_linear(op, rng):
    grad = op == "linear_grad"
    head, batch = rng.choice((64, 128)), rng.choice((1, 1, 2))
    x = "heads" if rng.random() < 0.25 else "rows"
    k = rng.randint(2, 20) * head if x == "heads" else _width(rng, 128, 6144)
    out = "heads" if not grad and rng.random() < 0.2 else "rows"
    n = rng.randint(2, 20) * head if out == "heads" else _width(rng, 64, 6144)
    most = 6.0e11 / ((4 if grad else 2) * k * n * batch)
    rows = batch * _log_int(rng, 1, min(65536, 201326592 // max(k, n), most))
    act = rng.choice(("", "", "gelu_tanh", "gelu", "silu", "relu"))
    gate = rng.random() < 0.4
    if grad:
        return _case(op, rows, k, n, act=act, bias=rng.random() < 0.6, gate=gate, batch=batch, x=x, head=head, dy=rng.choice(("bf16", "fp32")))
    return _case(op, rows, k, n, act=act, bias=rng.random() < 0.6, gate=gate, residual="" if out == "heads" else rng.choice(("", "bf16", "fp32")), pre=rng.random() < 0.3, batch=batch,
                 x=x, out=out, head=head)


def draw(rng):
    op = rng.choice(("rotary", "qk", "qk_grad", "linear", "linear", "linear_grad"))
    return _draw_linear(op, rng) if op.startswith("linear") else _draw_turn(op, rng)


# ------------------------------------------------------------------------------------------------ the table of a rotation, plainly
def _ints(text):
    return [int(v) for v in text.split(",")]


def _frequencies(n, c):
    """The angles of one position, of an axis of n pairs, in 64 bits, and the amplitude of its values."""
    i = torch.arange(n, dtype=torch.float64, device="cuda")
    s = c["factor"]
    if c["scaling"] == "ntk":
        return (BASE * s ** (n / (n - 1))) ** (-i / n), 1.0
    f = BASE ** (-i / n)
    if c["scaling"] == "linear":
        return f / s, 1.0
    if c["scaling"] == "yarn":                               # turns over the original context: 1 and fewer are interpolated, 32 and more left alone
        keep = ((c["original"] * f / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
        return f * keep + f / s * (1 - keep), 0.1 * math.log(s) + 1.0
    return f, 1.0


def _table(c):
    """[positions of all axes, pairs, 2] in fp32, from angles in 64 bits (those of far positions are thousands of turns)."""
    sizes, pairs = _ints(c["sizes"]), _ints(c["pairs"])
    table = torch.zeros((sum(sizes), sum(pairs), 2), dtype=torch.float32, device="cuda")
    row = col = 0
    for size, n in zip(sizes, pairs):
        f, amplitude = _frequencies(n, c)
        angle = torch.arange(size, dtype=torch.float64, device="cuda")[:, None] * f
        table[row:row + size, col:col + n, 0] = amplitude * torch.cos(angle)
        table[row:row + size, col:col + n, 1] = amplitude * torch.sin(angle)
        row, col = row + size, col + n
    return table


def _rows_of_axes(c, positions):
    """For each axis the table's row of every token, [b or 1, n]."""
    sizes = _ints(c["sizes"])
    if positions is not None:
        return [positions.long()]
    t = torch.arange(c["n"], device="cuda")
    if len(sizes) == 1:
        return [t[None]]
    frame = sizes[1] * sizes[2]
    return [(t // frame)[None], (sizes[0] + t % frame // sizes[2])[None], (sizes[0] + sizes[1] + t % sizes[2])[None]]


def _factors(c, table, positions):
    """(cos, sin) of every token, [b or 1, 1, n, pairs]."""
    cols, col = [], 0
    for n, rows in zip(_ints(c["pairs"]), _rows_of_axes(c, positions)):
        cols.append(table[rows][:, :, col:col + n])
        col += n
    cs = torch.cat(cols, 2)[:, None]
    return cs[..., 0], cs[..., 1]


def _turned(c, x, cos, sin):
    """x [b, h, n, d] in fp32, its pairs turned."""
    p = cos.shape[-1]
    y = x.clone()
    if c["layout"] == "interleaved":
        a, b = x[..., 0:2 * p:2], x[..., 1:2 * p:2]
        y[..., 0:2 * p:2], y[..., 1:2 * p:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :p], x[..., p:2 * p]
        y[..., :p], y[..., p:2 * p] = a * cos - b * sin, a * sin + b * cos
    return y


# ------------------------------------------------------------------------------------------------ inputs
def _activations(g, rows, width, spread=1.0):
    x = torch.randn((rows, width), generator=g, device="cuda")
    return x * torch.exp(0.5 * torch.randn((width,), generator=g, device="cuda")) * spread


def _heads(x, b, d):
    return x.reshape(b, x.shape[0] // b, -1, d).permute(0, 2, 1, 3)


def _uniform(g, rows, cols):
    return ((2 * torch.rand((rows, cols), generator=g, device="cuda") - 1) * math.sqrt(6.0 / (rows + cols))).to(torch.bfloat16)


def prepare(case, seed):
    """Activations are N(0, 1) with channels of their own spread, as behind a trained layer, the residual stream is twice as wide; weights are Glorot-uniform and those of norms spread
    around 1; gradients are small."""
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)
    s = SimpleNamespace(c=c)

    def vector(n, spread, mean=0.0):
        return mean + spread * torch.randn((n,), generator=g, device="cuda")

    if not c["op"].startswith("linear"):
        b, n, d, h, hk = c["b"], c["n"], c["d"], c["h"], c["hk"]
        fused = _activations(g, b * n, (h + 2 * hk) * d).to(TYPES[c["x"]])       # queries, keys and values lie next to each other
        parts = [_heads(fused[:, :h * d], b, d), _heads(fused[:, h * d:(h + hk) * d], b, d)]
        s.x = [v if c["memory"] == "rows" else v.contiguous() for v in parts[:1 if hk == 0 else 2]]
        if c["norm"]:
            s.w = [vector(d * (v.shape[1] if c["norm"] == "row" else 1), 0.2, 1.0).to(TYPES[c["weight"]]) for v in s.x]
        if c["op"] == "qk_grad":
            s.dy = [(1e-3 * torch.randn(v.shape, generator=g, device="cuda")).to(TYPES[c["x"]]) for v in s.x]
        s.positions = torch.randint(0, _ints(c["sizes"])[0], (b, n), generator=g, device="cuda", dtype=torch.int32) if c["given"] else None
        s.table = None if c["build"] else _table(c)
        return s
    rows, k, n = c["rows"], c["k"], c["n"]
    s.x = _activations(g, rows, k).to(torch.bfloat16)
    if c["x_layout"] == "heads":
        s.x = _heads(s.x, c["batch"], c["head"]).contiguous()
    s.w = _uniform(g, n, k)
    s.bias = vector(n, 0.1).to(torch.bfloat16) if c["bias"] else None
    s.gate = torch.stack([vector(n, 0.3) for _ in range(c["batch"])]) if c["gate"] else None
    if c["op"] == "linear":
        s.residual = _activations(g, rows, n, 2.0).to(TYPES[c["residual"]]) if c["residual"] else None
    else:
        s.dy = (1e-3 * torch.randn((rows, n), generator=g, device="cuda")).to(TYPES[c["dy"]])
        s.pre = _activations(g, rows, n).to(torch.bfloat16) if c["act"] or c["gate"] else None
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _run_own(s):
    import paper_2509_24899_b200 as pkg
    c = s.c
    if c["op"] == "linear":
        out = None
        if c["out_layout"] == "heads":
            out = torch.empty((c["batch"], c["n"] // c["head"], c["rows"] // c["batch"], c["head"]), dtype=torch.bfloat16, device="cuda")
        got = pkg.linear(s.x, s.w, bias=s.bias, activation=c["act"] or None, gate=s.gate, residual=s.residual, out=out, keep_pre=c["pre"])
        return {"y": got[0], "pre": got[1]} if c["pre"] else {"y": got}
    if c["op"] == "linear_grad":
        got = pkg.linear_backward(s.dy, s.x, s.w, pre=s.pre, activation=c["act"] or None, gate=s.gate, bias=s.bias)
        return {name: v for name, v in got._asdict().items() if v is not None}
    sizes, pairs = tuple(_ints(c["sizes"])), tuple(_ints(c["pairs"]))
    table = (s.table, sizes, pairs)
    if c["build"]:
        table = pkg.rotary_table(sizes, pairs, base=BASE, scaling=c["scaling"] or None, factor=c["factor"], original=c["original"])
    if c["op"] == "rotary":
        got = {"x": pkg.rotary(s.x[0], table, layout=c["layout"], positions=s.positions)}
        return dict(got, table=table[0]) if c["build"] else got
    how = dict(norm=c["norm"], eps=EPS, layout=c["layout"], positions=s.positions)
    if c["op"] == "qk":
        q, k = pkg.qk_norm_rotary(s.x[0], s.x[1], s.w[0], s.w[1], table, **how)
        return {"q": q, "k": k}
    got = pkg.qk_norm_rotary_backward(s.dy[0], s.dy[1], s.x[0], s.x[1], s.w[0], s.w[1], table, **how)
    return got._asdict()


def _activated(z, act):
    if act == "gelu_tanh":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z.clamp(min=0) if act == "relu" else z


def _slope(z, act):
    if act == "gelu_tanh":
        a = 2 * math.sqrt(2 / math.pi)
        y = 1 / (1 + torch.exp(-a * (z + 0.044715 * z * z * z)))
        return y + z * y * (1 - y) * a * (1 + 3 * 0.044715 * z * z)
    if act == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "silu":
        y = 1 / (1 + torch.exp(-z))
        return y + z * y * (1 - y)
    return (z > 0).to(z.dtype) if act == "relu" else torch.ones_like(z)


def _rows(x):
    """[batch, heads, tokens, head] as rows [batch * tokens, heads * head]; rows as they are."""
    return x if x.dim() == 2 else x.permute(0, 2, 1, 3).reshape(x.shape[0] * x.shape[2], -1)


def _spread(gate, rows):
    return gate.float().repeat_interleave(rows // gate.shape[0], 0)


def _normed(c, x, w):
    """(x over its root mean square, that root's inverse, the weights laid out like x)."""
    dims = (3,) if c["norm"] == "head" else (1, 3)
    r = torch.rsqrt((x * x).mean(dims, keepdim=True) + EPS)
    return x * r, r, w.float() if c["norm"] == "head" else w.float().reshape(1, -1, 1, x.shape[3])


def run(s):
    if own:
        return _run_own(s)
    c = s.c
    if c["op"] == "linear":
        z = _rows(s.x).float() @ s.w.float().T
        if s.bias is not None:
            z = z + s.bias.float()
        y = _activated(z, c["act"])
        if s.gate is not None:
            y = y * _spread(s.gate, c["rows"])
        if s.residual is not None:
            y = y + s.residual.float()
        y = y.to(TYPES[c["residual"] or "bf16"])
        got = {"y": _heads(y, c["batch"], c["head"]).contiguous() if c["out_layout"] == "heads" else y}
        return dict(got, pre=z.to(torch.bfloat16)) if c["pre"] else got
    if c["op"] == "linear_grad":
        x, dy = _rows(s.x).float(), s.dy.float()
        dz, got = dy, {}
        if s.gate is not None:
            z = s.pre.float()
            got["gate"] = (dy * _activated(z, c["act"])).reshape(c["batch"], -1, c["n"]).sum(1).to(s.gate.dtype)
            dz = dz * _spread(s.gate, c["rows"])
        if c["act"]:
            dz = dz * _slope(s.pre.float(), c["act"])
        if s.bias is not None:
            got["bias"] = dz.sum(0).to(s.bias.dtype)
        dx = (dz @ s.w.float()).to(torch.bfloat16)
        got["x"] = _heads(dx, c["batch"], c["head"]).contiguous() if c["x_layout"] == "heads" else dx
        got["w"] = (dz.T @ x).to(torch.bfloat16)
        return got
    table = _table(c) if c["build"] else s.table
    cos, sin = _factors(c, table, s.positions)
    if c["op"] == "rotary":
        y = _turned(c, s.x[0].float(), cos, sin).to(s.x[0].dtype)
        return {"x": y, "table": table} if c["build"] else {"x": y}
    got = {}
    for i, name in enumerate("qk"):
        x = s.x[i].float()
        n, r, w = _normed(c, x, s.w[i])
        if c["op"] == "qk":
            got[name] = _turned(c, n * w, cos, sin).to(s.x[i].dtype).contiguous()
            continue
        dn = _turned(c, s.dy[i].float(), cos, -sin)
        dims = (3,) if c["norm"] == "head" else (1, 3)
        d = dn * w
        got[name] = (r * (d - n * (d * n).mean(dims, keepdim=True))).to(s.x[i].dtype).contiguous()
        dw = dn * n
        got[name + "_weight"] = (dw.sum((0, 1, 2)) if c["norm"] == "head" else dw.sum((0, 2)).reshape(-1)).to(s.w[i].dtype)
    return got


def work(case):
    """Bytes of the inputs and outputs and operations of the formulas (multiply and add counted as two)."""
    c, size = case, {"": 0, "bf16": 2, "fp32": 4}
    if c["op"].startswith("linear"):
        rows, k, n = c["rows"], c["k"], c["n"]
        small = (2 * n if c["bias"] else 0) + (4 * n * c["batch"] if c["gate"] else 0)
        if c["op"] == "linear":
            out = size[c["residual"] or "bf16"] + size[c["residual"]] + (2 if c["pre"] else 0)
            return {"bytes": 2 * (rows * k + n * k) + rows * n * out + small, "flops": 2 * rows * k * n}
        return {"bytes": 4 * (rows * k + n * k) + rows * n * (size[c["dy"]] + (2 if c["act"] or c["gate"] else 0)) + 2 * small, "flops": 4 * rows * k * n}
    elements = c["b"] * c["n"] * (c["h"] + c["hk"]) * c["d"]
    sizes, pairs = _ints(c["sizes"]), _ints(c["pairs"])
    table = sum(min(s, c["b"] * c["n"]) * p * 8 for s, p in zip(sizes, pairs)) + (4 * c["b"] * c["n"] if c["given"] else 0)
    if c["build"]:
        table = sizes[0] * pairs[0] * 8
    weights = 0 if not c["norm"] else size[c["weight"]] * c["d"] * (c["h"] + c["hk"] if c["norm"] == "row" else 2)
    if c["op"] == "qk_grad":
        return {"bytes": elements * 3 * size[c["x"]] + table + 2 * weights, "flops": 14 * elements}
    return {"bytes": elements * 2 * size[c["x"]] + table + weights, "flops": (3 if c["op"] == "rotary" else 7) * elements}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _angles(c, positions):
    """Each token's rotation as complex numbers [b or 1, 1, n, pairs], from the definition."""
    f64 = torch.float64
    sizes, n = _ints(c["sizes"]), c["n"]
    where = [positions] if positions is not None else None
    if where is None:
        index, where = torch.arange(n, device="cuda"), []
        for size in reversed(sizes):
            where.insert(0, index.remainder(size)[None])
            index = torch.div(index, size, rounding_mode="floor")
    out = []
    for at, pairs in zip(where, _ints(c["pairs"])):
        for i in range(pairs):
            base, turn = BASE, 1.0
            if c["scaling"] == "ntk":
                base *= c["factor"] ** (2 * pairs / (2 * pairs - 2))
            freq = math.exp(-math.log(base) * i / pairs)
            if c["scaling"] == "linear":
                freq /= c["factor"]
            if c["scaling"] == "yarn":
                turns = c["original"] * freq / math.tau
                gamma = min(1.0, max(0.0, (turns - 1) / (32 - 1)))
                freq = (1 - gamma) * freq / c["factor"] + gamma * freq
                turn = 0.1 * math.log(c["factor"]) + 1
            out.append(torch.polar(torch.full_like(at, 1, dtype=f64) * turn, at.to(f64) * freq))
    return torch.stack(out, -1)[:, None]


def _kept(c, table, positions):
    """The same from the table that the call is given."""
    z = torch.complex(table[..., 0].to(torch.float64), table[..., 1].to(torch.float64))
    first, col, cols = 0, 0, []
    sizes = _ints(c["sizes"])
    for a, (size, pairs) in enumerate(zip(sizes, _ints(c["pairs"]))):
        index = positions.long() if positions is not None else (torch.arange(c["n"], device="cuda") // math.prod(sizes[a + 1:]) % size)[None]
        cols.append(z[first + index, col:col + pairs])
        first, col = first + size, col + pairs
    return torch.cat(cols, -1)[:, None]


def _rotate64(c, x, z):
    """x [b, h, n, d] (64 bits) times the complex numbers z."""
    p = z.shape[-1]
    turned, rest = x[..., :2 * p], x[..., 2 * p:]
    if c["layout"] == "interleaved":
        v = torch.view_as_real(torch.view_as_complex(turned.reshape(*turned.shape[:-1], p, 2).contiguous()) * z).flatten(-2)
    else:
        a, b = turned.split(p, -1)
        v = torch.complex(a.contiguous(), b.contiguous()) * z
        v = torch.cat((v.real, v.imag), -1)
    return torch.cat((v, rest), -1)


def _act64(z, act):
    """(value, derivative)"""
    if act == "relu":
        return z.relu(), (z > 0).to(z.dtype)
    if act == "silu":
        sig = torch.sigmoid(z)
        return z * sig, sig * (1 + z * torch.sigmoid(-z))
    if act == "gelu":
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z.square() / 2) / math.sqrt(math.tau)
    if act == "gelu_tanh":
        u = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        half = torch.sigmoid(2 * u)                                              # (1 + tanh u) / 2
        return z * half, half + 2 * z * half * torch.sigmoid(-2 * u) * math.sqrt(2 / math.pi) * (1 + 0.134145 * z.square())
    return z, torch.ones_like(z)


def exact(case, seed):
    """Each output from its formula in 64 bits, unrounded."""
    c, s, f64 = case, prepare(case, seed), torch.float64

    def rows_of(x):
        x = x.to(f64)
        return x if x.dim() == 2 else torch.cat([torch.cat(list(entry), 1) for entry in x])

    def heads_of(y):
        per = c["rows"] // c["batch"]
        return torch.stack([torch.stack(y[i * per:(i + 1) * per].split(c["head"], 1)) for i in range(c["batch"])])

    if c["op"] == "linear":
        w, x, step = s.w.to(f64), rows_of(s.x), 8192
        z = torch.cat([x[r:r + step] @ w.T for r in range(0, c["rows"], step)])
        if s.bias is not None:
            z += s.bias.to(f64)
        y = torch.cat([_act64(z[r:r + step], c["act"])[0] for r in range(0, c["rows"], step)])
        per = c["rows"] // c["batch"]
        if s.gate is not None:
            for i in range(c["batch"]):
                y[i * per:(i + 1) * per] *= s.gate[i].to(f64)
        if s.residual is not None:
            y += s.residual.to(f64)
        got = {"y": heads_of(y) if c["out_layout"] == "heads" else y}
        return dict(got, pre=z) if c["pre"] else got
    if c["op"] == "linear_grad":
        w, x, per = s.w.to(f64), rows_of(s.x), c["rows"] // c["batch"]
        dx, dw, db, dg = [], 0, 0, []
        for i in range(c["batch"]):
            total = 0
            for r in range(i * per, (i + 1) * per, 8192):
                at = slice(r, min(r + 8192, (i + 1) * per))
                dz = s.dy[at].to(f64)
                if s.pre is not None:
                    value, slope = _act64(s.pre[at].to(f64), c["act"])
                    total = total + (dz * value).sum(0)
                    dz = dz * slope
                if s.gate is not None:
                    dz = dz * s.gate[i].to(f64)
                dx.append(dz @ w)
                dw, db = dw + dz.T @ x[at], db + dz.sum(0)
            dg.append(total)
        dx = torch.cat(dx)
        got = {"x": heads_of(dx) if c["x_layout"] == "heads" else dx, "w": dw}
        if s.bias is not None:
            got["bias"] = db
        return dict(got, gate=torch.stack(dg)) if s.gate is not None else got
    if c["build"]:
        z = _angles(c, s.positions)
        y = _rotate64(c, s.x[0].to(f64), z)
        whole = dict(c, n=_ints(c["sizes"])[0])
        return {"x": y, "table": torch.view_as_real(_angles(whole, None)[0, 0])}
    z = _kept(c, s.table, s.positions)
    if c["op"] == "rotary":
        return {"x": _rotate64(c, s.x[0].to(f64), z)}
    got = {}
    for name, x, w, i in (("q", s.x[0], s.w[0], 0), ("k", s.x[1], s.w[1], 1)):
        x = x.to(f64)
        b, h, n, d = x.shape
        scale = w.to(f64).expand(h, d) if c["norm"] == "head" else w.to(f64).reshape(h, d)
        mean = x.square().mean(-1, keepdim=True)
        if c["norm"] == "row":
            mean = mean.mean(1, keepdim=True).expand(b, h, n, 1)
        root = torch.sqrt(mean + EPS)
        if c["op"] == "qk":
            got[name] = _rotate64(c, x / root * scale[None, :, None], z)
            continue
        dn = _rotate64(c, s.dy[i].to(f64), z.conj())
        along = (dn * scale[None, :, None] * x).mean(-1, keepdim=True)
        if c["norm"] == "row":
            along = along.mean(1, keepdim=True)
        got[name] = dn * scale[None, :, None] / root - x * along / root ** 3
        dw = torch.einsum("bhnd,bhnd->hd", dn, x / root)
        got[name + "_weight"] = dw.sum(0) if c["norm"] == "head" else dw.reshape(-1)
    return got
