"""Cases for the operators on token tables and 8-bit rows: what they compute, at which sizes.

Four operators.  "lookup": rows of a token table by token, scaled, with dropout where p > 0,
and "grad": its gradient, summed by token into a dense table gradient.  "dropout": dropout
(and a residual sum) from a counter-based generator, forward and backward.  "cache": rows
quantised to 8 bits as they are written into a cache, then rows of the cache read back.
"product": products of 8-bit rows with a scale for each row of both sides.

Where `own` is false, run() computes them from elementary torch operations in 32 bits; where
it is true, it calls the framework.  exact() computes them from their definition in 64 bits.
"""
import functools
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
          "i32": torch.int32, "i64": torch.int64,
          "int8": torch.int8, "fp8": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}
TOP = {"int8": 127.0, "fp8": 448.0}  # the largest magnitude that 8 bits hold


def _lookup(name=None, **kw):
    return _case("lookup", name, dict(n=1024, rows=32768, dim=512, table="bf16", out="bf16",
                                      tokens="i64", p=0.0, pad=0.0), kw)


def _grad(name=None, **kw):
    return _case("grad", name, dict(n=1024, rows=32768, dim=512, grad="bf16", out="f32",
                                    tokens="i64", p=0.0, pad=0.0), kw)


def _dropout(name=None, **kw):
    return _case("dropout", name, dict(n=1024, dim=512, type="bf16", p=0.1, residual=True), kw)


def _cache(name=None, **kw):
    return _case("cache", name, dict(slots=65536, writes=1024, reads=1024, dim=1024, group=128,
                                     kind="int8", type="bf16", index="i32", pad=0.0), kw)


def _product(name=None, **kw):
    return _case("product", name, dict(m=256, n=4096, k=1024, out="bf16", quantize=False), kw)


def _case(op, name, base, kw):
    c = dict(base, op=op)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # serving: the embedding of one decoded token
        _lookup("lookup-one-token", n=1, dim=1024),
        # training: the embeddings of a step's tokens with their dropout
        _lookup("lookup-16k-d2048-dropout", n=16384, rows=131072, dim=2048, p=0.1),
        # training: the table gradient of a very small step
        _grad("grad-256-d512", n=256, rows=8192, grad="f32"),
        # odd sizes: ragged sequences padded with -1, a dropout in front, 32-bit tokens
        _grad("grad-5003-d1001-padded", n=5003, rows=50_001, dim=1001, p=0.1, pad=0.3,
              tokens="i32"),
        # the largest step: a large table's gradient, a GB of it
        _grad("grad-128k-d2048", n=131072, rows=131072, dim=2048),
        # a small activation of an odd width in 32 bits, as a small model's backward has it
        _dropout("dropout-65x1001-f32", n=65, dim=1001, type="f32", residual=False),
        # a large activation and its residual
        _dropout("dropout-16k-d4096-residual", n=16384, dim=4096),
        # serving: a decode step writes a row for each sequence and reads 500 of each back
        _cache("cache-64-in-32k-out", writes=64, reads=32_000, pad=0.05),
        # prompts: many rows in and out, in 8-bit floats
        _cache("cache-64k-fp8", slots=200_000, writes=65536, reads=65536, kind="fp8"),
        # serving: one token against every row of a table, quantised within the call
        _product("product-one-token-128k", m=1, n=131072, k=2048, quantize=True),
        # a ragged batch against a table of odd size and width
        _product("product-777x10001x1000", m=777, n=10_001, k=1000),
        # a large batch: bound by the matrix cores
        _product("product-8k-16k-4k", m=8192, n=16384, k=4096, quantize=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _dim(rng, hi=4096):
    d = _log_int(rng, 16, hi)
    if rng.random() < 0.25:
        return d | 1
    return d // 2048 * 2048 if d >= 2048 else max(16, d // 32 * 32)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["lookup", "grad", "dropout", "cache", "product"])
        if op == "lookup":
            c = _lookup(n=_log_int(rng, 1, 65536), rows=_log_int(rng, 500, 262_144),
                        dim=_dim(rng), table=rng.choice(["bf16", "f32", "f16"]),
                        out=rng.choice(["bf16", "f32"]), tokens=rng.choice(["i32", "i64"]),
                        p=rng.choice([0.0, 0.0, 0.1, 0.25]), pad=rng.choice([0.0, 0.0, 0.2]))
        elif op == "grad":
            c = _grad(n=_log_int(rng, 1, 131_072), rows=_log_int(rng, 500, 131_072),
                      dim=_dim(rng, 2048), grad=rng.choice(["bf16", "bf16", "f32"]),
                      out=rng.choice(["f32", "f32", "bf16"]), tokens=rng.choice(["i32", "i64"]),
                      p=rng.choice([0.0, 0.0, 0.1]), pad=rng.choice([0.0, 0.0, 0.3]))
        elif op == "dropout":
            c = _dropout(n=_log_int(rng, 1, 16384), dim=_dim(rng),
                         type=rng.choice(["bf16", "f32", "f16"]),
                         p=rng.choice([0.1, 0.1, 0.25, 0.5]), residual=rng.random() < 0.5)
        elif op == "cache":
            heads, width = rng.choice([1, 1, 2, 4, 8, 16]), rng.choice([32, 64, 128, 256, 512])
            slots = _log_int(rng, 1000, 200_000)
            c = _cache(slots=slots, dim=heads * width, group=width,
                       writes=_log_int(rng, 1, min(slots, 65536)), reads=_log_int(rng, 1, 65536),
                       kind=rng.choice(["int8", "int8", "fp8"]),
                       type=rng.choice(["bf16", "bf16", "f32"]), index=rng.choice(["i32", "i64"]),
                       pad=rng.choice([0.0, 0.1]))
        else:
            c = _product(m=_log_int(rng, 1, 8192), n=_log_int(rng, 64, 131_072),
                         k=_dim(rng, 8192), out=rng.choice(["bf16", "bf16", "f32"]),
                         quantize=rng.random() < 0.5)
        if _cost(c) <= 0.9 * most and _held(c) < 6e9:
            return c


# ------------------------------------------------------------------ sizes

@functools.lru_cache(maxsize=4096)
def _touched(n, rows):
    """Expected distinct rows of n draws from the token distribution."""
    p = np.arange(1, rows + 1, dtype=np.float64) ** -1.0
    p /= p.sum()
    return float(-np.expm1(n * np.log1p(-p)).sum())


def work(case):
    c = case
    if c["op"] == "lookup":
        live = c["n"] * (1 - c["pad"])
        rows = _touched(max(1, round(live)), c["rows"])
        return {"bytes": c["n"] * SIZE[c["tokens"]] + rows * c["dim"] * SIZE[c["table"]]
                + c["n"] * c["dim"] * SIZE[c["out"]], "flops": c["n"] * c["dim"]}
    if c["op"] == "grad":
        live = c["n"] * (1 - c["pad"])
        return {"bytes": c["n"] * SIZE[c["tokens"]] + live * c["dim"] * SIZE[c["grad"]]
                + c["rows"] * c["dim"] * SIZE[c["out"]], "flops": 2 * live * c["dim"]}
    if c["op"] == "dropout":
        moved = 2 + bool(c["residual"])
        return {"bytes": moved * c["n"] * c["dim"] * SIZE[c["type"]],
                "flops": 2 * c["n"] * c["dim"]}
    if c["op"] == "cache":
        scales = 4 * (c["dim"] // c["group"])
        size, index = SIZE[c["type"]], SIZE[c["index"]]
        live = c["reads"] * (1 - c["pad"])
        return {"bytes": c["writes"] * (c["dim"] * (size + 1) + scales + index)
                + live * (c["dim"] + scales) + c["reads"] * (c["dim"] * size + index),
                "flops": 3 * c["writes"] * c["dim"] + live * c["dim"]}
    m, n, k = c["m"], c["n"], c["k"]
    given = 2 * m * k if c["quantize"] else m * k + 4 * m
    return {"bytes": given + n * k + 4 * n + m * n * SIZE[c["out"]], "flops": 2 * m * n * k}


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 1e14


def _held(c):
    """Bytes that a state and its plain pass hold, about."""
    if c["op"] in ("lookup", "grad"):
        return 8 * (c["rows"] + c["n"]) * c["dim"]
    if c["op"] == "dropout":
        return 24 * c["n"] * c["dim"]
    if c["op"] == "cache":
        return (c["slots"] + 16 * (c["writes"] + c["reads"])) * c["dim"]
    return 5 * (c["m"] + c["n"]) * c["k"] + 8 * c["m"] * c["n"]


# ------------------------------------------------------------------ inputs

def _padded(rows, dim, dtype):
    """Rows of 8-bit values, each starting at a multiple of 16 bytes."""
    return torch.zeros((rows, (dim + 15) // 16 * 16), dtype=dtype, device="cuda")[:, :dim]


def _tokens(c, g):
    """Tokens by Zipf's law over a permutation of the rows; a share of padding (-1)."""
    w = torch.arange(1, c["rows"] + 1, device="cuda", dtype=torch.float64) ** -1.0
    cdf = w.cumsum(0)
    u = torch.rand(c["n"], generator=g, device="cuda", dtype=torch.float64) * cdf[-1]
    rank = torch.searchsorted(cdf, u).clamp_(max=c["rows"] - 1)
    tok = torch.randperm(c["rows"], generator=g, device="cuda")[rank]
    if c["pad"]:
        gone = torch.rand(c["n"], generator=g, device="cuda") < c["pad"]
        tok = torch.where(gone, torch.full_like(tok, -1), tok)
    return tok.to(DTYPES[c["tokens"]])


def _normal(shape, g, dtype, by=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(by).to(DTYPES[dtype])


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 29)
    s = {"case": c, "seed": (seed * 0x9E3779B97F4A7C15 + 7) % 2 ** 64, "offset": seed % 1000 + 2 ** 33}
    if c["op"] == "lookup":
        s["tokens"] = _tokens(c, g)
        s["table"] = _normal((c["rows"], c["dim"]), g, c["table"], 0.02)
        s["scale"] = math.sqrt(c["dim"])
    elif c["op"] == "grad":
        s["tokens"] = _tokens(c, g)
        s["grad"] = _normal((c["n"], c["dim"]), g, c["grad"], 0.01)
        s["scale"] = math.sqrt(c["dim"])
    elif c["op"] == "dropout":
        s["x"] = _normal((c["n"], c["dim"]), g, c["type"])
        s["residual"] = _normal((c["n"], c["dim"]), g, c["type"]) if c["residual"] else None
    elif c["op"] == "cache":
        S, D, G = c["slots"], c["dim"], c["dim"] // c["group"]
        s["q"] = _padded(S, D, DTYPES[c["kind"]])
        held = torch.randn((S, D), generator=g, device="cuda").mul_(TOP[c["kind"]] / 4)
        held.clamp_(-TOP[c["kind"]], TOP[c["kind"]])
        s["q"].copy_(held.round_() if c["kind"] == "int8" else held)
        s["scales"] = torch.rand((S, G), generator=g, device="cuda").add_(0.5).mul_(0.01)
        index = DTYPES[c["index"]]
        where = torch.randperm(S, generator=g, device="cuda")[:c["writes"]]
        s["to"] = where.to(index)
        spread = torch.exp(torch.randn((c["writes"], 1), generator=g, device="cuda"))
        s["x"] = (torch.randn((c["writes"], D), generator=g, device="cuda") * spread).to(DTYPES[c["type"]])
        at = torch.randint(S, (c["reads"],), generator=g, device="cuda")
        both = min(c["reads"], c["writes"])
        at[:both] = where[:both]  # what was just written is read again
        if c["pad"]:
            gone = torch.rand(c["reads"], generator=g, device="cuda") < c["pad"]
            at = torch.where(gone, torch.full_like(at, -1), at)
        s["at"] = at.to(index)
    else:
        m, n, k = c["m"], c["n"], c["k"]
        s["w"], s["ws"] = _padded(n, k, torch.int8), torch.rand(n, generator=g, device="cuda").add_(0.5).mul_(1e-3)
        s["w"].copy_(torch.randn((n, k), generator=g, device="cuda").mul_(32).clamp_(-127, 127).round_())
        if c["quantize"]:
            s["x"] = _normal((m, k), g, "bf16")
        else:
            s["x"], s["xs"] = _padded(m, k, torch.int8), torch.rand(m, generator=g, device="cuda").add_(0.5).mul_(0.02)
            s["x"].copy_(torch.randn((m, k), generator=g, device="cuda").mul_(32).clamp_(-127, 127).round_())
    return s


# ------------------------------------------------------------------ the framework's calls

def _run_own(s):
    from paper_2205_04702_amd import tokens as tk
    c = s["case"]
    if c["op"] == "lookup":
        return {"rows": tk.lookup(s["tokens"], s["table"], scale=s["scale"], p=c["p"],
                                  seed=s["seed"], offset=s["offset"], dtype=DTYPES[c["out"]])}
    if c["op"] == "grad":
        return {"table_grad": tk.lookup_grad(s["tokens"], s["grad"], c["rows"], scale=s["scale"],
                                             p=c["p"], seed=s["seed"], offset=s["offset"],
                                             dtype=DTYPES[c["out"]])}
    if c["op"] == "dropout":
        return {"y": tk.dropout(s["x"], c["p"], s["seed"], s["offset"], residual=s["residual"])}
    if c["op"] == "cache":
        tk.cache_write(s["q"], s["scales"], s["x"], s["to"])
        rows = tk.cache_read(s["q"], s["scales"], s["at"], dtype=DTYPES[c["type"]])
        return {"rows": rows, "scales": s["scales"]}
    x, xs = tk.quantize(s["x"]) if c["quantize"] else (s["x"], s["xs"])
    return {"scores": tk.product(x, xs, s["w"], s["ws"], dtype=DTYPES[c["out"]])}


# ------------------------------------------------------------------ the plain forms

def _round(state, _):
    """One round of Philox 4x32 on counters held in 64-bit integers."""
    a, b, c, d, k0, k1 = state
    x, y, low = a * 0xD2511F53, c * 0xCD9E8D57, 0xFFFFFFFF
    return ((y >> 32) & low ^ b ^ k0, y & low, (x >> 32) & low ^ d ^ k1, x & low,
            (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low)


def _keep(n, dim, p, seed, offset):
    """The mask of dropout, and the factor of what is kept.  The generator's counter is
    (column / 8, row, offset), its key the seed; its 4 words are 16 bits for each of 8 columns,
    and a column is dropped where they are below 65536 p."""
    drop = int(math.floor(p * 65536 + 0.5))
    octets = (dim + 7) // 8
    a = torch.arange(octets, device="cuda").expand(n, octets)
    b = torch.arange(n, device="cuda")[:, None].expand(n, octets)
    zero = torch.zeros_like(a)
    words = functools.reduce(_round, range(10), (a, b, zero + (offset & 0xFFFFFFFF), zero + (offset >> 32),
                                                 seed & 0xFFFFFFFF, seed >> 32))[:4]
    bits = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=2)
    return bits.reshape(n, octets * 8)[:, :dim] >= drop, 65536.0 / (65536 - drop)


def _dropped(x, p, s):
    if not p:
        return x
    keep, factor = _keep(x.shape[0], x.shape[1], p, s["seed"], s["offset"])
    return torch.where(keep, x * factor, torch.zeros_like(x))


def _quantized(x, kind):
    """Rows of groups in 8 bits: their values and the scale of each group."""
    amax = x.abs().amax(-1, keepdim=True)
    scale = amax * (1.0 / TOP[kind])
    inverse = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    y = x * inverse
    return y.round().clamp(-127, 127).to(torch.int8) if kind == "int8" else y.to(DTYPES["fp8"]), scale


def run(state):
    s = state
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "lookup":
        tok = s["tokens"].long()
        x = s["table"][tok.clamp(min=0)].float() * s["scale"]
        x = torch.where(tok[:, None] >= 0, x, torch.zeros_like(x))
        return {"rows": _dropped(x, c["p"], s).to(DTYPES[c["out"]])}
    if c["op"] == "grad":
        tok = s["tokens"].long()
        x = _dropped(s["grad"].float() * s["scale"], c["p"], s)
        x = torch.where(tok[:, None] >= 0, x, torch.zeros_like(x))
        total = torch.zeros((c["rows"], c["dim"]), device="cuda")
        total.index_add_(0, tok.clamp(min=0), x)
        return {"table_grad": total.to(DTYPES[c["out"]])}
    if c["op"] == "dropout":
        y = _dropped(s["x"].float(), c["p"], s)
        return {"y": (y if s["residual"] is None else y + s["residual"].float()).to(DTYPES[c["type"]])}
    if c["op"] == "cache":
        to, at, groups = s["to"].long(), s["at"].long(), (-1, c["dim"] // c["group"], c["group"])
        q, scale = _quantized(s["x"].float().view(groups), c["kind"])
        s["q"].view(torch.uint8)[to] = q.view(c["writes"], c["dim"]).view(torch.uint8)
        s["scales"][to] = scale[..., 0]
        rows = s["q"].view(torch.uint8)[at.clamp(min=0)].view(DTYPES[c["kind"]]).float()
        rows = rows.view(groups) * s["scales"][at.clamp(min=0)][..., None]
        rows = torch.where(at[:, None] >= 0, rows.view(c["reads"], c["dim"]), torch.zeros((), device="cuda"))
        return {"rows": rows.to(DTYPES[c["type"]]), "scales": s["scales"]}
    x, xs = s["x"].float(), s.get("xs")
    if c["quantize"]:
        q, scale = _quantized(x, "int8")
        x, xs = q.float(), scale[:, 0]
    out = (x @ s["w"].float().t()) * xs[:, None] * s["ws"][None, :]
    return {"scores": out.to(DTYPES[c["out"]])}


# ------------------------------------------------------------------ the definition in 64 bits

def _exact_keep(n, dim, p, s):
    """The mask again, from the generator's definition, on the host in unsigned integers."""
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    octets = (dim + 7) // 8
    c = [np.tile(np.arange(octets, dtype=u), n), np.repeat(np.arange(n, dtype=u), octets),
         np.full(n * octets, s["offset"] % 2 ** 32, u), np.full(n * octets, s["offset"] // 2 ** 32, u)]
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32]
    for _ in range(10):
        left, right = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(right >> u(32)) ^ c[1] ^ u(key[0]), right & low, (left >> u(32)) ^ c[3] ^ u(key[1]), left & low]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    bits = np.empty((n * octets, 8), np.uint16)
    for i, w in enumerate(c):
        bits[:, 2 * i], bits[:, 2 * i + 1] = w & u(0xFFFF), w >> u(16)
    drop = int(math.floor(p * 65536 + 0.5))
    keep = torch.from_numpy(bits.reshape(n, octets * 8)[:, :dim] >= drop).cuda()
    return keep.double() * (65536 / (65536 - drop))


def _exact_q(x, kind):
    """The values that x, rounded to 8 bits by its group's scale, stands for; and the scales."""
    scale = x.abs().amax(-1, keepdim=True) / TOP[kind]
    y = torch.where(scale > 0, x / scale, torch.zeros_like(x))
    step = torch.ones_like(y)
    if kind == "fp8":  # 3 bits after the leading one, and 2^-9 at least
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * scale, scale


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] in ("lookup", "grad"):
        tok = s["tokens"].long()
        live = tok >= 0
        factor = s["scale"] * live.double()[:, None]
        if c["p"]:
            factor = factor * _exact_keep(c["n"], c["dim"], c["p"], s)
        if c["op"] == "lookup":
            return {"rows": s["table"][tok * live].double() * factor}
        total = torch.zeros((c["rows"], c["dim"]), dtype=torch.float64, device="cuda")
        return {"table_grad": total.index_add_(0, tok * live, s["grad"].double() * factor)}
    if c["op"] == "dropout":
        y = s["x"].double() * _exact_keep(c["n"], c["dim"], c["p"], s)
        return {"y": y + s["residual"].double() if c["residual"] else y}
    if c["op"] == "cache":
        groups = (-1, c["dim"] // c["group"], c["group"])
        to, at = s["to"].long(), s["at"].long()
        values, scale = _exact_q(s["x"].double().view(groups), c["kind"])
        scales = s["scales"].double()
        scales[to] = scale[..., 0]
        place = torch.full((c["slots"],), -1, device="cuda")
        place[to] = torch.arange(c["writes"], device="cuda")
        old = s["q"].view(torch.uint8)[at.clamp(min=0)].view(DTYPES[c["kind"]]).double()
        old = old.view(groups) * s["scales"].double()[at.clamp(min=0)][..., None]
        new = place[at.clamp(min=0)]
        rows = torch.where(new[:, None, None] >= 0, values[new.clamp(min=0)], old)
        return {"rows": rows.view(c["reads"], c["dim"]) * (at >= 0).double()[:, None], "scales": scales}
    x = _exact_q(s["x"].double(), "int8")[0] if c["quantize"] else s["x"].double() * s["xs"].double()[:, None]
    return {"scores": x @ (s["w"].double() * s["ws"].double()[:, None]).t()}
