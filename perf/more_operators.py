"""Cases for the operators on rows in 4 bits and on scores: what they compute, at which sizes.

Four operators.  "rows4": rows written into a cache of 4-bit floats with a power of two for
each 32 columns, then rows of the cache read back.  "product4": products of such rows.
"adjust": penalties for repeated tokens, biases and masks on the scores of a vocabulary.
"distill": the loss of scores against a teacher's top logits, with its gradient to the scores
where `grad` is set.

Where `own` is false, run() computes them from elementary torch operations in 32 bits; where
it is true, it calls the framework.  exact() computes them from their definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
          "i32": torch.int32, "i64": torch.int64}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}
BLOCK = 32  # columns that share a scale


def _rows4(name=None, **kw):
    return _case("rows4", name, dict(slots=65536, writes=1024, reads=1024, dim=1024, type="bf16",
                                     index="i32", pad=0.0), kw)


def _product4(name=None, **kw):
    return _case("product4", name, dict(m=256, n=4096, k=1024, out="bf16", quantize=False), kw)


def _adjust(name=None, **kw):
    return _case("adjust", name, dict(n=8, vocab=32768, type="bf16", previous=1000, tokens="i64",
                                      biases=0, mask=False, per_row=False), kw)


def _distill(name=None, **kw):
    return _case("distill", name, dict(n=1024, vocab=32768, k=64, type="bf16", teacher="f32",
                                       tokens="i64", temperature=1.0, pad=0.0, grad=True), kw)


def _case(op, name, base, kw):
    c = dict(base, op=op)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # serving: a decode step writes a row for each sequence and reads 500 of each back
        _rows4("rows4-64-in-32k-out", writes=64, reads=32_000, pad=0.05),
        # a table brought into 4 bits and rows of it read, an odd width, 32-bit inputs
        _rows4("rows4-64k-d1001-f32", slots=100_000, writes=65_536, reads=65_536, dim=1001, type="f32",
               index="i64"),
        # serving: one token against every row of a table, quantised within the call
        _product4("product4-one-token-128k", m=1, n=131072, k=2048, quantize=True),
        # a ragged batch against a table of odd size and width
        _product4("product4-777x10001x1000", m=777, n=10_001, k=1000, out="f32"),
        # a large batch: bound by the matrix cores
        _product4("product4-8k-16k-4k", m=8192, n=16384, k=4096, quantize=True),
        # serving one sequence: the smallest call
        _adjust("adjust-one-row", n=1, previous=300, biases=10, mask=True),
        # a decode step of many sequences with long texts behind them, biases and grammars
        _adjust("adjust-64x131072", n=64, vocab=131072, previous=4096, biases=300, mask=True, per_row=True),
        # odd sizes, 32-bit scores, ragged texts, parameters that differ from row to row
        _adjust("adjust-333x50001-f32", n=333, vocab=50_001, type="f32", previous=1777, tokens="i32",
                per_row=True),
        # training: a very small step
        _distill("distill-16x8192-f32", n=16, vocab=8192, k=16, type="f32"),
        # evaluation: the loss alone
        _distill("distill-2048x131072-loss", n=2048, vocab=131072, grad=False),
        # ragged sequences padded, odd sizes, a temperature
        _distill("distill-777x50001-padded", n=777, vocab=50_001, k=100, type="f32", teacher="bf16",
                 tokens="i32", temperature=2.0, pad=0.3),
        # the largest step: a GB of scores, a GB of gradients
        _distill("distill-4096x131072", n=4096, vocab=131072),
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
        op = rng.choice(["rows4", "product4", "adjust", "distill"])
        if op == "rows4":
            slots = _log_int(rng, 1000, 200_000)
            c = _rows4(slots=slots, dim=_dim(rng), writes=_log_int(rng, 1, min(slots, 65536)),
                       reads=_log_int(rng, 1, 65536), type=rng.choice(["bf16", "bf16", "f32", "f16"]),
                       index=rng.choice(["i32", "i64"]), pad=rng.choice([0.0, 0.1]))
        elif op == "product4":
            c = _product4(m=_log_int(rng, 1, 8192), n=_log_int(rng, 64, 131_072), k=_dim(rng, 8192),
                          out=rng.choice(["bf16", "bf16", "f32"]), quantize=rng.random() < 0.5)
        elif op == "adjust":
            c = _adjust(n=_log_int(rng, 1, 512), vocab=_log_int(rng, 1000, 262_144),
                        type=rng.choice(["bf16", "f32", "f16"]),
                        previous=rng.choice([0, _log_int(rng, 1, 16384), _log_int(rng, 1, 16384)]),
                        tokens=rng.choice(["i32", "i64"]), biases=rng.choice([0, 0, _log_int(rng, 1, 500)]),
                        mask=rng.random() < 0.5, per_row=rng.random() < 0.5)
        else:
            c = _distill(n=_log_int(rng, 1, 8192), vocab=_log_int(rng, 1000, 262_144),
                         k=_log_int(rng, 1, 512), type=rng.choice(["bf16", "f32", "f16"]),
                         teacher=rng.choice(["f32", "bf16"]), tokens=rng.choice(["i32", "i64"]),
                         temperature=rng.choice([1.0, 1.0, 2.0, 4.0]), pad=rng.choice([0.0, 0.0, 0.3]),
                         grad=rng.random() < 0.7)
        if _cost(c) <= 0.9 * most and _held(c) < 6e9:
            return c


# ------------------------------------------------------------------ sizes

def _blocks(dim):
    return (dim + BLOCK - 1) // BLOCK


def _row4(dim):
    """Bytes of a row in 4 bits and of its scales."""
    return _blocks(dim) * (BLOCK // 2 + 1)


def work(case):
    c = case
    if c["op"] == "rows4":
        size, index = SIZE[c["type"]], SIZE[c["index"]]
        return {"bytes": c["writes"] * (c["dim"] * size + _row4(c["dim"]) + index)
                + c["reads"] * ((1 - c["pad"]) * _row4(c["dim"]) + c["dim"] * size + index),
                "flops": 3 * c["writes"] * c["dim"] + c["reads"] * c["dim"]}
    if c["op"] == "product4":
        m, n, k = c["m"], c["n"], c["k"]
        given = 2 * m * k if c["quantize"] else m * _row4(k)
        return {"bytes": given + n * _row4(k) + m * n * SIZE[c["out"]], "flops": 2 * m * n * k}
    if c["op"] == "adjust":
        n, v, tok = c["n"], c["vocab"], SIZE[c["tokens"]]
        return {"bytes": 2 * n * v * SIZE[c["type"]] + n * c["previous"] * tok + c["biases"] * n * (tok + 4)
                + c["mask"] * n * ((v + 31) // 32) * 4, "flops": 4 * n * v}
    live = c["n"] * (1 - c["pad"])  # rows without a teacher need no scores
    size = SIZE[c["type"]]
    return {"bytes": live * c["vocab"] * size + c["grad"] * c["n"] * c["vocab"] * size
            + c["n"] * (c["k"] * (SIZE[c["tokens"]] + SIZE[c["teacher"]]) + 4),
            "flops": live * c["vocab"] * (4 + 4 * c["grad"])}


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 1e14


def _held(c):
    """Bytes that a state and its plain pass hold, about."""
    if c["op"] == "rows4":
        return (c["slots"] + 16 * (c["writes"] + c["reads"])) * c["dim"]
    if c["op"] == "product4":
        return 5 * (c["m"] + c["n"]) * c["k"] + 8 * c["m"] * c["n"]
    if c["op"] == "adjust":
        return 32 * c["n"] * c["vocab"]
    return 6 * c["n"] * c["vocab"]


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 31)
    return g


def _empty4(rows, dim):
    """Bytes and scales of rows in 4 bits: rows of bytes start at multiples of 128 (16 where they
    are short), rows of scales at multiples of 16."""
    width, blocks = _blocks(dim) * 16, _blocks(dim)
    to = 128 if width >= 512 else 16
    q = torch.zeros((rows, (width + to - 1) // to * to), dtype=torch.uint8, device="cuda")
    s = torch.zeros((rows, (blocks + 15) // 16 * 16), dtype=torch.uint8, device="cuda")
    return q[:, :width], s[:, :blocks]


def _some4(rows, dim, g, center):
    """Rows in 4 bits as quantised normal values are: any code, scales around 2^center."""
    q, s = _empty4(rows, dim)
    mag = torch.randn((rows, _blocks(dim) * BLOCK), generator=g, device="cuda").mul_(2.5)
    code = _code4(mag)
    code[:, dim:] = 0
    q.copy_(code[:, 0::2] | code[:, 1::2] << 4)
    s.copy_(torch.randint(center + 126, center + 129, s.shape, generator=g, device="cuda"))
    return q, s


def _zipf(shape, rows, g):
    """Tokens by Zipf's law over a permutation of the rows."""
    w = torch.arange(1, rows + 1, device="cuda", dtype=torch.float64) ** -1.0
    cdf = w.cumsum(0)
    u = torch.rand(shape, generator=g, device="cuda", dtype=torch.float64) * cdf[-1]
    rank = torch.searchsorted(cdf, u).clamp_(max=rows - 1)
    return torch.randperm(rows, generator=g, device="cuda")[rank]


def prepare(case, seed):
    c = case
    g = _gen(seed)
    s = {"case": c}
    if c["op"] == "rows4":
        s["q"], s["scales"] = _some4(c["slots"], c["dim"], g, -2)
        index = DTYPES[c["index"]]
        where = torch.randperm(c["slots"], generator=g, device="cuda")[:c["writes"]]
        s["to"] = where.to(index)
        spread = torch.exp(torch.randn((c["writes"], 1), generator=g, device="cuda"))
        s["x"] = torch.randn((c["writes"], c["dim"]), generator=g, device="cuda").mul_(spread).to(DTYPES[c["type"]])
        at = torch.randint(c["slots"], (c["reads"],), generator=g, device="cuda")
        both = min(c["reads"], c["writes"])
        at[:both] = where[:both]  # what was just written is read again
        if c["pad"]:
            gone = torch.rand(c["reads"], generator=g, device="cuda") < c["pad"]
            at = torch.where(gone, torch.full_like(at, -1), at)
        s["at"] = at.to(index)
    elif c["op"] == "product4":
        m, n, k = c["m"], c["n"], c["k"]
        s["w"], s["ws"] = _some4(n, k, g, -6)
        if c["quantize"]:
            s["x"] = torch.randn((m, k), generator=g, device="cuda").to(torch.bfloat16)
        else:
            s["x"], s["xs"] = _some4(m, k, g, -2)
    elif c["op"] == "adjust":
        n, v, t = c["n"], c["vocab"], DTYPES[c["tokens"]]
        s["scores"] = torch.randn((n, v), generator=g, device="cuda").mul_(3).to(DTYPES[c["type"]])
        s["previous"] = s["bias_tokens"] = s["bias"] = s["allowed"] = s["penalties"] = None
        if c["previous"]:
            length = torch.randint(c["previous"] // 4, c["previous"] + 1, (n, 1), generator=g, device="cuda")
            tok = _zipf((n, c["previous"]), v, g)
            behind = torch.arange(c["previous"], device="cuda")[None, :] >= length
            s["previous"] = torch.where(behind, torch.full_like(tok, -1), tok).to(t)
        if c["biases"]:
            s["bias_tokens"] = torch.randint(v, (n, c["biases"]), generator=g, device="cuda").to(t)
            s["bias"] = torch.randn((n, c["biases"]), generator=g, device="cuda").mul_(4)
        if c["mask"]:  # every other row follows a grammar, which leaves a few tokens
            words = (v + 31) // 32
            bits = torch.rand((n, words, 32), generator=g, device="cuda") < 1 / 64
            bits |= torch.arange(n, device="cuda")[:, None, None] % 2 == 1
            s["allowed"] = (bits.long() << torch.arange(32, device="cuda")).sum(2).to(torch.int32)
        if c["per_row"]:
            u = torch.rand((n, 3), generator=g, device="cuda")
            s["penalties"] = u * torch.tensor([0.5, 1.0, 0.5], device="cuda") + torch.tensor([1.0, 0.0, 0.0], device="cuda")
        s["numbers"] = (1.15, 0.25, 0.125)
    else:
        n, v, k = c["n"], c["vocab"], c["k"]
        s["scores"] = torch.empty((n, v), dtype=DTYPES[c["type"]], device="cuda")
        s["tokens"] = torch.empty((n, k), dtype=DTYPES[c["tokens"]], device="cuda")
        s["teacher"] = torch.empty((n, k), dtype=DTYPES[c["teacher"]], device="cuda")
        for i in range(0, n, 512):  # a teacher that agrees with the student in part
            x = torch.randn((min(512, n - i), v), generator=g, device="cuda").mul_(3)
            s["scores"][i:i + 512] = x
            top = torch.topk(x.add_(torch.randn(x.shape, generator=g, device="cuda"), alpha=2.0), k)
            s["tokens"][i:i + 512], s["teacher"][i:i + 512] = top.indices, top.values
        if c["pad"]:
            gone = torch.rand((n, 1), generator=g, device="cuda") < c["pad"]  # rows behind a sequence
            short = torch.rand((n, k), generator=g, device="cuda") < 0.1
            s["tokens"].masked_fill_(gone | short, -1)
        s["weight"] = torch.rand(n, generator=g, device="cuda").add_(0.5).div_(n)
    return s


# ------------------------------------------------------------------ the framework's calls

def _run_own(s):
    from paper_2205_04702_amd import tokens as tk
    c = s["case"]
    if c["op"] == "rows4":
        tk.cache_write4(s["q"], s["scales"], s["x"], s["to"])
        rows = tk.cache_read4(s["q"], s["scales"], s["at"], c["dim"], dtype=DTYPES[c["type"]])
        return {"rows": rows, "scales": s["scales"]}
    if c["op"] == "product4":
        x, xs = tk.quantize4(s["x"]) if c["quantize"] else (s["x"], s["xs"])
        return {"scores": tk.product4(x, xs, s["w"], s["ws"], dtype=DTYPES[c["out"]])}
    if c["op"] == "adjust":
        r, p, f = s["numbers"]
        return {"scores": tk.adjust(s["scores"], s["previous"], repetition=r, presence=p, frequency=f,
                                    penalties=s["penalties"], bias_tokens=s["bias_tokens"], bias=s["bias"],
                                    allowed=s["allowed"])}
    if not c["grad"]:
        return {"loss": tk.distill(s["scores"], s["tokens"], s["teacher"], c["temperature"])}
    loss, grad = tk.distill_grad(s["scores"], s["tokens"], s["teacher"], s["weight"], c["temperature"])
    return {"loss": loss, "grad": grad}


# ------------------------------------------------------------------ the plain forms

def _code4(y):
    """The codes (sign in bit 3) of the nearest of 0, .5, 1, 1.5, 2, 3, 4 and 6, ties to even
    codes, magnitudes above 6 at 6.  Borders lie half-way; which side they fall on is their code's."""
    a = y.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for border, above in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= border) if above else (a > border)
    return code | torch.signbit(y).to(torch.uint8) << 3


def _values4(q, scales):
    """The values of rows of bytes and scales, in 32 bits."""
    code = torch.stack([q & 15, q >> 4], dim=-1).view(q.shape[0], -1, BLOCK).long()
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    return (table[code] * torch.exp2(scales.float() - 127.0)[..., None]).view(q.shape[0], -1)


def _rows_in_4(x):
    """Bytes and scales of rows of finite values."""
    n, dim = x.shape
    blocks = torch.nn.functional.pad(x.float(), (0, _blocks(dim) * BLOCK - dim)).view(n, -1, BLOCK)
    amax = blocks.abs().amax(2)
    e = torch.where(amax > 0, torch.frexp(amax).exponent - 3, -127).clamp_(min=-127)
    code = _code4(torch.ldexp(blocks, -e[..., None])).view(n, -1)
    return code[:, 0::2] | code[:, 1::2] << 4, (e + 127).to(torch.uint8)


def run(state):
    s = state
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "rows4":
        to, at = s["to"].long(), s["at"].long()
        s["q"][to], s["scales"][to] = _rows_in_4(s["x"])
        rows = _values4(s["q"][at.clamp(min=0)], s["scales"][at.clamp(min=0)])[:, :c["dim"]]
        rows = torch.where(at[:, None] >= 0, rows, torch.zeros((), device="cuda"))
        return {"rows": rows.to(DTYPES[c["type"]]), "scales": s["scales"]}
    if c["op"] == "product4":
        x = _values4(*_rows_in_4(s["x"])) if c["quantize"] else _values4(s["x"], s["xs"])
        return {"scores": (x @ _values4(s["w"], s["ws"]).t()).to(DTYPES[c["out"]])}
    if c["op"] == "adjust":
        return {"scores": _adjusted(s, s["scores"].float()).to(DTYPES[c["type"]])}
    T, tok = c["temperature"], s["tokens"].long()
    z = s["scores"].float() / T
    live = tok >= 0
    t = torch.where(live, s["teacher"].float() / T, float("-inf"))
    some = live.any(1)
    logp = t - torch.logsumexp(t, 1, keepdim=True)
    p = torch.where(live, logp.exp(), torch.zeros((), device="cuda"))
    top = z.amax(1, keepdim=True)
    q = torch.exp(z - top)
    total = q.sum(1, keepdim=True)
    at = z.gather(1, tok.clamp(min=0))
    term = torch.where(live, p * (logp - (at - top - total.log())), torch.zeros((), device="cuda"))
    loss = torch.where(some, term.sum(1) * (T * T), torch.zeros((), device="cuda"))
    if not c["grad"]:
        return {"loss": loss}
    q = (q / total).scatter_add_(1, tok.clamp(min=0), torch.where(live, -p, torch.zeros((), device="cuda")))
    grad = torch.where(some[:, None], q * (s["weight"] * T)[:, None], torch.zeros((), device="cuda"))
    return {"loss": loss, "grad": grad.to(DTYPES[c["type"]])}


def _adjusted(s, x):
    n, v = x.shape
    if s["penalties"] is None:
        r, p, f = s["numbers"]
    else:
        r, p, f = s["penalties"][:, 0:1], s["penalties"][:, 1:2], s["penalties"][:, 2:3]
    if s["previous"] is not None:
        tok = s["previous"].long()
        count = torch.zeros((n, v + 1), device="cuda")
        count.scatter_add_(1, torch.where(tok >= 0, tok, v), torch.ones(tok.shape, device="cuda"))
        count = count[:, :v]
        y = torch.where(x > 0, x / r, x * r) - (p + f * count)
        x = torch.where(count > 0, y, x)
    if s["bias"] is not None:
        tok = s["bias_tokens"].long()  # of several entries for a token the last counts
        last = torch.full((n, v), -1, device="cuda")
        last.scatter_reduce_(1, tok, torch.arange(tok.shape[1], device="cuda").expand(n, -1), "amax")
        x = torch.where(last >= 0, x + s["bias"].gather(1, last.clamp(min=0)), x)
    if s["allowed"] is not None:
        bit = s["allowed"].long()[:, :, None] >> torch.arange(32, device="cuda") & 1
        x = torch.where(bit.view(n, -1)[:, :v] > 0, x, float("-inf"))
    return x


# ------------------------------------------------------------------ the definition in 64 bits

_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_values(q, scales):
    low, high = (q % 16).double(), torch.div(q, 16, rounding_mode="floor").double()
    code = torch.stack([low, high], 2).reshape(q.shape[0], -1)
    m = code % 8  # below 4: halves; above, 1 or 1.5 times a power of two
    big = (1 + 0.5 * (m % 2)) * torch.exp2(torch.floor(m / 2) - 1)
    value = torch.where(m < 2, m / 2, big)
    value = torch.where(code >= 8, -value, value)
    return value * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, 1)


def _exact_rounded(x):
    """The values that rows in 4 bits stand for, and their exponents."""
    n, dim = x.shape
    blocks = torch.zeros((n, _blocks(dim) * BLOCK), dtype=torch.float64, device="cuda")
    blocks[:, :dim] = x.double()
    blocks = blocks.view(n, -1, BLOCK)
    amax = blocks.abs().amax(2, keepdim=True)
    e = torch.floor(torch.log2(amax.clamp(min=2.0 ** -160)))
    e = torch.where(torch.exp2(e) > amax, e - 1, torch.where(torch.exp2(e + 1) <= amax, e + 1, e))
    e = (e - 2).clamp(min=-127.0)
    y = blocks / torch.exp2(e)
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
    y = torch.round(y / step).mul_(step).clamp_(-_MAGNITUDES[-1], _MAGNITUDES[-1])
    return (y * torch.exp2(e)).view(n, -1), (e[..., 0] + 127).to(torch.uint8)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rows4":
        to, at = s["to"].long(), s["at"].long()
        values, scales = _exact_rounded(s["x"])
        place = torch.full((c["slots"],), -1, device="cuda")
        place[to] = torch.arange(c["writes"], device="cuda")
        rows = torch.zeros((c["reads"], c["dim"]), dtype=torch.float64, device="cuda")
        for i in range(0, c["reads"], 16384):
            a = at[i:i + 16384]
            old, new = a.clamp(min=0), place[a.clamp(min=0)]
            part = torch.where(new[:, None] >= 0, values[new.clamp(min=0)],
                               _exact_values(s["q"][old], s["scales"][old]))
            rows[i:i + 16384] = part[:, :c["dim"]] * (a >= 0).double()[:, None]
        s["scales"][to] = scales
        return {"rows": rows, "scales": s["scales"]}
    if c["op"] == "product4":
        x = _exact_rounded(s["x"])[0] if c["quantize"] else _exact_values(s["x"], s["xs"])
        return {"scores": x @ _exact_values(s["w"], s["ws"]).t()}
    if c["op"] == "adjust":
        return {"scores": _exact_adjusted(c, s)}
    T, n = c["temperature"], c["n"]
    loss = torch.zeros(n, dtype=torch.float64, device="cuda")
    grad = torch.zeros((n, c["vocab"]), dtype=torch.float64, device="cuda") if c["grad"] else None
    for i in range(0, n, 256):
        z, tok = s["scores"][i:i + 256].double() / T, s["tokens"][i:i + 256].long()
        live = (tok >= 0).double()
        t = s["teacher"][i:i + 256].double() / T
        up = torch.exp(t - t.max(1, keepdim=True).values) * live
        mass = up.sum(1, keepdim=True)
        some = (mass > 0).double()
        p = up / (mass + (1 - some))
        logq = torch.log_softmax(z, 1)
        logp = torch.log(p + (1 - live))  # (live entries have p > 0 in 64 bits)
        at = logq[torch.arange(z.shape[0], device="cuda")[:, None], tok * (tok >= 0)]
        loss[i:i + 256] = T * T * (p * (logp - at) * live).sum(1)
        if c["grad"]:
            d = torch.exp(logq) * some
            d.scatter_add_(1, tok * (tok >= 0), -p)
            grad[i:i + 256] = d * (T * s["weight"][i:i + 256].double())[:, None]
    return {"loss": loss, "grad": grad} if c["grad"] else {"loss": loss}


def _exact_adjusted(c, s):
    out = torch.empty((c["n"], c["vocab"]), dtype=torch.float64, device="cuda")
    for i in range(c["n"]):
        x = s["scores"][i].double()
        r, p, f = s["numbers"] if s["penalties"] is None else s["penalties"][i].double()
        if s["previous"] is not None:
            tok = s["previous"][i].long()
            count = torch.bincount(tok[tok >= 0], minlength=c["vocab"]).double()
            seen = count > 0
            x = torch.where(seen, torch.where(x > 0, x / r, x * r) - f * count - p, x)
        if s["bias"] is not None:
            tok, b = s["bias_tokens"][i].long(), s["bias"][i].double()
            later = (tok[:, None] == tok[None, :]).triu(1).any(1)  # another entry for it follows
            x[tok[~later]] += b[~later]
        if s["allowed"] is not None:
            v = torch.arange(c["vocab"], device="cuda")
            word = s["allowed"][i].long() & 0xFFFFFFFF
            x = torch.where((word[v // 32] >> (v % 32)) % 2 == 1, x, float("-inf"))
        out[i] = x
    return out
