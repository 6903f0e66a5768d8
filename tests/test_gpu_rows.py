"""The operators on token tables and 8-bit rows against plain implementations in 64 bits.

Bounds: with U = 2^-24 (a rounding to fp32) and u, t half a unit and half the smallest number
of the output's type, a value computed by r roundings to fp32 and rounded once is within
|exact| ((1 + U)^r (1 + u) - 1) + t of the exact one, taken as |exact| (u + (r + 1) U) + t; a sum of c terms
of magnitudes adding up to S is within c U S of the exact sum in any order."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2205_04702_amd import scratchpipe as sp  # noqa: E402
from paper_2205_04702_amd import tokens as tk  # noqa: E402
from tests import rows_reference as ref  # noqa: E402
from tests.rows_reference import TINY, U32, UNIT  # noqa: E402

F32, BF16, F16, F8 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def near(got, want, bound):
    """Every element within its bound (float64 tensors on the CPU)."""
    got = got.double().cpu().reshape(want.shape)
    off = (got - want).abs() - bound
    assert not torch.isnan(off).any(), "NaN"
    assert off.max().item() <= 0 if off.numel() else True, off.max().item()


def rounded(want, dtype, r):
    return want.abs() * (UNIT[dtype] + (r + 1) * U32) + TINY[dtype]


def randn(shape, seed, dtype=F32, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * by).to(dtype)


def some_tokens(n, rows, seed, dtype=torch.int64, pad=0.2, hot=0.3):
    """Uniform tokens, some of them no rows (negative, the first past the table, far away), a
    share of them one hot token."""
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(max(rows, 1), (n,), generator=g)
    u = torch.rand(n, generator=g)
    t = torch.where(u < hot, torch.full_like(t, rows // 2), t)
    far = torch.tensor([-1, -2 ** 31, rows, 2 ** 31 - 1])[torch.randint(4, (n,), generator=g)]
    if dtype == torch.int64:
        far = torch.where(u < hot + pad / 2, far * 2 ** 20 - 1, far)
        far = torch.where((far >= 0) & (far < rows), torch.full_like(far, -1), far)
    return torch.where((u >= hot) & (u < hot + pad), far, t).to(dtype)


# ------------------------------------------------------------------ lookup

@pytest.mark.parametrize("n,dim,rows,table,out,idx,p", [
    (1, 1024, 1000, BF16, BF16, torch.int64, 0.0),
    (1, 1, 1, F32, F32, torch.int32, 0.0),
    (7, 5, 3, F16, F32, torch.int64, 0.5),
    (130, 33, 77, BF16, F32, torch.int32, 0.1),
    (64, 8, 500, F32, BF16, torch.int64, 0.0),
    (33, 1001, 50, F32, F16, torch.int64, 0.25),
    (5, 9000, 20, BF16, BF16, torch.int32, 0.1),
    (600, 64, 4096, F16, F16, torch.int64, 0.0),
    (300, 96, 0, F32, F32, torch.int64, 0.0),
])
def test_lookup(n, dim, rows, table, out, idx, p):
    tok, w = some_tokens(n, rows, 1, idx), randn((rows, dim), 2, table)
    seed, off = 0x123456789ABCDEF1, 2 ** 40 + 5
    got = tk.lookup(tok.cuda(), w.cuda(), 3.7, p, seed, off, dtype=out)
    assert got.shape == (n, dim) and got.dtype == out
    want = ref.lookup(tok, w, 3.7, p, seed, off)
    assert torch.equal(got.cpu() == 0, want.to(out) == 0)  # the mask and the padding
    near(got, want, rounded(want, out, 2))


def test_lookup_many_octets_and_strides():
    """Enough octets for the deep form; a table, output and tokens with strides and odd starts."""
    n, dim, rows = 40_000, 421, 3000
    base = randn((rows, 2 * dim + 1), 3, BF16).cuda()
    w = base[:, dim:2 * dim]
    tok = some_tokens(2 * n, rows, 4).cuda()[::2]
    buf = torch.full((n, dim + 3), 9.0, dtype=BF16, device="cuda")
    got = tk.lookup(tok, w, out=buf[:, 1:1 + dim])
    t = tok.cpu()
    live = (t >= 0) & (t < rows)
    want = torch.where(live[:, None], w.cpu()[t.clamp(0, rows - 1)], torch.zeros((), dtype=BF16))
    assert torch.equal(got.cpu(), want)
    assert (buf[:, :1] == 9).all() and (buf[:, 1 + dim:] == 9).all()


def test_lookup_of_rows_past_32_bits():
    """A table whose elements pass 2^32, and shapes of more dimensions."""
    rows, dim = 1_060_000, 4104
    w = torch.empty((rows, dim), dtype=BF16, device="cuda")
    at = [0, rows // 2, rows - 1]
    for i, r in enumerate(at):
        w[r] = float(i + 1)
    got = tk.lookup(torch.tensor([[at[2], at[0]], [at[1], -1]], device="cuda"), w)
    assert got.shape == (2, 2, dim)
    for (i, j), v in {(0, 0): 3, (0, 1): 1, (1, 0): 2, (1, 1): 0}.items():
        assert (got[i, j] == v).all()
    g = torch.ones((3, dim), device="cuda", dtype=BF16)
    w.zero_()
    tk.lookup_grad(torch.tensor(at, device="cuda"), g, rows, 2.0, out=w, accumulate=True)
    for r in at:
        assert (w[r] == 2).all()
    assert int(torch.count_nonzero(w[rows // 2 - 1]) + torch.count_nonzero(w[1])) == 0


# ------------------------------------------------------------------ gradient

def grad_bound(size, count, want, dtype, base=None):
    """c terms of a sum, the factor and the base's addition, then the output's rounding."""
    b = size * (count + 3) * U32 + rounded(want, dtype, 1)
    return b if base is None else b + base.abs() * 2 * U32


@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 300, 512, 513, 1500, 8192, 8193, 20_000])
@pytest.mark.parametrize("dim,grad,out", [(16, F32, F32), (33, BF16, F32), (300, F16, BF16)])
def test_grad_lengths(n, dim, grad, out):
    rows = 700
    tok, g = some_tokens(n, rows, 5), randn((n, dim), 6, grad)
    got = tk.lookup_grad(tok.cuda(), g.cuda(), rows, 0.3, dtype=out)
    want, size, count = ref.lookup_grad(tok, g, rows, 0.3)
    near(got, want, grad_bound(size, count, want, out))


@pytest.mark.parametrize("n,dim,rows,idx,p", [
    (200, 1001, 1, torch.int32, 0.1),         # every live token in one row
    (3000, 1, 5, torch.int64, 0.5),
    (3000, 1030, 3_000, torch.int32, 0.1),    # more than one slab of columns
    (40_000, 8, 100_000, torch.int64, 0.0),   # many rows, few of them used
    (30_000, 4, 2_000_000, torch.int32, 0.1),  # three digits of the sort
    (9_000, 40, 511, torch.int32, 0.0),       # one digit
    (9_000, 24, 512, torch.int64, 0.0),       # two
    (300_000, 4, 3_000, torch.int32, 0.0),    # more tiles than a tile adds up itself
])
def test_grad_shapes(n, dim, rows, idx, p):
    tok, g = some_tokens(n, rows, 7, idx), randn((n, dim), 8, BF16)
    seed, off = 99, 1
    if p and n * dim > 400_000:  # (the reference draws its mask in Python)
        tok[400_000 // dim:] = -1
    got = tk.lookup_grad(tok.cuda(), g.cuda(), rows, 1.5, p, seed, off)
    few = min(n, 400_000 // dim) if p else n
    want, size, count = ref.lookup_grad(tok[:few], g[:few], rows, 1.5, p, seed, off)
    near(got, want, grad_bound(size, count, want, F32))


@pytest.mark.parametrize("n", [100, 512, 4_000, 50_000])
@pytest.mark.parametrize("what", ["one", "sorted", "padding", "pairs"])
def test_grad_runs(n, what):
    """Runs of every kind: one token only, rows in order, nothing but padding, runs of two."""
    rows, dim = 30_000, 72
    tok = {"one": torch.full((n,), 17), "sorted": torch.arange(n) % rows,
           "padding": torch.full((n,), -1), "pairs": torch.arange(n) // 2 % rows}[what]
    g = randn((n, dim), 9, BF16)
    got = tk.lookup_grad(tok.cuda(), g.cuda(), rows)
    want, size, count = ref.lookup_grad(tok, g, rows)
    near(got, want, grad_bound(size, count, want, F32))


@pytest.mark.parametrize("n", [40, 3000, 10_000])
@pytest.mark.parametrize("out", [F32, BF16])
def test_grad_is_added(n, out):
    """accumulate: rows without a token keep their bits, NaN included; strides of the output
    are kept to; the same call twice gives the same bits."""
    rows, dim = 5000, 50
    tok, g = some_tokens(n, 900, 10), randn((n, dim), 11, BF16)
    base = randn((rows, dim + 6), 12, out)
    base[3000:] = float("nan")
    results = []
    for _ in range(2):
        buf = base.cuda()
        tk.lookup_grad(tok.cuda(), g.cuda(), rows, 2.0, out=buf[:, 3:3 + dim], accumulate=True)
        results.append(buf.cpu())
    assert torch.equal(results[0].nan_to_num(7.5), results[1].nan_to_num(7.5))
    want, size, count = ref.lookup_grad(tok, g, rows, 2.0)
    used = count[:, 0] > 0
    b = base[:, 3:3 + dim].double()
    near(results[0][used, 3:3 + dim], (b + want)[used],
         grad_bound(size, count, b + want, out, b)[used])
    kept = results[0].clone()
    kept[used, 3:3 + dim] = base[used, 3:3 + dim]
    assert torch.equal(kept.nan_to_num(7.5), base.nan_to_num(7.5))


def test_grad_ignores_what_padding_holds():
    """NaN and infinities in the gradients of padding, and in dropped places, go nowhere."""
    n, dim, rows, seed = 700, 40, 100, 5
    tok = some_tokens(n, rows, 13, pad=0.3)
    g = randn((n, dim), 14)
    gone = ~((tok >= 0) & (tok < rows))
    keep = ref.keep_mask(n, dim, 0.5, seed, 0)
    dirty = torch.where(keep & ~gone[:, None], g, torch.tensor([float("nan"), float("inf")]).repeat(20))
    for k in (n, 400):
        got = tk.lookup_grad(tok[:k].cuda(), dirty[:k].cuda(), rows, 1.0, 0.5, seed)
        want, size, count = ref.lookup_grad(tok[:k], g[:k], rows, 1.0, 0.5, seed)
        near(got, want, grad_bound(size, count, want, F32))


def test_grad_of_expanded_gradients():
    """The gradient of a plain sum is one broadcast number."""
    tok = some_tokens(600, 50, 15)
    one = torch.ones((), device="cuda").expand(600, 24)
    got = tk.lookup_grad(tok.cuda(), one, 50)
    assert torch.equal(got.cpu(), ref.lookup_grad(tok, torch.ones(600, 24), 50)[0].float())
    row = torch.arange(24.0, device="cuda").expand(600, 24)  # one row for all
    got = tk.lookup_grad(tok.cuda(), row, 50)
    assert torch.equal(got.cpu(), ref.lookup_grad(tok, row.cpu(), 50)[0].float())


@pytest.mark.parametrize("n", [200, 2000, 12_000])
def test_grad_agrees_with_differences(n):
    """(L(W + hE) - L(W - hE)) / 2h of L(W) = sum of C * lookup(W) is the gradient's entry; the
    lookup is linear, so only its rounding is left: at most 2 U |out| per output and side."""
    rows, dim, h, p = 60, 20, 0.25, 0.3
    tok = some_tokens(n, rows, 16).cuda()
    w, c = randn((rows, dim), 17).cuda(), randn((n, dim), 18).cuda()
    got = tk.lookup_grad(tok, c, rows, 1.7, p, 3, 4).double()

    def loss(x):
        out = tk.lookup(tok, x, 1.7, p, 3, 4).double()
        return (out * c.double()).sum().item(), (out * c.double()).abs().sum().item()
    hot = (rows // 2, rows // 2, 0, rows - 1)
    for r, d in zip(hot, (0, dim - 1, 3, 7)):
        up, down = w.clone(), w.clone()
        up[r, d] += h
        down[r, d] -= h
        h2 = up[r, d].double().item() - down[r, d].double().item()
        (a, sa), (b, sb) = loss(up), loss(down)
        of_grad = ref.lookup_grad(tok.cpu(), c.cpu(), rows, 1.7, p, 3, 4)
        bound = 3 * U32 * (sa + sb) / h2 + grad_bound(*(x[r] for x in of_grad[1:]), of_grad[0][r], F32)[d].item()
        assert abs((a - b) / h2 - got[r, d].item()) <= bound


# ------------------------------------------------------------------ dropout

@pytest.mark.parametrize("n,dim,dtype,p,res", [
    (1, 1, F32, 0.5, False), (1, 2000, BF16, 0.1, True), (65, 101, F32, 0.1, False),
    (17, 8, F16, 0.9, True), (3, 4100, BF16, 0.5, False), (40, 64, F32, 0.25, True),
    (9, 7, BF16, 0.0, True), (2, 33, F32, 1 - 2.0 ** -16, False),
])
def test_dropout(n, dim, dtype, p, res):
    x, r = randn((n, dim), 20, dtype), randn((n, dim), 21, dtype)
    seed, off = 2 ** 64 - 3, 2 ** 63 + 1
    got = tk.dropout(x.cuda(), p, seed, off, residual=r.cuda() if res else None)
    y = ref.drop(x.double(), p, seed, off)
    want = y + r.double() if res else y
    # factor and product, then the sum with the residual
    near(got, want, y.abs() * 3 * U32 + rounded(want, dtype, 1))
    if not res:
        assert torch.equal(got.cpu() == 0, (want == 0) | (want.to(dtype) == 0))


def test_dropout_backward_agrees_with_differences():
    """y is linear in x: the call on C gives the gradient of sum(C * y), element by element."""
    n, dim, p, h = 6, 37, 0.4, 0.5
    x, c = randn((n, dim), 22).cuda(), randn((n, dim), 23).cuda()
    dx = tk.dropout(c, p, 11, 12).double().cpu()
    y0 = tk.dropout(x, p, 11, 12).double()
    moved = x + h
    step = moved.double() - x.double()
    slope = ((tk.dropout(moved, p, 11, 12).double() - y0) / step * c.double()).cpu()
    # two roundings of y on each side, divided by the step; two of dx
    bound = 4 * U32 * (y0.abs().cpu() + 2 * h) / step.cpu() * c.abs().double().cpu() + 3 * U32 * dx.abs() + 1e-30
    near(slope, dx, bound)


def test_dropout_in_place_strided_and_masked_infinities():
    n, dim, p = 300, 61, 0.5
    x = randn((n, dim), 24)
    keep = ref.keep_mask(n, dim, p, 1, 2)
    x = torch.where(keep, x, torch.tensor(float("inf")))
    buf = torch.full((n, dim + 9), 5.0)
    buf[:, 4:4 + dim] = x
    buf = buf.cuda()
    view = buf[:, 4:4 + dim]
    res = randn((n, dim), 25).cuda()
    want = ref.drop(torch.where(keep, x, torch.zeros(())).double(), p, 1, 2)
    got = tk.dropout(view, p, 1, 2, residual=res, out=res)
    assert got is res
    assert torch.isfinite(res).all()
    tk.dropout(view, p, 1, 2, out=view)
    near(view, want, rounded(want, F32, 2))
    assert (buf[:, :4] == 5).all() and (buf[:, 4 + dim:] == 5).all()


def test_dropout_shares_the_lookup_s_mask_and_large_matrices_agree_in_parts():
    """lookup's dropout is dropout's; the deep form (many octets) draws what the shallow does."""
    n, dim, p = 5000, 4096, 0.1
    x = torch.ones((n, dim), dtype=BF16, device="cuda")
    big = tk.dropout(x, p, 77, 3)
    assert torch.equal(big[:50], tk.dropout(x[:50], p, 77, 3))
    tok = torch.zeros(n, dtype=torch.int64, device="cuda")
    assert torch.equal(big, tk.lookup(tok, x[:1], 1.0, p, 77, 3))
    share = (big != 0).double().mean().item()
    assert abs(share - 0.9) < 5 * (0.09 / (n * dim)) ** 0.5 + 2.0 ** -17
    assert not torch.equal(big, tk.dropout(x, p, 77, 4))
    wide = torch.ones((1, 3_000_001), device="cuda")
    assert torch.equal(tk.dropout(wide, p, 77, 3)[0, :5000], tk.dropout(wide[:, :5000], p, 77, 3)[0])


# ------------------------------------------------------------------ cache

CACHE_SHAPES = [(1, 1024, 128), (3, 1, 1), (50, 24, 8), (33, 101, 101), (64, 96, 32), (9, 1000, 1000),
                (5, 2048, 256), (7, 2050, 2050), (3, 9000, 9000), (2, 5000, 5000), (40, 512, 512),
                (600, 64, 64), (2, 16384, 8192)]


@pytest.mark.parametrize("kind", [torch.int8, F8])
@pytest.mark.parametrize("n,dim,group", CACHE_SHAPES)
def test_cache_write_and_read(n, dim, group, kind):
    """Values within half a step of their group's scale of what was written: the bytes are the
    nearest, up to the 4 U that scale and product carry; scales within 2 U."""
    slots = n + 20
    dtype, idx = (BF16, torch.int32) if n % 2 else (F32, torch.int64)
    x = randn((n, dim), 30, dtype) * torch.exp(randn((n, 1), 31)).to(dtype)
    at = torch.randperm(slots, generator=torch.Generator().manual_seed(32))[:n].to(idx)
    q, s = tk.empty_cache(slots, dim, group, kind)
    q.view(torch.uint8).fill_(3)
    s.fill_(5.0)
    tk.cache_write(q, s, x.cuda(), at.cuda())
    scale = ref.group_scales(x, group, kind)
    got_s = s.cpu()[at.long()].double()
    assert ((got_s - scale).abs() <= 2 * U32 * scale).all()
    wide = scale.repeat_interleave(group, 1)
    y = x.double() / wide
    byte = q.cpu()[at.long()].double()
    if kind == torch.int8:
        half = torch.full_like(y, 0.5)
    else:  # half of the step at the value's, or the byte's, binary place, the coarser one
        big = torch.maximum(y.abs(), byte.abs()).clamp(min=2.0 ** -6)
        half = torch.exp2(torch.floor(torch.log2(big))) / 16
    assert ((byte - y).abs() <= half + 4 * U32 * y.abs()).all()
    others = torch.ones(slots, dtype=torch.bool)
    others[at.long()] = False
    assert (q.view(torch.uint8).cpu()[others] == 3).all() and (s.cpu()[others] == 5).all()
    back = torch.cat([at, at.new_tensor([-1, slots])])
    for out in (F32, BF16, F16):
        got = tk.cache_read(q, s, back.cuda(), dtype=out)
        assert (got[n:] == 0).all()
        want = byte * got_s.repeat_interleave(group, 1)
        near(got[:n], want, rounded(want, out, 1))


@pytest.mark.parametrize("kind", [torch.int8, F8])
def test_cache_of_odd_values(kind):
    """Zeros, one value, NaN and infinities in one group only, subnormal scales, the type's
    largest values; rows without a slot are not read."""
    q, s = tk.empty_cache(16, 64, 32, kind)
    x = torch.zeros((8, 64))
    x[1, 5] = -3.0
    x[2, 1] = float("nan")
    x[2, 40] = 2.0
    x[3, 33] = float("-inf")
    x[3, 2] = 1.0
    x[4] = 1e-38
    x[5] = 3e38
    x[6] = float("nan")  # no slot
    x[7, :] = torch.linspace(-1, 1, 64)
    at = torch.tensor([0, 1, 2, 3, 4, 5, -1, 7], dtype=torch.int32)
    tk.cache_write(q, s, x.cuda(), at.cuda())
    got = tk.cache_read(q, s, at.cuda(), dtype=F32).cpu()
    assert (got[0] == 0).all() and (got[6] == 0).all() and (got[4] == 0).all()
    assert abs(got[1, 5].item() + 3.0) <= 3.0 * 3 * U32 and (got[1, :5] == 0).all() and (got[1, 6:] == 0).all()
    assert got[2, :32].isnan().all() and abs(got[2, 40].item() - 2) <= 2 * 3 * U32
    assert got[3, 32:].isnan().all() and abs(got[3, 2].item() - 1) <= 3 * U32
    assert ((got[5] - 3e38).abs() <= 3e38 * 4 * U32).all()
    assert (s[8:] == 0).all() and (s[6] == 0).all()


def test_cache_of_heads_strides_and_positions():
    """Keys [tokens, heads, width] written through views with strides; a cache inside a larger
    buffer; slots of any shape."""
    tokens, heads, width, slots = 40, 3, 64, 100
    buf = torch.zeros((slots, 2, heads * width + 16), dtype=torch.int8, device="cuda")
    q = buf[:, 1, :heads * width]
    sbuf = torch.zeros((slots, 8), device="cuda")
    s = sbuf[:, 2:2 + heads]
    x = randn((tokens, heads, width), 33, BF16).cuda()
    both = torch.stack([x, -x], 1)  # [tokens, 2, heads, width]
    at = torch.randperm(slots)[:tokens].cuda()
    tk.cache_write(q, s, both[:, 0], at)
    got = tk.cache_read(q, s, at.view(8, 5))
    assert got.shape == (8, 5, heads * width)
    plain, ps = tk.quantize(x.view(tokens, -1), group=width)
    assert torch.equal(q[at], plain) and torch.equal(s[at], ps)
    assert (buf[:, 0] == 0).all() and (buf[:, 1, heads * width:] == 0).all()
    assert (sbuf[:, :2] == 0).all() and (sbuf[:, 5:] == 0).all()


def test_cache_past_32_bits():
    slots, dim = 1_050_000, 4112
    q = torch.empty((slots, dim), dtype=torch.int8, device="cuda")
    s = torch.empty((slots, 1), device="cuda")
    at = torch.tensor([slots - 1, 0, slots // 2], device="cuda")
    x = randn((3, dim), 34, BF16).cuda()
    tk.cache_write(q, s, x, at)
    want, ws = tk.quantize(x)
    assert torch.equal(q[at], want) and torch.equal(s[at], ws)
    assert torch.equal(tk.cache_read(q, s, at, dtype=F32), want.float() * ws)


# ------------------------------------------------------------------ product

def ints(shape, seed, lo=-128, hi=127, pad=True):
    g = torch.Generator().manual_seed(seed)
    v = torch.randint(lo, hi + 1, shape, generator=g, dtype=torch.int8)
    if not pad:
        return v.cuda()
    buf = torch.full((shape[0], (shape[1] + 15) // 16 * 16), 77, dtype=torch.int8)
    buf[:, :shape[1]] = v
    return buf.cuda()[:, :shape[1]]


def scores(x, xs, w, ws):
    """Exact sums in 64 bits (float64 holds them), then the scales."""
    return (x.cpu().double() @ w.cpu().double().t()) * xs.cpu().double()[:, None] * ws.cpu().double()[None, :]


PRODUCT_SHAPES = [(1, 1, 1), (1, 1000, 64), (1, 257, 1000), (2, 130, 48), (3, 70, 17), (4, 512, 256),
                  (15, 333, 129), (16, 64, 128), (17, 65, 127), (31, 100, 640), (33, 1030, 1016),
                  (63, 40, 4096), (64, 300, 512), (65, 129, 2000), (100, 1, 300), (127, 257, 33),
                  (128, 128, 128), (129, 384, 1152), (200, 513, 96), (257, 1025, 260), (300, 300, 5000),
                  (700, 2, 64), (1000, 770, 144), (513, 2049, 320)]


@pytest.mark.parametrize("pad", [True, False])
@pytest.mark.parametrize("m,n,k", PRODUCT_SHAPES)
def test_product(m, n, k, pad):
    """The sum is one rounding, each scale another."""
    x, w = ints((m, k), 40, pad=pad), ints((n, k), 41, pad=pad)
    g = torch.Generator().manual_seed(42)
    xs, ws = (torch.rand(m, generator=g) + 0.5).cuda(), (torch.rand(n, generator=g) * 0.01 + 0.001).cuda()
    want = scores(x, xs, w, ws)
    for out in (F32, BF16) if m % 2 else (F32, F16):
        xs2 = xs * (1e-3 if out == F16 else 1.0)
        want2 = scores(x, xs2, w, ws)
        near(tk.product(x, xs2, w, ws, dtype=out), want2, rounded(want2, out, 3))
    assert want.shape == (m, n)


@pytest.mark.parametrize("m", [1, 9, 40, 90, 200])
def test_product_at_the_largest_sums(m):
    """k = 131071 with nothing but -128: sums of 2^31 - 2^14, exact in 32 bits."""
    k, n = 131_071, 33
    x = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    w = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(max(m, n), device="cuda")
    got = tk.product(x, one[:m], w, one[:n], dtype=F32)
    assert (got == float(k * 128 * 128)).all()


@pytest.mark.parametrize("m", [1, 5, 20, 50, 300])
def test_product_of_strided_rows(m):
    """Rows inside larger matrices, output inside a larger one, infinite and NaN scales."""
    n, k = 150, 200
    xb, wb = ints((m, 3 * 208), 43), ints((n, 2 * 208), 44)
    x, w = xb[:, 208:208 + k], wb[:, 16:16 + k]
    xs, ws = torch.ones(m, device="cuda"), torch.full((n,), 0.5, device="cuda")
    buf = torch.full((m, n + 7), 3.0, device="cuda")
    tk.product(x, xs, w, ws, dtype=F32, out=buf[:, 3:3 + n])
    want = scores(x, xs, w, ws)
    near(buf[:, 3:3 + n], want, rounded(want, F32, 3))
    assert (buf[:, :3] == 3).all() and (buf[:, 3 + n:] == 3).all()
    ws[7] = float("nan")
    xs[0] = float("inf")
    got = tk.product(x, xs, w, ws, dtype=F32)
    assert got[:, 7].isnan().all()
    rest = torch.arange(n, device="cuda") != 7
    assert not torch.isfinite(got[0, rest]).any() and torch.isfinite(got[1:, rest]).all()


def test_product_past_32_bits():
    """A table of more than 2^32 bytes: its last rows."""
    n, k = 1_050_000, 4112
    w = torch.zeros((n, k), dtype=torch.int8, device="cuda")
    w[-1] = 2
    w[n // 2] = 1
    x = torch.ones((3, k), dtype=torch.int8, device="cuda")
    ws, xs = torch.ones(n, device="cuda"), torch.ones(3, device="cuda")
    for m in (1, 3):
        got = tk.product(x[:m], xs[:m], w, ws, dtype=F32)
        assert (got[:, -1] == 2 * k).all() and (got[:, n // 2] == k).all()
        assert int(torch.count_nonzero(got)) == 2 * m


# ------------------------------------------------------------------ streams, graphs, refusals

def test_other_streams_and_graphs():
    """On a stream of its own, and captured into a graph that is replayed on new inputs with
    eager work in between, every operator gives what it gives eagerly."""
    tok, n, rows, dim = some_tokens(2000, 300, 50).cuda(), 2000, 300, 96
    w, g = randn((rows, dim), 51).cuda(), randn((n, dim), 52, BF16).cuda()
    q, s = tk.empty_cache(n, dim)
    slots = torch.randperm(n, device="cuda")

    def work():
        a = tk.lookup(tok, w, 2.0, 0.1, 5, 6)
        b = tk.lookup_grad(tok, g, rows, 2.0, 0.1, 5, 6)
        c = tk.dropout(g, 0.2, 7, 8, residual=g)
        tk.cache_write(q, s, g, slots)
        d = tk.cache_read(q, s, slots)
        x, xs = tk.quantize(w)
        return [a, b, c, d, tk.product(x, xs, x, xs), tk.product(x[:3], xs[:3], x, xs)]
    eager = [t.clone() for t in work()]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        other = work()
    st.synchronize()
    for x, y in zip(eager, other):
        assert torch.equal(x, y)
    given = tk.lookup_grad(tok, g, rows, 2.0, 0.1, 5, 6, stream=st)
    st.synchronize()
    assert torch.equal(given, eager[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = work()
    for k in range(3):
        tok.copy_(some_tokens(2000, 300, 60 + k).cuda())
        g.copy_(randn((n, dim), 70 + k, BF16).cuda())
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for x, y in zip(work(), got):
            assert torch.equal(x, y)


def test_binding_refusals():
    t, w = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros((5, 8), device="cuda")
    q, s = tk.empty_cache(10, 8)
    for call, text in [
            (lambda: tk.lookup(t.float(), w), "tokens"),
            (lambda: tk.lookup(t, w[0]), "rows, dim"),
            (lambda: tk.lookup(t, w.double()), "table"),
            (lambda: tk.lookup(t, w, out=torch.zeros((4, 9), device="cuda")), "out is"),
            (lambda: tk.lookup(t, w, out=torch.zeros((8, 4), device="cuda").t()), "follow one another"),
            (lambda: tk.lookup(t, w, p=1.0), "p 1"),
            (lambda: tk.lookup(t.cpu(), w), "tensors on"),
            (lambda: tk.lookup_grad(t, w, 5), "tokens"),
            (lambda: tk.lookup_grad(t, w[:4], 5, accumulate=True), "accumulate"),
            (lambda: tk.lookup_grad(t, w[:4], -1), "rows"),
            (lambda: tk.dropout(w, 0.5, 1, residual=w.bfloat16()), "residual"),
            (lambda: tk.cache_write(q, s, w, t), "slots"),
            (lambda: tk.cache_write(q.float(), s, w[:4], t), "cache"),
            (lambda: tk.cache_read(q, s[:, :0], t), "scales"),
            (lambda: tk.cache_read(q, s, t, dtype=torch.int8), "out"),
            (lambda: tk.quantize(w, group=3), "group"),
            (lambda: tk.product(q, s, q[:, :4], s), "are needed"),
            (lambda: tk.product(w, s, q, s), "int8"),
            (lambda: tk.product(q, s[:3], q, s), "scales")]:
        with pytest.raises(sp.SPError, match=text) as e:
            call()
        assert e.value.status == sp.SP_ERR_INVALID_ARG


def test_empty_shapes():
    t, w = torch.zeros((0, 3), dtype=torch.int64, device="cuda"), randn((5, 8), 80).cuda()
    assert tk.lookup(t, w).shape == (0, 3, 8)
    assert tk.lookup_grad(t, torch.zeros((0, 3, 8), device="cuda"), 5).eq(0).all()
    assert tk.dropout(w[:0], 0.5, 1).shape == (0, 8)
    q, s = tk.quantize(w[:0])
    assert q.shape == (0, 8) and tk.product(q, s, *tk.quantize(w)).shape == (0, 5)
    assert tk.product(*tk.quantize(w), q, s).shape == (5, 0)
    assert tk.cache_read(q, s, t).eq(0).all()
