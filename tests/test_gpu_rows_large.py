"""The forms of the row operators that only larger calls take, and the example that runs them
together.  Bounds as in test_gpu_rows.py."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2205_04702_amd import tokens as tk  # noqa: E402
from tests.rows_reference import U32, UNIT, TINY  # noqa: E402

F32, BF16, F16, F8 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def near(got, want, r):
    """Within r roundings to fp32 and one to the output's type, on the GPU in 64 bits."""
    bound = want.abs() * (UNIT[got.dtype] + (r + 1) * U32) + TINY[got.dtype]
    off = (got.double() - want).abs() - bound
    assert not torch.isnan(off).any()
    assert off.max().item() <= 0


@pytest.mark.parametrize("n,dim,table,out", [
    (2_200_000, 5, F32, BF16),      # rows narrower than an octet, many of them
    (300_000, 65, F32, F32),        # a last octet of one column; fp32 exchanged among lanes
    (300_001, 68, F16, F32),        # ... of four, and a width of 9 octets
    (66_000, 264, BF16, F32),       # 33 octets: not a multiple of four lanes
    (262_145, 64, BF16, F16),
])
def test_lookup_of_many(n, dim, table, out):
    g = rng(1)
    w = torch.randn((1000, dim), generator=g, device="cuda").to(table)
    tok = torch.randint(-50, 1050, (n,), generator=g, device="cuda")
    got = tk.lookup(tok, w, 1.7, dtype=out)
    live = (tok >= 0) & (tok < 1000)
    want = w.double()[tok.clamp(0, 999)] * 1.7 * live[:, None]
    near(got, want, 2)
    assert (got[~live] == 0).all()
    # with dropout: what is kept is scaled, and the mask is that of single rows
    p = 0.25
    kept = tk.lookup(tok, w, 1.7, p, 5, 6, dtype=out)
    ones = tk.dropout(torch.ones((n, dim), device="cuda"), p, 5, 6)
    near(kept, torch.where(ones != 0, want / 0.75, torch.zeros_like(want)), 3)
    some = tk.dropout(torch.ones((3000, dim), device="cuda"), p, 5, 6)
    assert torch.equal(ones[:3000], some)


@pytest.mark.parametrize("kind", [torch.int8, F8])
@pytest.mark.parametrize("n,dim,group,dtype", [
    (70_000, 256, 32, BF16), (40_000, 192, 64, F32), (20_001, 384, 128, F16), (30_000, 200, 200, BF16),
    (9_000, 512, 512, BF16), (5_000, 1400, 1400, F32), (50_000, 61, 61, BF16)])
def test_cache_of_many(n, dim, group, dtype, kind):
    """Rows written in bulk are what a few at a time are, and read back in bulk."""
    g = rng(2)
    x = torch.randn((n, dim), generator=g, device="cuda").to(dtype)
    slots = n + 1000
    at = torch.randperm(slots, generator=g, device="cuda")[:n]
    at[::97] = -1
    q, s = tk.empty_cache(slots, dim, group, kind)
    tk.cache_write(q, s, x, at)
    live = at >= 0
    for i in range(0, n, n // 3):
        some = slice(i, i + 37)
        p, ps = tk.quantize(x[some], group, kind)
        rows = live[some]
        assert torch.equal(q.view(torch.uint8)[at[some][rows]], p.view(torch.uint8)[rows])
        assert torch.equal(s[at[some][rows]], ps[rows])
    rest = torch.ones(slots, dtype=torch.bool, device="cuda")
    rest[at[live]] = False
    assert (q.view(torch.uint8)[rest] == 0).all() and (s[rest] == 0).all()
    for out in (F32, BF16):
        got = tk.cache_read(q, s, at, dtype=out)
        want = q[at.clamp(min=0)].double().view(n, -1, group) * s[at.clamp(min=0)].double()[..., None]
        near(got, want.view(n, dim) * live[:, None], 1)
    # and the values are those that were written, up to half a step
    step = s[at[live]].double().repeat_interleave(group, 1) * (1.0 if kind == torch.int8 else 32.0)
    off = (tk.cache_read(q, s, at[live], dtype=F32).double() - x[live].double()).abs()
    assert (off <= step * 0.5 + x[live].double().abs() * 6 * U32).all()


@pytest.mark.parametrize("pad", [True, False])
@pytest.mark.parametrize("m,n,k", [(3000, 5000, 260), (520, 40_001, 100), (4100, 2300, 64),
                                   (8, 30_000, 1000), (40, 20_000, 3000), (1, 50_000, 777),
                                   (64, 512, 20_000), (200, 64, 9_000), (700, 900, 4_000)])
def test_product_cuts(m, n, k, pad):
    """Every tile, whole and in parts of k."""
    g = rng(3)
    ld = (k + 15) // 16 * 16 if pad else k + (k % 16 == 0)
    x = torch.randint(-128, 128, (m, ld), generator=g, device="cuda", dtype=torch.int8)[:, :k]
    w = torch.randint(-128, 128, (n, ld), generator=g, device="cuda", dtype=torch.int8)[:, :k]
    xs, ws = torch.rand(m, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda")
    want = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()[None, :]
    for out in (F32, BF16):
        near(tk.product(x, xs, w, ws, dtype=out), want, 3)


@pytest.mark.parametrize("dim,dtype", [(20, BF16), (100, F32), (130, F16), (520, BF16), (1100, F32)])
def test_grad_of_many(dim, dtype):
    """Runs over the edges of teams, blocks and tiles: Zipf tokens, against sums in 64 bits."""
    g, n, rows = rng(4), 150_000, 40_000
    w = torch.arange(1, rows + 1, device="cuda", dtype=torch.float64) ** -1.0
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * w.sum()
    tok = torch.searchsorted(w.cumsum(0), u).clamp_(max=rows - 1)
    x = torch.randn((n, dim), generator=g, device="cuda").to(dtype)
    got = tk.lookup_grad(tok, x, rows)
    total = torch.zeros((rows, dim), dtype=torch.float64, device="cuda")
    size, count = torch.zeros_like(total), torch.bincount(tok, minlength=rows).double()[:, None]
    total.index_add_(0, tok, x.double())
    size.index_add_(0, tok, x.double().abs())
    off = (got.double() - total).abs()
    assert (off <= size * (count + 3) * U32 + total.abs() * 2 * U32 + 1e-40).all()
    assert (got[count[:, 0] == 0] == 0).all()
    assert torch.equal(got, tk.lookup_grad(tok, x, rows))
    base = torch.randn((rows, dim), generator=g, device="cuda")
    sums = base.clone()
    tk.lookup_grad(tok, x, rows, out=sums, accumulate=True)
    off = (sums.double() - (base.double() + total)).abs()
    assert (off <= size * (count + 3) * U32 + (base.double().abs() + total.abs()) * 3 * U32 + 1e-40).all()
    unused = count[:, 0] == 0
    assert torch.equal(sums[unused], base[unused])


def test_example_trains_and_serves():
    """The entropy of the noise is about 0.53; 8 bits hold a row's values within 0.4 % of its
    largest, some 0.6 % of their size, twice."""
    from paper_2205_04702_amd import token_example
    r = token_example.run(vocab=512, dim=64, steps=200, batch=4096)
    assert r["first_loss"] > 4.0 and r["last_loss"] < 1.0
    assert r["right"] > 0.99 and r["right_in_8_bits"] > 0.99
    assert r["off_in_8_bits"] < 0.03
