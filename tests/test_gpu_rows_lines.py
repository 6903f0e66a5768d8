"""The row operators at the lines between their forms, and used as their header allows: outputs
with strides, several threads.  Bounds as in test_gpu_rows.py."""
import threading

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2205_04702_amd import tokens as tk  # noqa: E402
from tests import rows_reference as ref  # noqa: E402
from tests.rows_reference import U32  # noqa: E402
from tests.test_gpu_rows import BF16, F16, F32, grad_bound, near, randn, some_tokens  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("n", [959, 960, 961])
@pytest.mark.parametrize("dim,p", [(16, 0.0), (45, 0.25), (1030, 0.0)])
def test_grad_around_the_one_launch_form(n, dim, p):
    """Up to 960 tokens one launch, while positions times stretches of 512 columns are 2048 at most."""
    rows = 300
    tok, g = some_tokens(n, rows, 90), randn((n, dim), 91, BF16)
    got = tk.lookup_grad(tok.cuda(), g.cuda(), rows, 0.7, p, 3, 4)
    want, size, count = ref.lookup_grad(tok, g, rows, 0.7, p, 3, 4)
    near(got, want, grad_bound(size, count, want, F32))


@pytest.mark.parametrize("n,dim", [(682, 1030), (683, 1030), (1024, 1), (512, 2048), (513, 2048), (2, 524_288), (2, 524_800)])
def test_grad_around_the_limit_of_its_blocks(n, dim):
    rows = 40
    tok, g = some_tokens(n, rows, 92, pad=0.4 if n > 2 else 0.0, hot=0.3 if n > 2 else 1.0), randn((n, dim), 93, BF16)
    got = tk.lookup_grad(tok.cuda(), g.cuda(), rows)
    want, size, count = ref.lookup_grad(tok, g, rows)
    near(got, want, grad_bound(size, count, want, F32))


def test_grad_of_the_widest_rows():
    """Two tokens of 2^20 columns, added to an output; one is padding."""
    dim, rows = 1 << 20, 3
    g, base = randn((2, dim), 94, F16), randn((rows, dim), 95)
    for tok in (torch.tensor([1, -1]), torch.tensor([2, 2])):
        out = base.cuda()
        tk.lookup_grad(tok.cuda(), g.cuda(), rows, 2.0, out=out, accumulate=True)
        want, size, count = ref.lookup_grad(tok, g, rows, 2.0)
        b = base.double()
        near(out, b + want, grad_bound(size, count, b + want, F32, b))
        unused = count[:, 0] == 0
        assert torch.equal(out.cpu()[unused], base[unused])


@pytest.mark.parametrize("rows", [600, 100_000, 300_000])  # digits of 5, 9 and 7 bits
@pytest.mark.parametrize("n", [131_072, 131_073, 262_145, 530_000, 2_100_000])
def test_grad_around_the_sort_s_prefix(n, rows):
    dim = 4
    g = torch.Generator(device="cuda")
    g.manual_seed(n + rows)
    tok = torch.randint(-rows // 50, rows, (n,), generator=g, device="cuda")
    x = torch.randn((n, dim), generator=g, device="cuda").to(BF16)
    got = tk.lookup_grad(tok, x, rows)
    live = tok >= 0
    total = torch.zeros((rows, dim), dtype=torch.float64, device="cuda")
    size, count = torch.zeros_like(total), torch.bincount(tok[live], minlength=rows).double()[:, None]
    total.index_add_(0, tok[live], x[live].double())
    size.index_add_(0, tok[live], x[live].double().abs())
    off = (got.double() - total).abs()
    assert (off <= size * (count + 3) * U32 + total.abs() * 2 * U32 + 1e-40).all()
    assert torch.equal(got, tk.lookup_grad(tok, x, rows))


@pytest.mark.parametrize("n", [30, 3000, 20_000])  # one launch, counted, sorted
@pytest.mark.parametrize("out,dim,left,right", [(F32, 33, 1, 2), (F32, 64, 4, 4), (BF16, 50, 3, 5), (F16, 7, 1, 1)])
def test_grad_into_rows_inside_a_larger_matrix(n, out, dim, left, right):
    """Zeros and sums between foreign columns, which keep what they hold."""
    rows = 3000
    tok, g = some_tokens(n, 700, 96), randn((n, dim), 97, F16)
    buf = torch.full((rows, left + dim + right), 9.0, dtype=out, device="cuda")
    tk.lookup_grad(tok.cuda(), g.cuda(), rows, 0.5, out=buf[:, left:left + dim])
    assert (buf[:, :left] == 9).all() and (buf[:, left + dim:] == 9).all()
    want, size, count = ref.lookup_grad(tok, g, rows, 0.5)
    near(buf[:, left:left + dim], want, grad_bound(size, count, want, out))


def test_several_threads():
    """Each on its own stream and tensors: what one thread gives."""
    def work(i, outs):
        tok, w, g = some_tokens(3000, 500, 100 + i).cuda(), randn((500, 96), 110 + i).cuda(), \
            randn((3000, 96), 120 + i, BF16).cuda()
        st = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            for _ in range(20):
                x = tk.lookup(tok, w, 2.0, 0.1, 5, i)
                d = tk.lookup_grad(tok, g, 500, 2.0, 0.1, 5, i)
                q, s = tk.quantize(w)
                y = tk.product(*tk.quantize(x), q, s)
                z = tk.dropout(tk.cache_read(q, s, tok), 0.2, 6, i)
        st.synchronize()
        outs[i] = [t.cpu() for t in (x, d, y, z)]
    alone, together = {}, {}
    for i in range(4):
        work(i, alone)
    threads = [threading.Thread(target=work, args=(i, together)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(4):
        assert len(together[i]) == 4 and all(torch.equal(a, b) for a, b in zip(alone[i], together[i]))


@pytest.mark.parametrize("n,dim,ld,left", [(130_000, 65, 72, 0), (130_000, 65, 72, 8), (130_000, 65, 72, 1),
                                           (130_000, 65, 67, 0), (40_000, 256, 256, 0), (40_000, 250, 250, 0)])
@pytest.mark.parametrize("out", [F32, BF16])
def test_many_rows_into_whole_and_shared_pieces(n, dim, ld, left, out):
    """More than 2^20 octets, fp32 rows at multiples of 32 bytes and elsewhere: a lookup and a read of
    the cache give what a few rows at a time give, and keep to their columns."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n + dim)
    w = torch.randn((500, dim), generator=g, device="cuda")
    tok = torch.randint(-20, 520, (n,), generator=g, device="cuda")
    q, s = tk.quantize(w)
    for call in (lambda t, o: tk.lookup(t, w, 1.5, out=o), lambda t, o: tk.cache_read(q, s, t, dtype=out, out=o)):
        buf = torch.full((n, left + ld), 9.0, dtype=out, device="cuda")
        call(tok, buf[:, left:left + dim])
        few = torch.empty((1000, dim), dtype=out, device="cuda")
        every = torch.cat([torch.arange(500, device="cuda"), torch.full((500,), -1, device="cuda")])
        call(every, few)
        where = torch.where((tok >= 0) & (tok < 500), tok, torch.full_like(tok, 999))
        assert torch.equal(buf[:, left:left + dim], few[where])
        assert (buf[:, :left] == 9).all() and (buf[:, left + dim:] == 9).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("octets", [2 ** 20 - 1000, 2 ** 20, 2 ** 21])
def test_dropout_around_its_deep_form(dtype, octets):
    dim = 1000
    n = octets // 125 + 1
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x, r = torch.randn((n, dim), generator=g, device="cuda").to(dtype), torch.randn((n, dim), device="cuda").to(dtype)
    got = tk.dropout(x, 0.25, 8, 9, residual=r)
    assert torch.equal(got[:700], tk.dropout(x[:700], 0.25, 8, 9, residual=r[:700]))
    mask = tk.dropout(torch.ones((n, dim), device="cuda"), 0.25, 8, 9) != 0
    assert torch.equal(mask[:50].cpu(), ref.keep_mask(50, dim, 0.25, 8, 9))
    y = torch.where(mask, x.double() / 0.75, torch.zeros((), dtype=torch.float64, device="cuda"))
    want = y + r.double()
    off = (got.double() - want).abs() - (y.abs() * 3 * U32 + want.abs() * (ref.UNIT[dtype] + 2 * U32) + ref.TINY[dtype])
    assert off.max().item() <= 0
