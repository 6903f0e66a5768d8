"""The operators on 4-bit rows and scores as they are used: one after the other, in the example, in captured
graphs, on another stream, from several threads, beside autograd."""
import threading

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2205_04702_amd import token_example as ex  # noqa: E402
from paper_2205_04702_amd import tokens as tk  # noqa: E402
from tests import scores_reference as ref  # noqa: E402
from tests.rows_reference import TINY, U32, UNIT  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def test_from_rows_to_answers_and_to_a_loss():
    """Rows into a cache, back, quantised, scored, adjusted; the same scores against a teacher."""
    vocab, dim, n, k = 300, 100, 9, 12
    table, out = torch.randn((vocab, dim), generator=gen(1)), torch.randn((vocab, dim), generator=gen(2))
    now = torch.randint(vocab, (n,), generator=gen(3))
    q, s = tk.empty_cache4(vocab, dim)
    tk.cache_write4(q, s, table.cuda(), torch.arange(vocab, device="cuda"))
    x = tk.cache_read4(q, s, now.cuda(), dim, F32)
    w, ws = tk.quantize4(out.cuda())
    scores = tk.product4(*tk.quantize4(x), w, ws, F32)
    tq, ts = ref.quantize4(table)
    rows = ref.values4(tq, ts)[now][:, :dim]
    assert torch.equal(x.cpu().double(), rows)
    want, off = ref.product4(*ref.quantize4(rows), *ref.quantize4(out))
    assert ((scores.cpu().double() - want).abs() <= off + want.abs() * UNIT[F32]).all()
    had = scores.cpu()
    previous, allowed = torch.randint(-1, vocab, (n, 40), generator=gen(4)), torch.randint(-2 ** 31, 2 ** 31, (n, 10), generator=gen(5)).int()
    numbers = (1.5, 0.25, 0.125)
    got = tk.adjust(scores, previous.cuda(), *numbers, allowed=allowed.cuda()).cpu().double()
    want, size = ref.adjust(had, previous, numbers, None, None, None, allowed)
    assert torch.equal(got == -ref.INF, want == -ref.INF)
    inside = want != -ref.INF
    assert ((got - want).abs() <= ref.adjust_bound(want, size, F32))[inside].all()
    assert torch.equal(scores.cpu(), had)
    tok, t, weight = torch.randint(vocab, (n, k), generator=gen(6)), torch.randn((n, k), generator=gen(7)), torch.full((n,), 1 / n)
    loss, grad = tk.distill_grad(scores, tok.cuda(), t.cuda(), 1 / n, 2.0, out=scores)
    want, want_grad, loss_off, grad_off = ref.distill(had, tok, t, weight, 2.0)
    assert ((loss.cpu().double() - want).abs() <= loss_off + want.abs() * UNIT[F32]).all()
    assert ((grad.cpu().double() - want_grad).abs() <= grad_off + (want_grad.abs() + grad_off) * UNIT[F32] + TINY[F32]).all()


def test_example_runs():
    r = ex.run(vocab=130, dim=24, steps=3, batch=64)
    assert r["allowed"] == 1.0 and all(v == v for v in r.values())


def test_example_gradients():
    """A student's step against autograd in 64 bits.  The products with its tables are torch's, in fp32: a sum of c
    terms is within (c + 2) U of the sum of their magnitudes, which the gradient's own bound joins."""
    vocab, dim, n, k, T, scale = 70, 12, 33, 8, 2.0, 3.0
    Es, Ws = torch.randn((vocab, dim), generator=gen(8)), torch.randn((vocab, dim), generator=gen(9))
    now, tok = torch.randint(vocab, (n,), generator=gen(10)), torch.stack([torch.randperm(vocab, generator=gen(i))[:k] for i in range(n)])
    t = torch.randn((n, k), generator=gen(11)) * 2
    loss, dE, dW = ex.student_step(now.cuda(), (tok.cuda(), t.cuda()), Es.cuda(), Ws.cuda(), scale, T)
    E, W = Es.double().requires_grad_(), Ws.double().requires_grad_()
    x = E[now] * scale
    s = x @ W.t()
    p = torch.softmax(t.double() / T, 1)
    each = T * T * (p * (p.log() - torch.log_softmax(s / T, 1).gather(1, tok))).sum(1)
    each.mean().backward()
    s_off = ((dim + 4) * U32 * (x.abs() @ W.abs().t())).detach().max().item()
    _, d, loss_off, d_off = ref.distill(s.detach(), tok, t, torch.full((n,), 1 / n), T)
    d_off = d_off + 2 * s_off * d.abs().max() + d.abs() * 4 * U32  # a score that is off by s moves q by at most q s / T
    dx_off = d_off @ W.abs() + (vocab + 4) * U32 * (d.abs() @ W.abs())
    want = torch.zeros_like(E).index_add_(0, now, dx_off * scale) + E.grad.abs() * (n + 4) * U32
    assert ((dE.cpu().double() - E.grad).abs() <= want.detach()).all()
    want = d_off.t() @ x.abs() + (n + 4) * U32 * (d.abs().t() @ x.abs())
    assert ((dW.cpu().double() - W.grad).abs() <= want.detach()).all()
    # (a loss moves by at most 2 T times what a score does: T^2 / T by the entries' and by the sum's logarithm)
    assert ((loss.cpu().double() - each.detach()).abs() <= loss_off + 2 * T * s_off + each.detach().abs() * UNIT[F32]).all()


def all_calls(seed):
    """Every operator in each of its forms at a small size: the tensors that they read, and the calls."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, dtype=F32):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    x, wide = randn(20, 100), randn(4200, 300, dtype=BF16)
    q, s = tk.empty_cache4(30, 100)
    slots = torch.randperm(30, generator=g, device="cuda")[:20]
    long = randn(3, 8192)
    tok, t = torch.randint(0, 500, (6, 9), generator=g, device="cuda"), randn(6, 9)
    few, many = randn(6, 60_001, dtype=BF16), randn(6, 500)
    words = torch.randint(-2 ** 31, 2 ** 31, (6, 16), generator=g, device="cuda").int()

    def go():
        tk.cache_write4(q, s, x, slots)
        big = tk.quantize4(wide)
        return [q.clone(), s.clone(), tk.cache_read4(q, s, slots, 100), *big, tk.product4(*big, *big), tk.product4(*tk.quantize4(long), *tk.quantize4(long)),
                tk.adjust(many, tok, 1.2, 0.5, 0.25, bias_tokens=tok, bias=t, allowed=words), tk.distill(many, tok, t), tk.distill(few, tok, t),
                *tk.distill_grad(many, tok, t, 0.5), *tk.distill_grad(few, tok, t, 0.5, 2.0)]

    return (x, wide, long, t, few, many), go


def test_captured_and_replayed():
    graphs = []
    for seed in (1, 2):
        inputs, go = all_calls(seed)
        go()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = go()
        graphs.append((inputs, go, graph, outs))
    for turn in range(3):
        for inputs, go, graph, outs in graphs:
            for t in inputs:
                t.mul_(-0.75).add_(0.01 * turn)
            graph.replay()
            torch.cuda.synchronize()
            for i, (got, want) in enumerate(zip(outs, go())):
                assert torch.equal(got, want), (turn, i)


def test_on_another_stream_and_from_threads():
    work = [all_calls(seed) for seed in (3, 4, 5)]
    wants = [go() for _, go in work]
    torch.cuda.synchronize()
    got = [None] * 3

    def one(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(5):
                got[i] = work[i][1]()
        stream.synchronize()

    threads = [threading.Thread(target=one, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for a, b in zip(got, wants):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    x = torch.randn((5, 64), device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for call in (lambda **kw: tk.quantize4(x, **kw)[0], lambda **kw: tk.adjust(x, **kw),
                 lambda **kw: tk.distill(x, torch.arange(5, device="cuda")[:, None], x[:, :1], **kw)):
        want = call()
        torch.cuda.synchronize()
        got = call(stream=stream)
        stream.synchronize()
        assert torch.equal(got, want)


def test_what_is_written_into_counts_as_changed():
    q, s = tk.quantize4(torch.randn((4, 64), device="cuda"))
    t, i = torch.randn((4, 70), device="cuda"), torch.arange(4, device="cuda")
    for shape, call in (((4, 64), lambda out: tk.cache_read4(q, s, i, dtype=F32, out=out)), ((4, 4), lambda out: tk.product4(q, s, q, s, F32, out=out)),
                        ((4, 70), lambda out: tk.adjust(t, out=out)), ((4, 70), lambda out: tk.distill_grad(t, i[:, None], t[:, :1], out=out)[1])):
        buf, x = torch.ones(shape, device="cuda"), torch.ones(shape, device="cuda", requires_grad=True)
        y = (x * buf).sum()
        assert call(buf) is buf and not call(buf).requires_grad
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    before = q._version, s._version
    tk.cache_write4(q, s, t[:, :64], i)
    assert q._version > before[0] and s._version > before[1]


def test_long_lists_and_rows_past_32_bits():
    """Scores whose elements pass 2^32, a cache whose bytes do."""
    rows, vocab = 4200, 1 << 20
    s = torch.zeros((rows, vocab), dtype=BF16, device="cuda")
    s[-1, 7], s[-1, -1] = 4.0, 2.0
    tok = torch.full((rows, 2), -1, device="cuda")
    tok[-1, 0], tok[-1, 1] = 7, vocab - 1
    t = torch.zeros((rows, 2), device="cuda")
    allowed = torch.full((vocab // 32,), -1, dtype=torch.int32, device="cuda")
    tk.adjust(s, tok, 2.0, 0.5, 0.0, allowed=allowed, out=s)
    assert s[-1, 7] == 1.5 and s[-1, -1] == 0.5 and int(torch.count_nonzero(s[-2:])) == 2
    loss, grad = tk.distill_grad(s, tok, t, out=s)
    assert grad is s and int(torch.count_nonzero(loss)) == 1 and not s[0].any() and not s[-2].any()
    want, want_grad, loss_off, _ = ref.distill(torch.zeros((1, vocab)).index_put_((torch.tensor([0, 0]), torch.tensor([7, vocab - 1])), torch.tensor([1.5, 0.5])),
                                               tok[-1:].cpu(), t[-1:].cpu(), torch.ones(1), 1.0)
    assert (loss[-1].cpu().double() - want).abs() <= loss_off + want.abs() * UNIT[F32]
    assert torch.allclose(s[-1].cpu().double(), want_grad[0], rtol=2 ** -7, atol=0)
    del s, grad
    q, sc = tk.empty_cache4(9_000_000, 1024)
    x = torch.full((3, 1024), 1.5, device="cuda")
    at = torch.tensor([0, 8_999_999, 5_000_000], device="cuda")
    tk.cache_write4(q, sc, x, at)
    assert torch.equal(tk.cache_read4(q, sc, at, dtype=F32), x)
    assert not tk.cache_read4(q, sc, at[1:] - 1).any()
    scores = tk.product4(*tk.quantize4(x[:1]), q, sc, F32)
    assert scores.shape == (1, 9_000_000) and (scores[0, at] == 1024 * 2.25).all() and int(torch.count_nonzero(scores)) == 3


def test_more_rows_than_one_launch_has_blocks():
    """Calls of 2^22 blocks and more of 1024 threads, and of a block for each of as many rows."""
    n, vocab = (1 << 22) + 3, 2
    s = torch.zeros((n, vocab), dtype=BF16, device="cuda")
    s[:, 1] = 2.0
    previous = torch.cat([torch.ones(3, dtype=torch.int64), torch.full((8200,), -1)]).cuda()  # for all rows
    got = tk.adjust(s, previous, 2.0, 0.25, 0.125)
    assert not got[:, 0].any() and (got[:, 1] == 2.0 / 2 - 0.25 - 3 * 0.125).all()
    tok, t = torch.ones((n, 1), dtype=torch.int32, device="cuda"), torch.zeros((n, 1), device="cuda")
    loss = tk.distill(s, tok, t)
    again, grad = tk.distill_grad(s, tok, t)
    want, want_grad, off, grad_off = ref.distill(s[:1].cpu(), tok[:1].cpu(), t[:1].cpu(), torch.ones(1), 1.0)
    for one in (loss, again):
        assert (one == one[0]).all() and (one[0].cpu().double() - want[0]).abs() <= off[0] + want[0].abs() * UNIT[F32]
    assert (grad == grad[0]).all()
    assert ((grad[0].cpu().double() - want_grad[0]).abs() <= grad_off[0] + (want_grad[0].abs() + grad_off[0]) * UNIT[BF16] + TINY[BF16]).all()


def test_lists_of_no_width():
    s = torch.randn((2, 3, 40), device="cuda")
    none = torch.empty((2, 3, 0), dtype=torch.int64, device="cuda")
    assert torch.equal(tk.adjust(s, none, bias_tokens=none, bias=none.float()), s)
