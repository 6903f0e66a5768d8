"""Adjusted scores and distillation against plain implementations in 64 bits, within the bounds that
scores_reference.py derives."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2205_04702_amd import scratchpipe as sp  # noqa: E402
from paper_2205_04702_amd import tokens as tk  # noqa: E402
from tests import scores_reference as ref  # noqa: E402
from tests.rows_reference import TINY, UNIT  # noqa: E402

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF, NAN = math.inf, math.nan


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def cuda(t):
    return None if t is None else t.cuda()


# ------------------------------------------------------------------ adjust

def request(n, vocab, length, biases, mask, per_row, dtype, seed, tokens=torch.int64):
    g = gen(seed)
    r = dict(scores=(torch.randn((n, vocab), generator=g) * 3).to(dtype), previous=None, penalties=None, bias_tokens=None,
             bias=None, allowed=None)
    if length:
        hot = torch.randint(vocab, (n, 3), generator=g)
        t = torch.randint(-1, vocab + 1, (n, length), generator=g)  # -1 and vocab: no columns
        often = torch.rand((n, length), generator=g) < 0.4
        r["previous"] = torch.where(often, hot.gather(1, torch.randint(3, (n, length), generator=g)), t).to(tokens)
    if biases:
        t = torch.randint(-2, vocab, (n, biases), generator=g)
        t[:, -1] = t[:, 0]  # twice
        r["bias_tokens"], r["bias"] = t.to(tokens), torch.randn((n, biases), generator=g) * 5
    if mask:
        w = torch.randint(-2 ** 31, 2 ** 31, (n, (vocab + 31) // 32), generator=g)
        w[0] = -1
        if n > 1:
            w[n - 1] = 0
        r["allowed"] = w.to(torch.int32)
    if per_row:
        r["penalties"] = torch.rand((n, 3), generator=g) + torch.tensor([0.6, -0.2, 0.0])
    return r


def check_adjust(r, numbers, got, dtype):
    want, size = ref.adjust(r["scores"], r["previous"], numbers, r["penalties"], r["bias_tokens"], r["bias"], r["allowed"])
    got = got.cpu().double()
    assert torch.equal(got == -INF, want == -INF)
    off = torch.where(want == -INF, torch.zeros_like(want), (got - want).abs()) - ref.adjust_bound(want, size, dtype)
    assert off.max() <= 0, off.max()


def adjusted(r, numbers, **kw):
    return tk.adjust(r["scores"].cuda(), cuda(r["previous"]), *numbers, penalties=cuda(r["penalties"]),
                     bias_tokens=cuda(r["bias_tokens"]), bias=cuda(r["bias"]), allowed=cuda(r["allowed"]), **kw)


@pytest.mark.parametrize("n,vocab,length,biases,mask,per_row,dtype,tokens", [
    (1, 1, 1, 1, True, False, F32, torch.int64),
    (2, 7, 5, 3, True, True, BF16, torch.int32),
    (3, 8, 1, 0, False, False, F16, torch.int64),
    (5, 33, 200, 4, True, False, F32, torch.int32),
    (4, 2047, 0, 0, True, False, BF16, torch.int64),
    (4, 2049, 30, 0, False, True, F32, torch.int64),
    (3, 4100, 5000, 100, True, True, BF16, torch.int64),
    (2, 50_001, 999, 20, True, True, F16, torch.int32),
    (1, 32_768, 0, 50, False, False, F32, torch.int64),
    (7, 1000, 0, 0, False, False, BF16, torch.int64),
    (1, 20_000, 2, 2, True, False, BF16, torch.int32),
    (70, 512, 17, 9, True, True, F32, torch.int64),
    (2, 3001, 40, 2047, False, True, BF16, torch.int32),
])
def test_adjust(n, vocab, length, biases, mask, per_row, dtype, tokens):
    r, numbers = request(n, vocab, length, biases, mask, per_row, dtype, vocab, tokens), (1.3, 0.25, 0.125)
    got = adjusted(r, numbers)
    assert got.dtype == dtype and got.shape == r["scores"].shape
    check_adjust(r, numbers, got, dtype)


@pytest.mark.parametrize("length,biases", [(300, 5), (300, 0), (0, 5), (0, 0)])
@pytest.mark.parametrize("vocab", [60_001, 65_536])
def test_adjust_large(length, biases, vocab):
    """Enough columns for the form with long stretches."""
    n, dtype, numbers = 150, BF16, (1.2, 0.5, 0.25)
    r = request(n, vocab, length, biases, False, False, dtype, 3)
    g = gen(4)
    r["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (n, (vocab + 31) // 32), generator=g).to(torch.int32)
    got = adjusted(r, numbers).cpu()
    x = r["scores"].double()
    if length:
        tok = r["previous"].long()
        count = torch.zeros((n, vocab + 1), dtype=torch.float64)
        count.scatter_add_(1, torch.where((tok >= 0) & (tok < vocab), tok, vocab), torch.ones(tok.shape, dtype=torch.float64))
        count = count[:, :vocab]
        y = torch.where(x > 0, x / numbers[0], x * numbers[0]) - numbers[1] - numbers[2] * count
        x = torch.where(count > 0, y, x)
    if biases:
        for i in range(n):
            for t, b in {t: b for t, b in zip(r["bias_tokens"][i].tolist(), r["bias"][i].tolist()) if t >= 0}.items():
                x[i, t] += b
    on = (r["allowed"].long()[:, :, None] >> torch.arange(32) & 1).view(n, -1)[:, :vocab] > 0
    x = torch.where(on, x, -INF)
    assert torch.equal(got == -INF, x == -INF)
    off = torch.where(on, (got.double() - x).abs(), torch.zeros(())) - ref.adjust_bound(x, 30 + 2 * r["scores"].double().abs(), BF16)
    assert off.max() <= 0


def test_adjust_of_infinities_and_nan():
    s = torch.tensor([[NAN, INF, -INF, NAN, 1.0, -1.0, INF, 0.0, -0.0]])
    allowed = torch.tensor([[0b111110110]], dtype=torch.int32)
    got = tk.adjust(s.cuda(), torch.arange(8).cuda(), 2.0, 0.5, 0.0, allowed=allowed.cuda())[0].tolist()
    assert got[0] == -INF and got[3] == -INF  # NaN where nothing is allowed
    assert got[1] == INF and got[2] == -INF and got[6] == INF
    assert got[4:6] == [0.0, -2.5] and got[7:] == [-0.5, 0.0]


def test_adjust_rows_for_all_and_dimensions():
    """One row of each thing for all rows of scores; scores of three dimensions and with strides."""
    g = gen(5)
    base = torch.randn((4, 5, 130), generator=g)
    scores = base.cuda()[:, :, 3:103]
    r = request(1, 100, 40, 6, True, True, F32, 6)
    got = tk.adjust(scores, r["previous"][0].cuda(), penalties=r["penalties"][0].cuda(), bias_tokens=r["bias_tokens"][0].cuda(),
                    bias=r["bias"][0].cuda(), allowed=r["allowed"][0].cuda())
    assert got.shape == (4, 5, 100)
    many = {k: None if v is None else v.expand(20, -1) for k, v in r.items()}
    many["scores"] = base[:, :, 3:103].reshape(20, 100)
    check_adjust(many, (1, 0, 0), got.reshape(20, 100), F32)


@pytest.mark.parametrize("vocab", [100, 9001])
def test_adjust_in_place_and_twice(vocab):
    r, numbers = request(3, vocab, 50, 5, True, True, BF16, 7), (1.0, 0.0, 0.0)
    want = adjusted(r, numbers)
    buf = torch.full((3, vocab + 5), 4.0, dtype=BF16, device="cuda")
    x = buf[:, 2:2 + vocab]
    x.copy_(r["scores"])
    got = tk.adjust(x, cuda(r["previous"]), penalties=cuda(r["penalties"]), bias_tokens=cuda(r["bias_tokens"]), bias=cuda(r["bias"]),
                    allowed=cuda(r["allowed"]), out=x)
    assert got is x and torch.equal(x, want)
    x.fill_(4.0)
    assert (buf == 4).all()
    assert torch.equal(adjusted(r, numbers), want)


@pytest.mark.parametrize("vocab", [3, 33, 200, 5001])
@pytest.mark.parametrize("dtype", [F32, F16])
def test_adjust_into_rows_that_start_anywhere(vocab, dtype):
    """Every place of an output's row in its 64 bytes; columns before, in and behind the units."""
    n, numbers = 33, (1.5, 0.25, 0.125)
    r = request(n, vocab, 40, 9, True, True, dtype, 8)
    for start in (0, 1, 7, 30):
        buf = torch.full((n * (vocab + 1) + 40,), 4.0, dtype=dtype, device="cuda")
        x = torch.as_strided(buf, (n, vocab), (vocab + 1, 1), start)
        check_adjust(r, numbers, adjusted(r, numbers, out=x), dtype)
        x.fill_(4.0)
        assert (buf == 4).all()


def test_adjust_one_token_all_the_time():
    """A text of one token, and rows that differ in nothing but their text's length."""
    n, vocab, length = 4, 3000, 20_000
    prev = torch.full((n, length), -1)
    for i, c in enumerate((0, 1, 777, length)):
        prev[i, :c] = 1234
    got = tk.adjust(torch.zeros((n, vocab), device="cuda"), prev.cuda(), 1.0, 0.5, 2.0 ** -4).cpu()
    assert got[:, 1234].tolist() == [0.0, -0.5625, -0.5 - 777 / 16, -0.5 - length / 16]
    got[:, 1234] = 0
    assert not got.any()


def test_adjust_refusals():
    s = torch.zeros((4, 70), device="cuda")
    i64 = torch.zeros((4, 3), dtype=torch.int64, device="cuda")
    for kw in (dict(previous=i64.float()), dict(previous=i64[:3]), dict(repetition=0.0), dict(repetition=-1.0), dict(repetition=NAN),
               dict(presence=INF), dict(penalties=torch.zeros((4, 2), device="cuda")), dict(bias=torch.zeros((4, 3), device="cuda")),
               dict(bias_tokens=i64, bias=torch.zeros((4, 2), device="cuda")), dict(bias_tokens=i64),
               dict(bias_tokens=i64, bias=torch.zeros((4, 3), device="cuda", dtype=BF16)),
               dict(allowed=torch.zeros((4, 2), dtype=torch.int32, device="cuda")),
               dict(allowed=torch.zeros((4, 3), dtype=torch.int64, device="cuda")),
               dict(out=torch.zeros((4, 70), dtype=BF16, device="cuda")), dict(out=torch.zeros((70, 4), device="cuda").t())):
        with pytest.raises(sp.SPError):
            tk.adjust(s, **kw)
    assert tk.adjust(s[:0], i64[:0]).shape == (0, 70)


# ------------------------------------------------------------------ distill

def lesson(n, vocab, k, dtype, teacher, seed, pad=0.0, tokens=torch.int64, by=3.0):
    """Scores, distinct tokens in no order, the teacher's logits, weights; a share of rows without
    entries and of entries without a token."""
    g = gen(seed)
    s = (torch.randn((n, vocab), generator=g) * by).to(dtype)
    tok = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(n)])
    if k > vocab:
        tok = torch.randint(vocab, (n, k), generator=g)
    t = (torch.randn((n, k), generator=g) * 2 + s.double().gather(1, tok.clamp(max=vocab - 1)).float() / 2).to(teacher)
    if pad:
        tok = torch.where(torch.rand((n, k), generator=g) < pad, -1, tok)
        tok[torch.rand(n, generator=g) < pad] = -1
        tok[0, 0] = vocab
    return s, tok.to(tokens), t, torch.rand(n, generator=g) + 0.5


def check_distill(s, tok, t, w, T, loss, grad, dtype):
    want, want_grad, loss_off, grad_off = ref.distill(s, tok, t, w, T)
    loss = loss.cpu().double()
    far = torch.isinf(want)
    assert torch.equal(loss[far], want[far])
    off = (loss - want).abs()[~far] - loss_off[~far] - want.abs()[~far] * UNIT[F32]
    assert off.numel() == 0 or (not torch.isnan(off).any() and off.max() <= 0), off.max()
    if grad is not None:
        grad = grad.cpu().double()
        off = (grad - want_grad).abs() - grad_off - (want_grad.abs() + grad_off) * UNIT[dtype] - TINY[dtype]
        assert not torch.isnan(off).any() and off.max() <= 0, off.max()


@pytest.mark.parametrize("n,vocab,k,dtype,teacher,T,pad,tokens", [
    (1, 1, 1, F32, F32, 1.0, 0.0, torch.int64),
    (3, 5, 3, BF16, F32, 2.0, 0.0, torch.int32),
    (4, 8, 8, F16, BF16, 1.0, 0.2, torch.int64),
    (16, 1000, 16, F32, F32, 1.0, 0.0, torch.int64),
    (33, 1001, 100, BF16, F16, 3.0, 0.3, torch.int32),
    (5, 2048, 1024, F32, BF16, 1.0, 0.3, torch.int64),
    (7, 10_007, 257, F16, F32, 0.5, 0.1, torch.int64),
    (2, 50_001, 64, BF16, F32, 1.0, 0.0, torch.int32),
    (300, 600, 5, F32, F32, 1.0, 0.3, torch.int64),
    (1, 131_072, 33, BF16, F32, 1.0, 0.0, torch.int64),
    (3, 70_003, 300, F32, F32, 4.0, 0.2, torch.int64),
])
def test_distill(n, vocab, k, dtype, teacher, T, pad, tokens):
    s, tok, t, w = lesson(n, vocab, k, dtype, teacher, n + vocab, pad, tokens)
    a = s.cuda(), tok.cuda(), t.cuda()
    check_distill(s, tok, t, w, T, tk.distill(*a, T), None, dtype)
    loss, grad = tk.distill_grad(*a, w.cuda(), T)
    assert grad.dtype == dtype and loss.dtype == F32
    check_distill(s, tok, t, w, T, loss, grad, dtype)
    if dtype != F32:
        loss, grad = tk.distill_grad(*a, w.cuda(), T, dtype=F32)
        check_distill(s, tok, t, w, T, loss, grad, F32)


@pytest.mark.parametrize("n,vocab", [(4, 300), (2, 40_000), (700, 3000)])
def test_tokens_listed_more_than_once(n, vocab):
    s, tok, t, w = lesson(n, vocab, 40, F32, F32, 9)
    tok[:, 5], tok[:, 17], tok[:, 39] = tok[:, 2], tok[:, 2], tok[:, 2]
    tok[1, :] = 7  # the same one everywhere
    loss, grad = tk.distill_grad(s.cuda(), tok.cuda(), t.cuda(), w.cuda())
    check_distill(s, tok, t, w, 1.0, loss, grad, F32)
    again = tk.distill_grad(s.cuda(), tok.cuda(), t.cuda(), w.cuda())
    assert torch.equal(loss, again[0]) and torch.equal(grad, again[1])


def test_tokens_that_meet_in_a_hash():
    """Tokens that are multiples of powers of two, neighbours, and a full list of them."""
    vocab = 1 << 20
    s = torch.randn((3, vocab), generator=gen(10))
    tok = torch.stack([torch.arange(1024) * 1024, torch.arange(1024), torch.arange(1024) * 512 + 1])
    t = torch.randn((3, 1024), generator=gen(11))
    w = torch.ones(3)
    check_distill(s, tok, t, w, 1.0, *tk.distill_grad(s.cuda(), tok.cuda(), t.cuda()), F32)


@pytest.mark.parametrize("n", [5, 600])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_infinities_and_nan(n, dtype):
    vocab, k = 900, 6
    s, tok, t, w = lesson(n, vocab, k, dtype, F32, 12)
    tok[0] = -1
    s[0, :] = NAN                 # no entries: not looked at
    t[1] = -INF                   # entries, none above -infinity
    s[1, 5] = INF
    s[2, tok[2, 3]] = -INF        # a teacher's column that the scores rule out: an infinite loss
    s[3] = -INF                   # a row that is masked everywhere
    t[4, 2] = -INF                # an entry that counts nothing, on a column that is ruled out
    s[4, tok[4, 2]] = -INF
    s[4, 100:200] = -INF
    s[4, tok[4, :2]] = 1.0
    loss, grad = tk.distill_grad(s.cuda(), tok.cuda(), t.cuda(), w.cuda())
    assert loss[:5].cpu().tolist()[:4] == [0.0, 0.0, INF, INF] and not grad[:2].any()
    check_distill(s, tok, t, w, 1.0, loss, grad, dtype)
    assert torch.equal(tk.distill(s.cuda(), tok.cuda(), t.cuda())[:4], loss[:4])
    s[4, 300] = NAN
    loss, grad = tk.distill_grad(s.cuda(), tok.cuda(), t.cuda(), w.cuda())
    assert torch.isnan(loss[4]) and torch.isnan(grad[4]).all() and not torch.isnan(grad[:4]).any()


@pytest.mark.parametrize("n,vocab", [(4, 500), (3, 60_000)])
def test_a_teacher_of_nan(n, vocab):
    """NaN of either sign among the entries, some of them of one token: a NaN loss, NaN in the teacher's columns."""
    s, tok, t, w = lesson(n, vocab, 10, F32, F32, 18)
    tok[:, 4] = tok[:, 7] = tok[:, 1]
    for i, bad in ((1, NAN), (2, -torch.tensor(NAN))):
        t[i, 7] = bad
    loss, grad = tk.distill_grad(s.cuda(), tok.cuda(), t.cuda(), w.cuda())
    assert torch.isnan(loss).cpu().tolist() == [False, True, True, False][:n]
    listed = torch.zeros((n, vocab), dtype=torch.bool).scatter_(1, tok, True)
    listed[[i for i in (0, 3) if i < n]] = False
    assert torch.equal(torch.isnan(grad).cpu(), listed)


@pytest.mark.parametrize("by", [1e-30, 1e4, 1e30])
def test_scores_of_any_size(by):
    """Far below and above where an exponential of the scores themselves would be a number."""
    s, tok, t, w = lesson(6, 700, 9, F32, F32, 13, by=by)
    t = t / t.abs().max() * 3
    check_distill(s, tok, t, w, 1.0, *tk.distill_grad(s.cuda(), tok.cuda(), t.cuda(), w.cuda()), F32)


@pytest.mark.parametrize("n,vocab", [(3, 1003), (600, 1003), (2, 200_003)])
def test_distill_in_place_with_strides_and_dimensions(n, vocab):
    s, tok, t, w = lesson(n, vocab, 20, BF16, F32, 14, 0.2)
    want = tk.distill_grad(s.cuda(), tok.cuda(), t.cuda(), 0.25, 2.0)
    check_distill(s, tok, t, torch.full((n,), 0.25), 2.0, *want, BF16)
    buf = torch.full((1, n, vocab + 9), 6.0, dtype=BF16, device="cuda")
    x = buf[:, :, 3:3 + vocab]
    x.copy_(s)
    wide = torch.stack([tok, tok], 2).cuda()[None, :, :, 0]
    loss, grad = tk.distill_grad(x, wide, t.cuda()[None], 0.25, 2.0, out=x)
    # (Not the same bits as above: a row's sums are taken in units that start where 64 aligned bytes of the
    # gradient do, so in another order; both are within what any order may be off.)
    assert grad is x
    check_distill(s, tok, t, torch.full((n,), 0.25), 2.0, loss[0], x[0], BF16)
    x.copy_(s)
    again = tk.distill_grad(x, wide, t.cuda()[None], 0.25, 2.0)
    x.fill_(6.0)
    assert (buf == 6).all()
    check_distill(s, tok, t, torch.full((n,), 0.25), 2.0, again[0][0], again[1][0], BF16)


@pytest.mark.parametrize("vocab", [5, 40, 129, 1001])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F32, F32), (F32, BF16), (F16, F32)])
def test_distill_gradient_that_starts_anywhere(vocab, dtype, out):
    """Every place of a gradient's row in its 64 bytes, with teacher's columns before, in and behind the units."""
    k = min(vocab, 30)
    s, tok, t, w = lesson(34, vocab, k, dtype, F32, 17)
    for start in (0, 1, 2, 5, 31):
        buf = torch.full((34 * (vocab + 1) + 40,), 6.0, dtype=out, device="cuda")
        x = torch.as_strided(buf, (34, vocab), (vocab + 1, 1), start)
        loss, grad = tk.distill_grad(s.cuda(), tok.cuda(), t.cuda(), w.cuda(), out=x)
        check_distill(s, tok, t, w, 1.0, loss, grad, out)
        x.fill_(6.0)
        assert (buf == 6).all()


def test_distill_gradient_against_differences():
    """Central differences of the losses in 64 bits at h = 2^-8 against the kernel's gradient.  Their own
    error is h^2 / 6 times w T^2 times a third derivative of the logarithm of the sum of exponentials of
    scores / T, which is 1 / T^3 times a third central moment of a truth value: below h^2 / 6 * w / T."""
    s, tok, t, w = lesson(4, 40, 6, F32, F32, 15)
    T, h = 2.0, 2.0 ** -8
    _, grad = tk.distill_grad(s.cuda(), tok.cuda(), t.cuda(), w.cuda(), T)
    num = torch.zeros((4, 40), dtype=torch.float64)
    for v in range(40):
        e = torch.zeros(40, dtype=torch.float64)
        e[v] = h
        up, down = (ref.distill(s.double() + d, tok, t, w, T)[0] for d in (e, -e))
        num[:, v] = w.double() * (up - down) / (2 * h)
    off = ref.distill(s, tok, t, w, T)[3] + num.abs() * UNIT[F32] + h * h / 6 * w.double()[:, None] / T
    assert ((grad.cpu().double() - num).abs() <= off).all()


def test_distill_refusals():
    s, tok, t, w = (x.cuda() for x in lesson(4, 50, 3, F32, F32, 16))
    for call in (lambda: tk.distill(s, tok[:3], t[:3]), lambda: tk.distill(s, tok, t[:, :2]), lambda: tk.distill(s, tok, t, 0.0),
                 lambda: tk.distill(s, tok, t, NAN), lambda: tk.distill(s, tok.float(), t), lambda: tk.distill(s.double(), tok, t),
                 lambda: tk.distill(s, tok[:, :0], t[:, :0]), lambda: tk.distill(s, tok.repeat(1, 400), t.repeat(1, 400)),
                 lambda: tk.distill_grad(s, tok, t, w[:3]), lambda: tk.distill_grad(s, tok, t, w.double()),
                 lambda: tk.distill_grad(s, tok, t, dtype=torch.int32),
                 lambda: tk.distill_grad(s, tok, t, out=torch.zeros((4, 51), device="cuda"))):
        with pytest.raises(sp.SPError):
            call()
    loss, grad = tk.distill_grad(s[:0], tok[:0], t[:0])
    assert loss.shape == (0,) and grad.shape == (0, 50)
