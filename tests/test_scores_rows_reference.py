"""The implementations for many rows at once against those row by row, and what they notice."""
import math

import pytest
import torch

from tests import scores_reference as one
from tests import scores_rows_reference as many
from tests.rows_reference import UNIT


def gen(seed):
    return torch.Generator().manual_seed(seed)


def lesson(n=30, vocab=70, k=9, seed=1):
    g = gen(seed)
    s, t = torch.randn((n, vocab), generator=g) * 3, torch.randn((n, k), generator=g) * 2
    tok = torch.randint(-1, vocab + 1, (n, k), generator=g)
    tok[3] = -1
    tok[4] = 5
    return s, tok, t, torch.rand(n, generator=g) + 0.5


@pytest.mark.parametrize("T", [1.0, 3.0])
def test_distill(T):
    s, tok, t, w = lesson()
    for a, b in zip(one.distill(s, tok, t, w, T), many.distill(s, tok, t, w, T)):
        assert torch.allclose(a, b, rtol=1e-12, atol=1e-16)


def test_rows_without_entries_may_hold_anything():
    s, tok, t, w = lesson()
    want = many.distill(s, tok, t, w, 1.0)
    s[3] = math.nan
    for a, b in zip(want, many.distill(s, tok, t, w, 1.0)):
        assert torch.equal(a, b)
    assert want[0][3] == 0 and not want[1][3].any()


def test_another_rows_entries_are_noticed():
    """What a kernel that kept a row's scores, tokens or masses for the next would return is far outside the bounds."""
    s, tok, t, w = lesson()
    loss, grad, loss_off, grad_off = many.distill(s, tok, t, w, 1.0)
    live = (tok >= 0).any(1)
    live[4] = False  # (one token in all entries: its mass is 1, whatever the teacher's logits)
    for args in ((s.roll(1, 0), tok, t), (s, tok.roll(1, 0), t), (s, tok, t.roll(1, 0))):
        l, g, _, _ = many.distill(*args, w, 1.0)
        assert (((g - grad).abs() > grad_off + grad.abs() * UNIT[torch.bfloat16]).any(1) | ~live).all()
        assert ((l - loss).abs() > loss_off)[live].double().mean() > 0.9


@pytest.mark.parametrize("per_row", [False, True])
def test_adjust(per_row):
    n, vocab = 12, 100
    g = gen(2)
    r = dict(scores=torch.randn((n, vocab), generator=g), previous=torch.randint(-1, vocab + 1, (n, 200), generator=g),
             penalties=torch.rand((n, 3), generator=g) + 0.5 if per_row else None, bias_tokens=torch.randint(-1, vocab, (n, 60), generator=g),
             bias=torch.randn((n, 60), generator=g), allowed=torch.randint(-2 ** 31, 2 ** 31, (n, 4), generator=g).int())
    numbers = (1.3, 0.25, 0.125)
    for drop in ((), ("previous",), ("bias", "bias_tokens"), ("allowed",)):
        kw = {k: None if k in drop else v for k, v in r.items()}
        kw["numbers"] = numbers
        a, b = one.adjust(**kw), many.adjust(**kw)
        for x, y in zip(a, b):
            assert torch.equal(torch.isinf(x), torch.isinf(y))
            assert torch.allclose(x[torch.isfinite(x)], y[torch.isfinite(y)], rtol=1e-14)
