"""The plain implementations themselves, on values worked out by hand."""
import math

import pytest
import torch

from tests import scores_reference as ref


def test_rows_in_4_bits():
    x = torch.zeros((1, 40))
    x[0, :5] = torch.tensor([1.0, -6.0, 0.25, 7.9, 0.75])  # scale 1: ties to even codes, 7.9 to 6
    x[0, 32:34] = torch.tensor([2.0 ** -126, -(2.0 ** -149)])  # below the smallest scale's 4
    q, s = ref.quantize4(x)
    assert q.shape == (1, 32) and s.tolist() == [[127, 0]]
    assert ref.values4(q, s)[0, :5].tolist() == [1.0, -6.0, 0.0, 6.0, 1.0]
    assert ref.values4(q, s)[0, 32:36].tolist() == [2.0 ** -126, -0.0, 0.0, 0.0]
    assert q[0, 0].item() == 0xF2


@pytest.mark.parametrize("a,byte", [(2.0 ** -149, 0), (2.0 ** -125, 0), (2.0 ** -124, 1), (3.99, 126), (4.0, 127), (2.0 ** 127, 252),
                                    (math.inf, 255), (math.nan, 255), (0.0, 0)])
def test_scales(a, byte):
    assert ref.quantize4(torch.tensor([[0.0, a]]))[1].item() == byte


def test_values_and_codes_are_inverse():
    codes = torch.arange(256, dtype=torch.uint8)[None, :].expand(1, 256)
    scales = torch.arange(1, 17, dtype=torch.uint8)[None, :] * 15
    assert torch.equal(ref.quantize4(ref.values4(codes, scales))[0], codes)


def test_adjust():
    s = torch.tensor([[2.0, -2.0, 1.0, 0.5, math.nan]])
    out, _ = ref.adjust(s, torch.tensor([[0, 1, 1, -1, 9]]), (2.0, 0.25, 0.5), None, torch.tensor([[3, 2, 3, -1]]),
                        torch.tensor([[5.0, 1.0, -1.0, 7.0]]), torch.tensor([[0b01111]]))
    assert out.tolist() == [[1.0 - 0.75, -4.0 - 1.25, 2.0, -0.5, -math.inf]]


def test_distill_against_autograd():
    g = torch.Generator().manual_seed(1)
    s = (torch.randn((3, 50), generator=g) * 3).double().requires_grad_()
    tok = torch.tensor([[3, 7, 49, -1], [0, 0, 5, 6], [-1, 50, -7, -1]])
    t = torch.randn((3, 4), generator=g) * 2
    w, T = torch.tensor([0.5, 2.0, 1.0]), 2.0
    loss, grad, _, _ = ref.distill(s.detach(), tok, t, w, T)
    total = 0
    for i in range(2):
        live = (tok[i] >= 0) & (tok[i] < 50)
        p = torch.softmax(t[i][live].double() / T, 0)
        mine = T * T * (p * (p.log() - torch.log_softmax(s[i] / T, 0)[tok[i][live]])).sum()
        assert abs(mine.item() - loss[i].item()) < 1e-12
        total = total + w[i] * mine
    total.backward()
    assert loss[2] == 0 and torch.allclose(s.grad, grad, atol=1e-14)
