"""The plain implementations of scores_reference.py for many rows at once, on any device: the same formulas
and the same bounds, whole rows as tensors of 64 bits.  Nothing here uses the library."""
import math

import torch

from tests.rows_reference import U32

INF = math.inf
LN2 = math.log(2)


def distill(scores, tokens, teacher, weight, T):
    """Loss and gradient [n], [n, vocab] and their bounds, of rows whose scores are finite where they have
    entries (rows without any may hold anything)."""
    n, vocab = scores.shape
    tok = tokens.long()
    live = (tok >= 0) & (tok < vocab)
    at = tok.clamp(0, vocab - 1)
    alive = live.any(1)
    t = torch.where(live, teacher.double() / T, torch.full((), -INF, dtype=torch.float64, device=tok.device))
    t = torch.where(alive[:, None], t, torch.zeros_like(t))
    p = torch.softmax(t, 1)
    p = torch.where(live, p, torch.zeros_like(p))
    z = torch.where(alive[:, None], scores.double() / T, torch.zeros((), dtype=torch.float64, device=tok.device))
    q, z_at = torch.softmax(z, 1), z.gather(1, at)
    log_q = torch.log_softmax(z, 1).gather(1, at)
    log_p = torch.where(live, torch.log_softmax(t, 1), torch.zeros_like(t))
    some = p > 0
    loss = T * T * torch.where(some, p * (log_p - log_q), torch.zeros_like(p)).sum(1)
    mass = torch.zeros_like(z).scatter_add_(1, at, p)

    def softmax_off(z, terms):
        top = z.amax(1, keepdim=True)
        a = torch.where(torch.isfinite(z), (top - z) / LN2, torch.zeros_like(z))
        reach = a.amax(1, keepdim=True).clamp(max=200.0)
        total = U32 * (4 * reach + 4 * 60 + terms / 64 + 101 + 4 * reach + 3)
        return U32 * (4 * a + 3) + total + 3 * U32, total

    k = tok.shape[1]
    p_off, teacher_off = softmax_off(t, k)
    q_off, total_off = softmax_off(z, vocab)
    far = torch.where(live, t.amax(1, keepdim=True) - t, torch.zeros_like(t))
    log_p_off = U32 * (4 * far + 4 * math.log(k + 1) + 4) + teacher_off
    log_q_off = U32 * (4 * (z.amax(1, keepdim=True) - z_at) + 4 * math.log(vocab + 1) + 4) + total_off
    off = p * (log_p_off + log_q_off) + p * (log_p.abs() + log_q.abs()) * (p_off + (k + 8) * U32)
    loss_off = T * T * torch.where(some, off, torch.zeros_like(off)).sum(1)
    mass_off = torch.zeros_like(z).scatter_add_(1, at, p * (p_off + (k + 4) * U32))
    w = weight.double()[:, None].abs() * T
    grad = (q - mass) * weight.double()[:, None] * T
    grad_off = w * (q * q_off + mass_off + 6 * U32 * (q + mass) + 2.0 ** -126)
    none = torch.zeros((), dtype=torch.float64, device=tok.device)
    return (torch.where(alive, loss, none), torch.where(alive[:, None], grad, none),
            torch.where(alive, loss_off, none) + 1e-44, torch.where(alive[:, None], grad_off, none))


def adjust(scores, previous=None, numbers=(1.0, 0.0, 0.0), penalties=None, bias_tokens=None, bias=None, allowed=None):
    """The adjusted scores and the sum of the magnitudes of the terms of each."""
    n, vocab = scores.shape
    x = scores.double()
    size = x.abs()
    if previous is not None:
        tok = previous.long()
        count = torch.zeros((n, vocab + 1), dtype=torch.float64, device=x.device)
        count.scatter_add_(1, torch.where((tok >= 0) & (tok < vocab), tok, vocab), torch.ones(tok.shape, dtype=torch.float64, device=x.device))
        count = count[:, :vocab]
        r, p, f = penalties.double()[:, :, None].unbind(1) if penalties is not None else numbers
        y = torch.where(x > 0, x / r, x * r)
        p = torch.as_tensor(p, dtype=torch.float64, device=x.device)
        x = torch.where(count > 0, y - (p + f * count), x)
        size = torch.where(count > 0, y.abs() + p.abs() + (f * count).abs(), size)
    if bias is not None:
        tok = bias_tokens.long()
        last = torch.full((n, vocab + 1), -1, dtype=torch.int64, device=x.device)
        entry = torch.arange(tok.shape[1], device=x.device).expand(n, -1)
        last.scatter_reduce_(1, torch.where((tok >= 0) & (tok < vocab), tok, vocab), entry, "amax")
        last = last[:, :vocab]
        by = torch.where(last >= 0, bias.double().gather(1, last.clamp(min=0)), torch.zeros_like(x))
        x, size = x + by, size + by.abs()
    if allowed is not None:
        on = (allowed.long()[:, :, None] >> torch.arange(32, device=x.device) & 1).view(n, -1)[:, :vocab] > 0
        x = torch.where(on, x, torch.full((), -INF, dtype=torch.float64, device=x.device))
    return x, size
