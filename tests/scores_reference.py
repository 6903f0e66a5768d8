"""Plain implementations in 64 bits of the operators on rows in 4 bits and on scores, and the error
bounds that their kernels' arithmetic allows.  Nothing here uses the library."""
import math

import torch

from tests.rows_reference import TINY, U32, UNIT

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # by code; an even code has an even last bit
INF = math.inf


# ------------------------------------------------------------------ rows in 4 bits

def quantize4(x):
    """Bytes [n, blocks * 16] and scales [n, blocks] of the rows of x (finite or not)."""
    n, dim = x.shape
    blocks = (dim + 31) // 32
    padded = torch.zeros((n, blocks * 32), dtype=torch.float64)
    padded[:, :dim] = x.double()
    b = padded.view(n, blocks, 32)
    finite = torch.isfinite(b).all(2)
    b = torch.where(finite[..., None], b, torch.zeros((), dtype=torch.float64))
    amax = b.abs().amax(2)
    e = torch.full(amax.shape, -127, dtype=torch.int64)
    for i in range(-126, 126):  # floor(log2(amax)) - 2, without a logarithm's rounding
        e[amax >= 2.0 ** (i + 2)] = i
    y = b / (2.0 ** e.double())[..., None]
    distance = (y.abs()[..., None] - torch.tensor(MAGNITUDES, dtype=torch.float64)).abs()
    distance[..., 1::2] = torch.nextafter(distance[..., 1::2], torch.tensor(INF, dtype=torch.float64))  # ties: even codes
    code = distance.argmin(-1) | torch.signbit(y).long() << 3
    scales = torch.where(finite, e + 127, torch.full_like(e, 255))
    code = torch.where(finite[..., None], code, torch.zeros_like(code)).view(n, -1)
    return (code[:, 0::2] | code[:, 1::2] << 4).to(torch.uint8), scales.to(torch.uint8)


def values4(q, scales):
    """The values that rows of bytes and scales stand for."""
    code = torch.stack([q & 15, q >> 4], 2).reshape(q.shape[0], -1).long()
    v = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float64)[code]
    s = 2.0 ** (scales.double() - 127)
    s = torch.where(scales == 255, torch.full_like(s, math.nan), s)
    return v * s.repeat_interleave(32, 1)


def product4(x, xs, w, ws):
    """The products and the bound of what k additions in fp32 may be off, each by a unit in the last
    place (matrix instructions may cut off where others round)."""
    a, b = values4(x, xs), values4(w, ws)
    return a @ b.t(), (a.shape[1] + 2) * 2 * U32 * (a.abs() @ b.abs().t())


# ------------------------------------------------------------------ adjusted scores

def adjust(scores, previous=None, numbers=(1.0, 0.0, 0.0), penalties=None, bias_tokens=None, bias=None, allowed=None):
    """Element by element, and the sum of the magnitudes of the terms of each."""
    n, vocab = scores.shape
    out, size = scores.double().clone(), scores.double().abs()
    for i in range(n):
        r, p, f = penalties[i].double().tolist() if penalties is not None else numbers
        counts = {}
        for t in previous[i].tolist() if previous is not None else ():
            if 0 <= t < vocab:
                counts[t] = counts.get(t, 0) + 1
        for t, c in counts.items():
            s = out[i, t].item()
            y = s / r if s > 0 else s * r
            out[i, t] = y - (p + f * c)
            size[i, t] = abs(y) + abs(p) + abs(f * c)
        last = {}
        for j, t in enumerate(bias_tokens[i].tolist() if bias_tokens is not None else ()):
            if 0 <= t < vocab:
                last[t] = bias[i, j].item()
        for t, b in last.items():
            out[i, t] += b
            size[i, t] += abs(b)
        if allowed is not None:
            words = allowed[i].tolist()
            for v in range(vocab):
                if not words[v // 32] >> (v % 32) & 1:
                    out[i, v] = -INF
    return out, size


def adjust_bound(want, size, dtype):
    """Five operations in fp32, each rounding something no larger than the terms' magnitudes (a little
    more by the roundings before), then the output's rounding."""
    size = torch.where(torch.isfinite(size), size, torch.zeros_like(size))
    w = torch.where(torch.isfinite(want), want.abs(), torch.zeros_like(want))
    return 6 * U32 * size + w * UNIT[dtype] + TINY[dtype]


# ------------------------------------------------------------------ distillation

def distill(scores, tokens, teacher, weight, T):
    """Loss and gradient [n], [n, vocab], and bounds of what fp32 may be off in them (before the
    gradient's last rounding).

    With U = 2^-24: a softmax's exponent is (v - top) * c with c = log2(e) / T: a difference, a product
    and c itself, off by 4 U of its size a at most, and the exponential by 3 U more: a term is within
    r(a) = U (4 a + 3) of itself.  A sum of them passes at most vocab / 64 + 100 additions and 60 joins,
    each of which scales by another exponential: the differences of its exponents add up to the largest
    a, so all of them cost U (4 a + 4 * 60).  Exponentials below 2^-126 of the largest are 0: as many of
    them as there are columns change a sum by less than U, and a column's gradient by w T 2^-126."""
    n, vocab = scores.shape
    loss = torch.zeros(n, dtype=torch.float64)
    grad = torch.zeros((n, vocab), dtype=torch.float64)
    loss_off, grad_off = torch.zeros_like(loss), torch.zeros_like(grad)
    for i in range(n):
        tok = tokens[i].long()
        live = (tok >= 0) & (tok < vocab)
        t = torch.where(live, teacher[i].double() / T, torch.full(tok.shape, -INF, dtype=torch.float64))
        if not live.any() or t.max() == -INF:
            continue
        p = torch.softmax(t, 0)
        some = p > 0
        z = scores[i].double() / T
        dead = bool((z == -INF).all())
        q = torch.zeros_like(z) if dead else torch.softmax(z, 0)
        log_q = torch.full_like(z, -INF) if dead else torch.log_softmax(z, 0)
        at = log_q[tok.clamp(0, vocab - 1)]
        loss[i] = T * T * (p * (torch.log(p) - at))[some].sum()
        grad[i] = q
        grad[i].index_add_(0, tok[live], -p[live])

        def softmax_off(z, terms):
            a = torch.where(torch.isfinite(z), (z.max() - z) / math.log(2), torch.zeros_like(z))
            reach = min(a.max().item(), 200.0)  # (terms past 2^-200 of the sum count nothing)
            total = U32 * (4 * reach + 4 * 60 + terms / 64 + 101 + 4 * reach + 3)
            return U32 * (4 * a + 3) + total + 3 * U32, total

        p_off, teacher_off = softmax_off(t, len(t))
        q_off, total_off = (torch.zeros_like(z), 0.0) if dead else softmax_off(z, vocab)
        # logarithms: the difference over T, the sum's logarithm (two units), their difference
        log_p_off = U32 * (4 * (t.max() - t) + 4 * math.log(len(t) + 1) + 4) + teacher_off
        z_at = z[tok.clamp(0, vocab - 1)]
        log_q_off = U32 * (4 * (z.max() - z_at).abs() + 4 * math.log(vocab + 1) + 4) + total_off
        terms = p * (torch.log(p).abs() + at.abs())
        off = p * (log_p_off + log_q_off) + terms * (p_off + (len(t) + 8) * U32)
        loss_off[i] = T * T * off[some & torch.isfinite(at)].sum()
        mass = torch.zeros_like(z).index_add_(0, tok[live], p[live])
        mass_off = torch.zeros_like(z).index_add_(0, tok[live], (p * (p_off + (len(t) + 4) * U32))[live])
        w = abs(float(weight[i])) * T
        grad[i] *= float(weight[i]) * T
        grad_off[i] = w * (q * q_off + mass_off + 6 * U32 * (q + mass) + 2.0 ** -126)
    return loss, grad, loss_off + 1e-44, grad_off
