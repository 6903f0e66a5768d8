"""Plain implementations in 64 bits of the operators on token tables and 8-bit rows, and the
error bounds that their kernels' arithmetic allows.  Nothing here uses the library."""
import numpy as np
import torch

# half a unit in the last place of 1, and half the smallest subnormal
UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
U32 = 2.0 ** -24


def philox(counter, key):
    """Philox 4x32-10 in Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        x, y = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(y >> 32) ^ c[1] ^ k[0], y % 2 ** 32, (x >> 32) ^ c[3] ^ k[1], x % 2 ** 32]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def dropped_below(p):
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def keep_mask(n, dim, p, seed, offset):
    """[n, dim] booleans, element by element from the generator."""
    octets = (dim + 7) // 8
    bits = np.zeros((n, octets * 8), np.int64)
    for i in range(n):
        for o in range(octets):
            w = philox([o, i, offset % 2 ** 32, offset >> 32], [seed % 2 ** 32, seed >> 32])
            for e in range(8):
                bits[i, o * 8 + e] = w[e // 2] >> (16 * (e % 2)) & 0xFFFF
    return torch.from_numpy(bits[:, :dim] >= dropped_below(p))


def keep_factor(p):
    return 65536.0 / (65536 - dropped_below(p))


def drop(x, p, seed, offset):
    """Dropout of a float64 matrix."""
    if dropped_below(p) == 0:
        return x
    keep = keep_mask(x.shape[0], x.shape[1], p, seed, offset)
    return torch.where(keep, x * keep_factor(p), torch.zeros((), dtype=x.dtype))


def lookup(tokens, table, scale=1.0, p=0.0, seed=0, offset=0):
    t = tokens.reshape(-1).long()
    live = (t >= 0) & (t < table.shape[0])
    w = table.double()
    if not w.shape[0]:
        w = torch.zeros((1, table.shape[1]), dtype=torch.float64)
    x = torch.where(live[:, None], w[torch.where(live, t, torch.zeros_like(t))] * scale,
                    torch.zeros((), dtype=torch.float64))
    return drop(x, p, seed, offset)


def lookup_grad(tokens, grad, rows, scale=1.0, p=0.0, seed=0, offset=0):
    """The sums, the sums of magnitudes and the number of terms of each row."""
    t = tokens.reshape(-1).long()
    live = (t >= 0) & (t < rows)
    g = drop(grad.reshape(t.shape[0], grad.shape[-1]).double(), p, seed, offset)[live] * scale
    total = torch.zeros((rows, grad.shape[-1]), dtype=torch.float64)
    size, count = torch.zeros_like(total), torch.zeros(rows, 1, dtype=torch.float64)
    total.index_add_(0, t[live], g)
    size.index_add_(0, t[live], g.abs())
    count.index_add_(0, t[live], torch.ones((int(live.sum()), 1), dtype=torch.float64))
    return total, size, count


def round_e4m3(y):
    """float64 values of magnitude at most 448 to the nearest with 4 exponent and 3 mantissa bits."""
    exponent = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(exponent - 3)
    return torch.round(y / step) * step


TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def group_scales(x, group, kind):
    """float64 scale of each group of a matrix of finite values."""
    n, d = x.shape
    return x.double().abs().view(n, d // group, group).amax(-1) / TOP[kind]
