"""Which form of the product a call takes: the library's estimate of how to cut m x n x k into
tiles and parts of k, written down again, so that tests can name the forms they run."""
import math

TILES = [(256, 256), (128, 128), (64, 128), (64, 64), (32, 64)]
# us of a step of 64 columns with the card mostly idle, busy, and of a tile before and after
_COST = [(0.56, 0.86, 7.3), (0.33, 0.31, 1.8), (0.22, 0.24, 1.0), (0.165, 0.19, 0.6), (0.155, 0.16, 0.5)]


def cut(m, n, k):
    """(rows and columns of a tile, parts of k)."""
    steps = (k + 63) // 64
    best, least = None, math.inf
    for (bm, bn), (idle, busy, fixed) in zip(TILES, _COST):
        tiles = -(-m // bm) * -(-n // bn)
        for parts in (1, 2, 4, 8, 16):
            if parts > 1 and (steps < 4 * parts or tiles * parts > 1024):
                break
            blocks = tiles * parts
            us = -(-blocks // 256) * (fixed + (idle if blocks <= 192 else busy) * -(-steps // parts))
            if parts > 1:
                us += 3.0 + m * n * 4.0 * (2 * parts) / 4e6
            if us < least:
                least, best = us, ((bm, bn), parts)
    return best
