"""tests/product_forms.py cuts products as the library does: its parts of k are those that the
library asks a workspace for."""
import ctypes as C
import random

from paper_2205_04702_amd import scratchpipe as sp
from paper_2205_04702_amd import tokens as tk
from tests.product_forms import cut


def test_parts_of_k_are_the_library_s():
    L, rng, b, seen = tk._load(), random.Random(11), C.c_int64(), set()
    for _ in range(30_000):
        m, n, k = (int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 15)), int(2 ** rng.uniform(0, 15)))
        tile, parts = cut(m, n, k)
        assert L.sp_product_workspace(m, n, k, C.byref(b)) == sp.SP_OK
        assert b.value == (4 * m * n * parts if parts > 1 else 0), (m, n, k)
        seen.add((tile, parts))
    assert len(seen) >= 20
