"""Refusals of the row operators' C entry points: reported with a text before any device
work, so they run without a GPU."""
import ctypes as C

import pytest

from paper_2205_04702_amd import scratchpipe as sp
from paper_2205_04702_amd import tokens as tk

A = 0x10000  # an address that no refused call touches
NAN, INF = float("nan"), float("inf")


def call(name, base, **over):
    L = tk._load()
    unknown = set(over) - set(base)
    assert not unknown
    st = getattr(L, name)(*{**base, **over}.values())
    return st, sp.sp_last_error(None)


LOOKUP = dict(tokens=A, token_type=tk.SP_I64, n=8, table=A, table_type=tk.SP_BF16, rows=100, dim=16,
              table_ld=16, scale=1.0, p=0.0, seed=0, offset=0, out=A, out_type=tk.SP_F32, out_ld=16,
              stream=0)
GRAD = dict(tokens=A, token_type=tk.SP_I64, n=1000, grad=A, grad_type=tk.SP_BF16, dim=16, grad_ld=16,
            scale=1.0, p=0.0, seed=0, offset=0, out=A, out_type=tk.SP_F32, rows=100, out_ld=16,
            accumulate=0, workspace=A, workspace_bytes=1 << 30, stream=0)
DROPOUT = dict(x=A, type=tk.SP_F32, n=8, dim=16, x_ld=16, residual=0, residual_ld=0, p=0.5, seed=0,
               offset=0, out=A, out_ld=16, stream=0)
WRITE = dict(x=A, type=tk.SP_F32, n=8, dim=64, x_ld=64, index=A, index_type=tk.SP_I32, group=32, q=A,
             kind=tk.SP_I8, slots=10, q_ld=64, scales=A, scales_ld=2, stream=0)
READ = dict(q=A, kind=tk.SP_I8, slots=10, dim=64, q_ld=64, scales=A, scales_ld=2, group=32, index=A,
            index_type=tk.SP_I32, n=8, out=A, out_type=tk.SP_F32, out_ld=64, stream=0)
PRODUCT = dict(x=A, x_scales=A, m=4, x_ld=64, w=A, w_scales=A, n=8, w_ld=64, k=64, out=A,
               out_type=tk.SP_BF16, out_ld=8, workspace=0, workspace_bytes=0, stream=0)


@pytest.mark.parametrize("name,base,over,needle", [
    ("sp_lookup", LOOKUP, dict(token_type=tk.SP_F32), "token type"),
    ("sp_lookup", LOOKUP, dict(table_type=tk.SP_I8), "element type"),
    ("sp_lookup", LOOKUP, dict(out_type=9), "element type"),
    ("sp_lookup", LOOKUP, dict(n=-1), "tokens"),
    ("sp_lookup", LOOKUP, dict(n=1 << 31), "tokens"),
    ("sp_lookup", LOOKUP, dict(rows=1 << 31), "rows"),
    ("sp_lookup", LOOKUP, dict(dim=0), "dim"),
    ("sp_lookup", LOOKUP, dict(dim=(1 << 20) + 1, table_ld=1 << 21, out_ld=1 << 21), "dim"),
    ("sp_lookup", LOOKUP, dict(p=1.0), "p 1"),
    ("sp_lookup", LOOKUP, dict(p=-0.1), "p -0.1"),
    ("sp_lookup", LOOKUP, dict(p=NAN), "p nan"),
    ("sp_lookup", LOOKUP, dict(p=1 - 2.0 ** -18), "p "),
    ("sp_lookup", LOOKUP, dict(tokens=0), "null tokens"),
    ("sp_lookup", LOOKUP, dict(table=0), "null table"),
    ("sp_lookup", LOOKUP, dict(out=0), "null output"),
    ("sp_lookup", LOOKUP, dict(tokens=A + 4), "aligned"),
    ("sp_lookup", LOOKUP, dict(table=A + 1), "aligned"),
    ("sp_lookup", LOOKUP, dict(table_ld=15), "stride"),
    ("sp_lookup", LOOKUP, dict(out_ld=-16), "stride"),
    ("sp_lookup_grad", GRAD, dict(token_type=0), "token type"),
    ("sp_lookup_grad", GRAD, dict(grad_type=tk.SP_I64), "element type"),
    ("sp_lookup_grad", GRAD, dict(grad=0), "null gradient"),
    ("sp_lookup_grad", GRAD, dict(out=0), "null output"),
    ("sp_lookup_grad", GRAD, dict(rows=-1), "rows"),
    ("sp_lookup_grad", GRAD, dict(p=INF), "p inf"),
    ("sp_lookup_grad", GRAD, dict(grad_ld=8), "stride"),
    ("sp_lookup_grad", GRAD, dict(workspace=0), "workspace"),
    ("sp_lookup_grad", GRAD, dict(workspace_bytes=8), "workspace"),
    ("sp_lookup_grad", GRAD, dict(workspace=A + 8), "workspace"),
    ("sp_dropout", DROPOUT, dict(type=tk.SP_I32), "element type"),
    ("sp_dropout", DROPOUT, dict(p=1.5), "p 1.5"),
    ("sp_dropout", DROPOUT, dict(dim=0), "dim"),
    ("sp_dropout", DROPOUT, dict(x=0), "null input"),
    ("sp_dropout", DROPOUT, dict(residual=A, residual_ld=4), "stride"),
    ("sp_dropout", DROPOUT, dict(residual=A + 2, residual_ld=16), "aligned"),
    ("sp_cache_write", WRITE, dict(index_type=tk.SP_F16), "index type"),
    ("sp_cache_write", WRITE, dict(kind=tk.SP_BF16), "cache type"),
    ("sp_cache_write", WRITE, dict(group=0), "group"),
    ("sp_cache_write", WRITE, dict(group=4), "group"),
    ("sp_cache_write", WRITE, dict(group=48), "group"),
    ("sp_cache_write", WRITE, dict(group=128), "group"),
    ("sp_cache_write", WRITE, dict(scales_ld=1), "stride"),
    ("sp_cache_write", WRITE, dict(q_ld=63), "stride"),
    ("sp_cache_write", WRITE, dict(index=0, n=11), "without an index"),
    ("sp_cache_write", WRITE, dict(scales=0), "null scales"),
    ("sp_cache_read", READ, dict(q=0), "null cache"),
    ("sp_cache_read", READ, dict(out_type=tk.SP_F8), "element type"),
    ("sp_cache_read", READ, dict(slots=-1), "slots"),
    ("sp_cache_read", READ, dict(out=0), "null rows"),
    ("sp_product", PRODUCT, dict(k=0), "k 0"),
    ("sp_product", PRODUCT, dict(k=131072), "k 131072"),
    ("sp_product", PRODUCT, dict(m=-1), "outputs"),
    ("sp_product", PRODUCT, dict(x=0), "null x"),
    ("sp_product", PRODUCT, dict(w_scales=0), "null w's scales"),
    ("sp_product", PRODUCT, dict(out_ld=7), "stride"),
    ("sp_product", PRODUCT, dict(w_ld=63), "stride"),
    ("sp_product", PRODUCT, dict(out_type=tk.SP_I8), "element type"),
])
def test_refused(name, base, over, needle):
    st, text = call(name, base, **over)
    assert st == sp.SP_ERR_INVALID_ARG
    assert needle in text


@pytest.mark.parametrize("name,base,over", [
    ("sp_lookup", LOOKUP, dict(n=0, tokens=0, out=0)),
    ("sp_lookup_grad", GRAD, dict(rows=0, out=0)),
    ("sp_dropout", DROPOUT, dict(n=0, x=0, out=0)),
    ("sp_cache_write", WRITE, dict(n=0, index=0, x=0)),
    ("sp_cache_read", READ, dict(n=0, index=0, out=0)),
    ("sp_product", PRODUCT, dict(m=0, x=0, out=0)),
    ("sp_product", PRODUCT, dict(n=0, w=0, out=0)),
])
def test_nothing_to_do_is_no_error(name, base, over):
    assert call(name, base, **over)[0] == sp.SP_OK


def test_workspace_sizes():
    """No workspace for a handful of tokens; otherwise room for the entries at least, and no
    more for a table of any size."""
    L = tk._load()
    b = C.c_int64(-1)
    assert L.sp_lookup_grad_workspace(8, 1000, 64, C.byref(b)) == sp.SP_OK and b.value == 0
    for n in (4000, 100_000, 1_000_000):
        assert L.sp_lookup_grad_workspace(n, 1000, 64, C.byref(b)) == sp.SP_OK
        few = b.value
        assert few >= 8 * n
        assert L.sp_lookup_grad_workspace(n, 2 ** 31 - 1, 64, C.byref(b)) == sp.SP_OK
        assert b.value == few
    assert L.sp_lookup_grad_workspace(-1, 1000, 64, C.byref(b)) == sp.SP_ERR_INVALID_ARG
    assert L.sp_product_workspace(4, 4, 0, C.byref(b)) == sp.SP_ERR_INVALID_ARG


def test_binding_refuses_host_tensors():
    import torch
    with pytest.raises(sp.SPError, match="GPU"):
        tk.lookup(torch.zeros(3, dtype=torch.int64), torch.zeros((4, 8)))
    with pytest.raises(sp.SPError, match="GPU"):
        tk.quantize(torch.zeros((4, 8)))
