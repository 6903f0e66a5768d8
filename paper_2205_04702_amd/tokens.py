"""Operators on token tables and 8-bit rows (include/scratchpipe.h, second part).

Argument marshalling only, as in scratchpipe.py: torch tensors on the GPU in, kernels
of the HIP library on the current stream (or the one given), torch tensors out.

    rows = lookup(tokens, table, scale, p, seed, offset)        # training
    table_grad = lookup_grad(tokens, rows_grad, len(table), scale, p, seed, offset)
    y = dropout(x, p, seed, offset, residual)                   # gradient: dropout(dy, p, seed, offset)
    q, scales = quantize(table)                                 # serving: rows in 8 bits
    cache_write(q, scales, x, slots); x = cache_read(q, scales, slots)
    scores = product(*quantize(x), q, scales)

Autograd does not see these calls: what they return requires no gradient even where an input
does, and gradients are taken by calls of their own (lookup_grad; dropout on the gradient).
What a call writes into (out, a cache) counts as changed in place, so a graph that saved it
refuses to go backward over it.  A call on a given stream waits for no other: what it reads
has to be ready there, and to stay allocated until it is done.
"""
from __future__ import annotations

import ctypes as C

import torch
from torch.autograd.graph import increment_version

from . import scratchpipe as sp

SP_F32, SP_BF16, SP_F16, SP_I32, SP_I64, SP_I8, SP_F8 = range(7)  # the header's element types
_FLOAT = {torch.float32: SP_F32, torch.bfloat16: SP_BF16, torch.float16: SP_F16}
_INDEX = {torch.int32: SP_I32, torch.int64: SP_I64}
_KIND = {torch.int8: SP_I8, torch.float8_e4m3fn: SP_F8}
_MASK = (1 << 64) - 1

# (the public forms build objects: torch.cuda.current_stream().cuda_stream takes 1 us)
_current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream

_lib = None


def _load():
    global _lib
    if _lib is None:
        L = sp.load()
        p, i, l, f, u = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_uint64
        for name, args in (
                ("sp_lookup", [p, i, l, p, i, l, l, l, f, f, u, u, p, i, l, p]),
                ("sp_lookup_grad_workspace", [l, l, l, C.POINTER(l)]),
                ("sp_lookup_grad", [p, i, l, p, i, l, l, f, f, u, u, p, i, l, l, i, p, l, p]),
                ("sp_dropout", [p, i, l, l, l, p, l, f, u, u, p, l, p]),
                ("sp_cache_write", [p, i, l, l, l, p, i, l, p, i, l, l, p, l, p]),
                ("sp_cache_read", [p, i, l, l, l, p, l, l, p, i, l, p, i, l, p]),
                ("sp_product_workspace", [l, l, l, C.POINTER(l)]),
                ("sp_product", [p, p, l, l, p, p, l, l, l, p, i, l, p, l, p])):
            fn = getattr(L, name)
            fn.argtypes, fn.restype = args, i
        _lib = L
    return _lib


def _bad(text):
    return sp.SPError(sp.SP_ERR_INVALID_ARG, text)


def _type(table, dtype, what):
    code = table.get(dtype)
    if code is None:
        raise _bad(f"{what}: {dtype} is none of " + ", ".join(str(k) for k in table))
    return code


def _rows(x, what, copy=True):
    """x as a matrix of its last dimension whose elements follow one another, and its row
    stride: x itself where its strides allow, else (inputs) a copy."""
    if x.dim() != 2:
        if x.dim() == 0:
            raise _bad(f"{what} has no dimension")
        try:
            x = x.view(-1, x.shape[-1]) if x.numel() else x.reshape(0, x.shape[-1])
        except RuntimeError:
            if not copy:
                raise _bad(f"{what}: its rows are not a constant stride apart") from None
            x = x.reshape(-1, x.shape[-1])
    n, d = x.shape
    ld, step = x.stride()
    if (d > 1 and step != 1) or (n > 1 and ld < d):
        if not copy:
            raise _bad(f"{what}: the elements of its rows do not follow one another")
        x, ld = x.contiguous(), d
    return x, (ld if ld > d else d)  # (the stride of a single row may be anything)


def _flat(x):
    return x if x.dim() == 1 and x.is_contiguous() else x.reshape(-1).contiguous()


def _stream(stream, first, others):
    """The raw current stream of the tensors' device, where the call can go ahead on it; None
    where another device or stream has to be made current first (_on)."""
    index = first.get_device()
    if index < 0:
        raise _bad(f"tensors on {first.device}: the operators run on the GPU")
    for t in others:
        if t is not None and t.get_device() != index:
            raise _bad(f"tensors on {first.device} and {t.device}")
    return _raw_stream(index) if stream is None and _current_device() == index else None


def _on(stream, first):
    """Makes the tensors' device and the given stream current: outputs and temporaries then
    belong to the stream that the call runs on."""
    if stream is None:
        return torch.cuda.device(first.device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=first.device) if int(stream) \
            else torch.cuda.default_stream(first.device)
    if stream.device != first.device:
        raise _bad(f"a stream of {stream.device}, tensors on {first.device}")
    return torch.cuda.stream(stream)


def _output(out, shape, dtype, device):
    """The output (allocated where none is given), its address and its row stride."""
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=device)
        return out, out.data_ptr(), shape[-1]
    if tuple(out.shape) != tuple(shape) or out.dtype != dtype:
        raise _bad(f"out is {tuple(out.shape)} {out.dtype}, {tuple(shape)} {dtype} is needed")
    rows, ld = _rows(out, "out", copy=False)
    return out, rows.data_ptr(), ld


def _workspace(size, device, *sizes):
    need = C.c_int64()
    _check(size(*sizes, C.byref(need)))
    return torch.empty(need.value, dtype=torch.uint8, device=device) if need.value else None


def _check(status):
    if status:
        sp._check(status)


def _changed(given):
    """What the caller handed in to be written into (or None), for autograd's checks."""
    if given is not None:
        increment_version(given)


def lookup(tokens, table, scale=1.0, p=0.0, seed=0, offset=0, dtype=None, out=None, stream=None):
    """scale * table[tokens], [*tokens.shape, dim], with dropout of probability p.

    Tokens outside the table (padding, -1) give rows of zeros.  dtype: the output's
    (default: the table's)."""
    st = _stream(stream, table, (tokens, out))
    if st is None:
        with _on(stream, table):
            return lookup(tokens, table, scale, p, seed, offset, dtype, out)
    if table.dim() != 2:
        raise _bad(f"table has shape {tuple(table.shape)}: [rows, dim] is needed")
    ids = _flat(tokens)
    w, ld = _rows(table, "table")
    rows, dim = w.shape
    if dtype is None:
        dtype = table.dtype if out is None else out.dtype
    looked_up, to, old = _output(out, (*tokens.shape, dim), dtype, table.device)
    _check((_lib or _load()).sp_lookup(
        ids.data_ptr(), _type(_INDEX, tokens.dtype, "tokens"), ids.shape[0], w.data_ptr(),
        _type(_FLOAT, table.dtype, "table"), rows, dim, ld, scale, p, seed & _MASK, offset & _MASK,
        to, _type(_FLOAT, dtype, "out"), old, st))
    _changed(out)
    return looked_up


def lookup_grad(tokens, grad, rows, scale=1.0, p=0.0, seed=0, offset=0, dtype=None, out=None,
                accumulate=False, stream=None):
    """The table's gradient [rows, dim] of lookup(tokens, table, scale, p, seed, offset) whose
    output's gradient is grad, summed token by token in a fixed order.

    accumulate: the sums are added to `out`, rows without a token stay as they are.  dtype:
    the result's (default float32)."""
    st = _stream(stream, grad, (tokens, out))
    if st is None:
        with _on(stream, grad):
            return lookup_grad(tokens, grad, rows, scale, p, seed, offset, dtype, out, accumulate)
    if grad.shape[:-1] != tokens.shape:
        raise _bad(f"tokens {tuple(tokens.shape)}, gradient {tuple(grad.shape)}")
    if accumulate and out is None:
        raise _bad("accumulate needs out")
    lib = _lib or _load()
    ids = _flat(tokens)
    g, ld = _rows(grad, "gradient")
    n, dim = g.shape
    if dtype is None:
        dtype = torch.float32 if out is None else out.dtype
    ws = _workspace(lib.sp_lookup_grad_workspace, grad.device, n, rows, dim)
    total, to, old = _output(out, (rows, dim), dtype, grad.device)
    _check(lib.sp_lookup_grad(
        ids.data_ptr(), _type(_INDEX, tokens.dtype, "tokens"), n, g.data_ptr(),
        _type(_FLOAT, grad.dtype, "gradient"), dim, ld, scale, p, seed & _MASK, offset & _MASK,
        to, _type(_FLOAT, dtype, "out"), rows, old, 1 if accumulate else 0,
        *((0, 0) if ws is None else (ws.data_ptr(), ws.shape[0])), st))
    _changed(out)
    return total


def dropout(x, p, seed, offset=0, residual=None, out=None, stream=None):
    """[residual +] dropout of x, whose mask is drawn from (seed, offset) and each element's
    place and never stored.  Its gradient to x is dropout(grad, p, seed, offset), the
    residual's is grad itself.  out may be x or residual.

    Captured into a graph, the call keeps its seed and offset: every replay drops the same
    places.  The same holds for lookup and lookup_grad with p > 0."""
    st = _stream(stream, x, (residual, out))
    if st is None:
        with _on(stream, x):
            return dropout(x, p, seed, offset, residual, out)
    v, ld = _rows(x, "x")
    r, rld = None, 0
    if residual is not None:
        if residual.shape != x.shape or residual.dtype != x.dtype:
            raise _bad(f"x {tuple(x.shape)} {x.dtype}, residual {tuple(residual.shape)} {residual.dtype}")
        r, rld = _rows(residual, "residual")
    y, to, old = _output(out, x.shape, x.dtype, x.device)
    n, dim = v.shape
    if dim:
        _check((_lib or _load()).sp_dropout(
            v.data_ptr(), _type(_FLOAT, x.dtype, "x"), n, dim, ld, 0 if r is None else r.data_ptr(), rld,
            p, seed & _MASK, offset & _MASK, to, old, st))
        _changed(out)
    return y


def _stride(dim):
    """Bytes from row to row of 8-bit rows: product() reads whole 16-byte pieces, and 64 bytes
    of a row at a time, which are one access where they lie in one line (55 tokens against
    80208 rows of 3848 bytes 105 us, of 3840 bytes 78)."""
    return (dim + 127) // 128 * 128 if dim >= 512 else (dim + 15) // 16 * 16


def _groups(dim, group):
    """The scales of a row."""
    group = group or dim
    if dim < 1 or group < 1 or dim % group:
        raise _bad(f"group {group} does not divide dim {dim}")
    return dim // group


def empty_cache(slots, dim, group=None, dtype=torch.int8, device="cuda"):
    """Bytes [slots, dim] and scales [slots, dim / group] of a cache (all zeros), the rows of
    bytes padded as product() likes them."""
    _type(_KIND, dtype, "dtype")
    groups = _groups(dim, group)
    q = torch.zeros((slots, _stride(dim)), dtype=dtype, device=device)[:, :dim]
    return q, torch.zeros((slots, groups), device=device)


def _cache(q, scales):
    """Bytes, their row stride, scales, theirs, columns per scale."""
    if q.dim() != 2 or scales.dim() != 2 or scales.shape[0] != q.shape[0] or not scales.shape[1] \
            or q.shape[1] % scales.shape[1]:
        raise _bad(f"cache {tuple(q.shape)}, scales {tuple(scales.shape)}: [slots, dim] and "
                   "[slots, dim / group] are needed")
    if scales.dtype != torch.float32:
        raise _bad(f"scales are {scales.dtype}")
    v, ld = _rows(q, "cache", copy=False)
    s, sld = _rows(scales, "scales", copy=False)
    return v, ld, s, sld, q.shape[1] // scales.shape[1]


def cache_write(q, scales, x, slots, stream=None):
    """Quantises the rows of x [*slots.shape, dim] (dim may be several dimensions, as heads and
    their width) into the given slots (distinct; rows of a slot outside the cache, as -1, are
    left out)."""
    st = _stream(stream, q, (scales, x, slots))
    if st is None:
        with _on(stream, q):
            return cache_write(q, scales, x, slots)
    v, ld, s, sld, group = _cache(q, scales)
    at = _flat(slots)
    n, (size, dim) = at.shape[0], v.shape
    if x.shape[:slots.dim()] != slots.shape or x.numel() != n * dim:
        raise _bad(f"cache {tuple(q.shape)}, {tuple(slots.shape)} slots, rows {tuple(x.shape)}")
    r = x
    if x.dim() != 2 or slots.dim() != 1:
        try:
            r = x.view(n, dim)
        except RuntimeError:
            r = x.reshape(n, dim)
    r, rld = _rows(r, "x")
    _check((_lib or _load()).sp_cache_write(
        r.data_ptr(), _type(_FLOAT, x.dtype, "x"), n, dim, rld, at.data_ptr(),
        _type(_INDEX, slots.dtype, "slots"), group, v.data_ptr(), _type(_KIND, q.dtype, "cache"), size, ld,
        s.data_ptr(), sld, st))
    _changed((q, scales))


def cache_read(q, scales, slots, dtype=torch.bfloat16, out=None, stream=None):
    """The rows [*slots.shape, dim] that the given slots stand for; zeros for a slot outside
    the cache (as -1)."""
    st = _stream(stream, q, (scales, slots, out))
    if st is None:
        with _on(stream, q):
            return cache_read(q, scales, slots, dtype, out)
    v, ld, s, sld, group = _cache(q, scales)
    at = _flat(slots)
    size, dim = v.shape
    rows, to, old = _output(out, (*slots.shape, dim), dtype, q.device)
    _check((_lib or _load()).sp_cache_read(
        v.data_ptr(), _type(_KIND, q.dtype, "cache"), size, dim, ld, s.data_ptr(), sld, group,
        at.data_ptr(), _type(_INDEX, slots.dtype, "slots"), at.shape[0], to,
        _type(_FLOAT, dtype, "out"), old, st))
    _changed(out)
    return rows


def quantize(x, group=None, dtype=torch.int8, stream=None):
    """The rows of x [..., dim] in 8 bits: bytes [n, dim] and scales [n, dim / group], laid out
    as empty_cache() does (group: the whole row)."""
    st = _stream(stream, x, ())
    if st is None:
        with _on(stream, x):
            return quantize(x, group, dtype)
    r, rld = _rows(x, "x")
    n, dim = r.shape
    groups = _groups(dim, group)
    kind = _type(_KIND, dtype, "dtype")
    ld = _stride(dim)
    q = torch.empty((n, ld), dtype=dtype, device=x.device)
    scales = torch.empty((n, groups), dtype=torch.float32, device=x.device)
    _check((_lib or _load()).sp_cache_write(
        r.data_ptr(), _type(_FLOAT, x.dtype, "x"), n, dim, rld, 0, 0, dim // groups, q.data_ptr(), kind, n, ld,
        scales.data_ptr(), groups, st))
    return (q if ld == dim else q[:, :dim]), scales


def product(x, x_scales, w, w_scales, dtype=torch.bfloat16, out=None, stream=None):
    """x_scales[:, None] * w_scales * (x @ w.T) of 8-bit integer rows x [m, k] and w [n, k],
    the sums exact; one scale per row of each ([m] or [m, 1], [n] or [n, 1]).  Fastest where
    rows start at multiples of 64 bytes, then of 16; quantize() and empty_cache() pad them so."""
    st = _stream(stream, x, (x_scales, w, w_scales, out))
    if st is None:
        with _on(stream, x):
            return product(x, x_scales, w, w_scales, dtype, out)
    if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1]:
        raise _bad(f"x {tuple(x.shape)}, w {tuple(w.shape)}: [m, k] and [n, k] are needed")
    (m, k), n = x.shape, w.shape[0]
    if x.dtype != torch.int8 or w.dtype != torch.int8:
        raise _bad(f"x is {x.dtype}, w {w.dtype}: int8 is needed")
    if x_scales.numel() != m or w_scales.numel() != n or x_scales.dtype != torch.float32 \
            or w_scales.dtype != torch.float32:
        raise _bad(f"scales {tuple(x_scales.shape)} {x_scales.dtype}, {tuple(w_scales.shape)} "
                   f"{w_scales.dtype}: {m} and {n} of float32 are needed")
    lib = _lib or _load()
    a, ald = _rows(x, "x")
    b, bld = _rows(w, "w")
    xs, ws = _flat(x_scales), _flat(w_scales)
    work = _workspace(lib.sp_product_workspace, x.device, m, n, k)
    scores, to, old = _output(out, (m, n), dtype, x.device)
    _check(lib.sp_product(
        a.data_ptr(), xs.data_ptr(), m, ald, b.data_ptr(), ws.data_ptr(), n, bld, k, to,
        _type(_FLOAT, dtype, "out"), old, *((0, 0) if work is None else (work.data_ptr(), work.shape[0])),
        st))
    _changed(out)
    return scores
