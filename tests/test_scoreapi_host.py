"""Refusals of the C entry points for rows in 4 bits and for scores: reported with a text before any
device work, so they run without a GPU."""
import ctypes as C

import pytest

from paper_2205_04702_amd import scratchpipe as sp
from paper_2205_04702_amd import tokens as tk
from tests.test_rowapi_host import A, INF, NAN, call

WRITE4 = dict(x=A, type=tk.SP_F32, n=8, dim=70, x_ld=70, index=A, index_type=tk.SP_I32, q=A, slots=10, q_ld=48, scales=A,
              scales_ld=3, stream=0)
READ4 = dict(q=A, slots=10, dim=70, q_ld=48, scales=A, scales_ld=3, index=A, index_type=tk.SP_I32, n=8, out=A,
             out_type=tk.SP_F32, out_ld=70, stream=0)
PRODUCT4 = dict(x=A, x_scales=A, m=4, x_ld=48, x_scales_ld=16, w=A, w_scales=A, n=8, w_ld=48, w_scales_ld=16, k=70, out=A,
                out_type=tk.SP_BF16, out_ld=8, workspace=0, workspace_bytes=0, stream=0)
ADJUST = dict(scores=A, type=tk.SP_F32, n=4, vocab=100, ld=100, previous=A, previous_type=tk.SP_I64, length=5, previous_ld=5,
              repetition=1.0, presence=0.0, frequency=0.0, penalties=A, penalties_ld=3, bias_tokens=A, bias_type=tk.SP_I32,
              bias_tokens_ld=2, bias=A, bias_ld=2, biases=2, allowed=A, allowed_ld=4, out=A, out_ld=100, stream=0)
DISTILL = dict(scores=A, type=tk.SP_BF16, n=1000, vocab=100, ld=100, tokens=A, token_type=tk.SP_I64, tokens_ld=5, teacher=A,
               teacher_type=tk.SP_F32, teacher_ld=5, k=5, temperature=1.0, loss=A, workspace=A, workspace_bytes=1 << 30, stream=0)
GRAD = dict(list(DISTILL.items())[:13] + [("weight", 1.0), ("weights", A), ("loss", A), ("grad", A), ("grad_type", tk.SP_BF16),
                                          ("grad_ld", 100)] + list(DISTILL.items())[14:])


@pytest.mark.parametrize("name,base,over,needle", [
    ("sp_cache4_write", WRITE4, dict(index_type=tk.SP_F32), "index type"),
    ("sp_cache4_write", WRITE4, dict(type=tk.SP_I8), "element type"),
    ("sp_cache4_write", WRITE4, dict(n=-1), "rows"),
    ("sp_cache4_write", WRITE4, dict(slots=1 << 31), "slots"),
    ("sp_cache4_write", WRITE4, dict(dim=0), "dim"),
    ("sp_cache4_write", WRITE4, dict(dim=97, x_ld=97), "stride"),
    ("sp_cache4_write", WRITE4, dict(q_ld=47), "stride"),
    ("sp_cache4_write", WRITE4, dict(scales_ld=2), "stride"),
    ("sp_cache4_write", WRITE4, dict(x=A + 2), "aligned"),
    ("sp_cache4_write", WRITE4, dict(q=0), "null cache"),
    ("sp_cache4_write", WRITE4, dict(index=0, n=11), "without an index"),
    ("sp_cache4_read", READ4, dict(scales=0), "null scales"),
    ("sp_cache4_read", READ4, dict(out=0), "null rows"),
    ("sp_cache4_read", READ4, dict(out_ld=69), "stride"),
    ("sp_cache4_read", READ4, dict(dim=(1 << 20) + 1), "dim"),
    ("sp_product4", PRODUCT4, dict(k=0), "k 0"),
    ("sp_product4", PRODUCT4, dict(k=(1 << 20) + 1), "k 1048577"),
    ("sp_product4", PRODUCT4, dict(m=-1), "outputs"),
    ("sp_product4", PRODUCT4, dict(x=0), "null x"),
    ("sp_product4", PRODUCT4, dict(w_scales=0), "null w"),
    ("sp_product4", PRODUCT4, dict(x=A + 8), "multiples of 16"),
    ("sp_product4", PRODUCT4, dict(w_scales=A + 4), "multiples of 16"),
    ("sp_product4", PRODUCT4, dict(w_ld=56), "multiples of 16"),
    ("sp_product4", PRODUCT4, dict(x_scales_ld=8), "multiples of 16"),
    ("sp_product4", PRODUCT4, dict(w_ld=32), "stride"),
    ("sp_product4", PRODUCT4, dict(w_ld=1 << 23), "stride"),
    ("sp_product4", PRODUCT4, dict(x_scales_ld=2), "stride"),
    ("sp_product4", PRODUCT4, dict(w_scales_ld=1 << 23), "stride"),
    ("sp_product4", PRODUCT4, dict(out_ld=7), "stride"),
    ("sp_product4", PRODUCT4, dict(out_ld=1 << 23), "stride"),
    ("sp_product4", PRODUCT4, dict(out_type=tk.SP_I8), "element type"),
    ("sp_adjust", ADJUST, dict(type=tk.SP_F8), "element type"),
    ("sp_adjust", ADJUST, dict(n=1 << 31), "rows"),
    ("sp_adjust", ADJUST, dict(vocab=0), "columns"),
    ("sp_adjust", ADJUST, dict(vocab=(1 << 20) + 1, ld=1 << 21, out_ld=1 << 21), "columns"),
    ("sp_adjust", ADJUST, dict(length=-1), "previous tokens"),
    ("sp_adjust", ADJUST, dict(biases=-1), "biases"),
    ("sp_adjust", ADJUST, dict(biases=2048, bias_tokens_ld=2048, bias_ld=2048), "biases"),
    ("sp_adjust", ADJUST, dict(previous_type=tk.SP_F32), "previous tokens' type"),
    ("sp_adjust", ADJUST, dict(bias_type=tk.SP_F32), "token type"),
    ("sp_adjust", ADJUST, dict(repetition=0.0), "repetition"),
    ("sp_adjust", ADJUST, dict(repetition=NAN), "repetition"),
    ("sp_adjust", ADJUST, dict(repetition=INF), "repetition"),
    ("sp_adjust", ADJUST, dict(frequency=INF), "frequency"),
    ("sp_adjust", ADJUST, dict(previous=0), "null previous"),
    ("sp_adjust", ADJUST, dict(previous=A + 4), "aligned"),
    ("sp_adjust", ADJUST, dict(previous_ld=4), "stride"),
    ("sp_adjust", ADJUST, dict(penalties_ld=2), "stride"),
    ("sp_adjust", ADJUST, dict(bias=0), "null biases"),
    ("sp_adjust", ADJUST, dict(bias_tokens=0), "null biases' tokens"),
    ("sp_adjust", ADJUST, dict(allowed=A + 2), "aligned"),
    ("sp_adjust", ADJUST, dict(allowed_ld=3), "stride"),
    ("sp_adjust", ADJUST, dict(scores=0), "null scores"),
    ("sp_adjust", ADJUST, dict(out_ld=99), "stride"),
    ("sp_distill", DISTILL, dict(type=tk.SP_I32), "element type"),
    ("sp_distill", DISTILL, dict(teacher_type=tk.SP_I32), "element type"),
    ("sp_distill", DISTILL, dict(token_type=tk.SP_F32), "token type"),
    ("sp_distill", DISTILL, dict(k=0), "entries"),
    ("sp_distill", DISTILL, dict(k=1025, tokens_ld=1025, teacher_ld=1025), "entries"),
    ("sp_distill", DISTILL, dict(vocab=0), "columns"),
    ("sp_distill", DISTILL, dict(temperature=0.0), "temperature"),
    ("sp_distill", DISTILL, dict(temperature=-1.0), "temperature"),
    ("sp_distill", DISTILL, dict(temperature=1e-45), "temperature"),
    ("sp_distill", DISTILL, dict(temperature=4e-39), "temperature"),
    ("sp_distill", DISTILL, dict(temperature=NAN), "temperature"),
    ("sp_distill", DISTILL, dict(tokens_ld=4), "stride"),
    ("sp_distill", DISTILL, dict(loss=0), "null loss"),
    ("sp_distill_grad", GRAD, dict(grad=0), "null gradient"),
    ("sp_distill_grad", GRAD, dict(grad_type=tk.SP_I8), "element type"),
    ("sp_distill_grad", GRAD, dict(weights=A + 2), "aligned"),
    ("sp_distill_grad", GRAD, dict(grad_ld=99), "stride"),
])
def test_refused(name, base, over, needle):
    st, text = call(name, base, **over)
    assert st == sp.SP_ERR_INVALID_ARG
    assert needle in text


@pytest.mark.parametrize("name,base,over", [
    ("sp_cache4_write", WRITE4, dict(n=0, index=0, x=0)),
    ("sp_cache4_read", READ4, dict(n=0, index=0, out=0)),
    ("sp_product4", PRODUCT4, dict(m=0, x=0, out=0)),
    ("sp_product4", PRODUCT4, dict(n=0, w=0, out=0)),
    ("sp_adjust", ADJUST, dict(n=0, scores=0, previous=0, penalties=0, bias=0, bias_tokens=0, allowed=0, out=0)),
    ("sp_distill", DISTILL, dict(n=0, scores=0, tokens=0, teacher=0, loss=0)),
    ("sp_distill_grad", GRAD, dict(n=0, scores=0, tokens=0, teacher=0, weights=0, loss=0, grad=0)),
])
def test_nothing_to_do_is_no_error(name, base, over):
    assert call(name, base, **over)[0] == sp.SP_OK


def test_workspace_sizes():
    L = tk._load()
    b = C.c_int64(-1)
    assert L.sp_product4_workspace(4, 4, 0, C.byref(b)) == sp.SP_ERR_INVALID_ARG
    assert L.sp_product4_workspace(8192, 8192, 64, C.byref(b)) == sp.SP_OK and b.value == 0
    assert L.sp_product4_workspace(1, 1, 1 << 20, C.byref(b)) == sp.SP_OK and 0 <= b.value < 1 << 20
    assert L.sp_distill_workspace(1, 0, 1, 0, C.byref(b)) == sp.SP_ERR_INVALID_ARG
    assert L.sp_distill_workspace(2 ** 31 - 1, 1 << 20, 1024, 1, C.byref(b)) == sp.SP_OK and b.value == 0


def test_binding_refuses_host_tensors():
    import torch
    s, i = torch.zeros((4, 64)), torch.zeros((4, 1), dtype=torch.int64)
    for go in (lambda: tk.quantize4(s), lambda: tk.adjust(s, i), lambda: tk.distill(s, i, s[:, :1]), lambda: tk.distill_grad(s, i, s[:, :1])):
        with pytest.raises(sp.SPError, match="GPU"):
            go()
