"""The row operators beside autograd: it does not see them, but it sees what they overwrite."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2205_04702_amd import scratchpipe as sp  # noqa: E402
from paper_2205_04702_amd import tokens as tk  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def calls():
    t, w = torch.arange(4, device="cuda"), torch.randn((5, 64), device="cuda")
    q, s = tk.quantize(w)
    return {
        "lookup": ((4, 64), lambda out: tk.lookup(t, w, out=out)),
        "lookup_grad": ((5, 64), lambda out: tk.lookup_grad(t, w[:4], 5, out=out)),
        "lookup_grad added": ((5, 64), lambda out: tk.lookup_grad(t, w[:4], 5, out=out, accumulate=True)),
        "dropout": ((5, 64), lambda out: tk.dropout(w, 0.5, 1, out=out)),
        "cache_read": ((4, 64), lambda out: tk.cache_read(q, s, t, dtype=torch.float32, out=out)),
        "product": ((5, 5), lambda out: tk.product(q, s, q, s, dtype=torch.float32, out=out)),
    }


@pytest.mark.parametrize("name", ["lookup", "lookup_grad", "lookup_grad added", "dropout", "cache_read", "product"])
def test_a_saved_tensor_that_is_written_into_is_noticed(name):
    shape, call = calls()[name]
    buf = torch.ones(shape, device="cuda")
    x = torch.ones(shape, device="cuda", requires_grad=True)
    y = (x * buf).sum()
    assert call(buf) is buf
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    y = (x * buf).sum()  # saved after the call: nothing to object to
    y.backward()
    assert torch.equal(x.grad, buf)


def test_a_cache_that_is_written_into_is_noticed():
    q, s = tk.empty_cache(8, 64)
    x = torch.ones((8, 1), device="cuda", requires_grad=True)
    y = (x * s).sum()
    before = q._version
    tk.cache_write(q, s, torch.ones((3, 64), device="cuda"), torch.arange(3, device="cuda"))
    assert q._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_a_refused_call_changes_nothing():
    t, w = torch.arange(4, device="cuda"), torch.randn((5, 64), device="cuda")
    out = torch.zeros((4, 64), device="cuda")
    before = out._version
    with pytest.raises(sp.SPError):
        tk.lookup(t, w, p=1.0, out=out)
    assert out._version == before and (out == 0).all()


def test_outputs_require_no_gradient_and_inference_tensors_are_taken():
    t, w = torch.arange(4, device="cuda"), torch.randn((5, 64), device="cuda", requires_grad=True)
    assert not tk.lookup(t, w).requires_grad and not tk.dropout(w, 0.5, 1).requires_grad
    with torch.inference_mode():
        q, s = tk.empty_cache(8, 64)
        out = torch.empty((4, 64), device="cuda")
    tk.cache_write(q, s, w[:4], t)
    assert tk.cache_read(q, s, t, dtype=torch.float32, out=out) is out
    assert torch.equal(out, q[:4].float() * s[:4])
