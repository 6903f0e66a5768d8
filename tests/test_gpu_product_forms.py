"""Every form of the product: each tile, whole and in each number of parts of k, with rows in
aligned pieces and without.  Bounds as in test_gpu_rows.py: the sum is one rounding, each scale
another."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2205_04702_amd import tokens as tk  # noqa: E402
from tests.product_forms import cut  # noqa: E402
from tests.rows_reference import TINY, U32, UNIT  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


FORMS = [
    ((32, 64), 1, (33, 100, 700)), ((32, 64), 2, (12, 7050, 2925)), ((32, 64), 4, (5, 53, 1784)),
    ((32, 64), 8, (40, 70, 3000)), ((32, 64), 16, (5, 100, 5001)),
    ((64, 64), 1, (63, 8292, 180)), ((64, 64), 2, (1560, 134, 3623)), ((64, 64), 4, (37, 2161, 2431)),
    ((64, 64), 8, (1073, 30, 2100)), ((64, 64), 16, (515, 33, 4900)),
    ((64, 128), 1, (67, 9976, 333)), ((64, 128), 2, (3, 8325, 7256)), ((64, 128), 4, (1, 5135, 2483)),
    ((64, 128), 8, (1, 2298, 3546)), ((64, 128), 16, (1, 1025, 6747)),
    ((128, 128), 1, (264, 6937, 450)), ((128, 128), 2, (65, 12_422, 6018)),
    ((128, 128), 4, (92, 4548, 7009)), ((128, 128), 4, (596, 1420, 8047)),
    ((128, 128), 8, (70, 2132, 11_188)),
    ((256, 256), 1, (2300, 5000, 4100)),
    ((256, 256), 2, (455, 8457, 4357)), ((256, 256), 2, (1493, 3302, 8938)),
    ((256, 256), 4, (202, 8293, 8115)), ((256, 256), 8, (138, 6026, 12_361)),
]


def test_every_form_is_among_them():
    want = {((32, 64), p) for p in (1, 2, 4, 8, 16)} | {((64, 64), p) for p in (1, 2, 4, 8, 16)} \
        | {((64, 128), p) for p in (1, 2, 4, 8, 16)} | {((128, 128), p) for p in (1, 2, 4, 8)} \
        | {((256, 256), p) for p in (1, 2, 4, 8)}
    assert {(t, p) for t, p, _ in FORMS} == want
    for tile, parts, shape in FORMS:
        assert cut(*shape) == (tile, parts), shape


@pytest.mark.parametrize("pad", [True, False])
@pytest.mark.parametrize("tile,parts,shape", FORMS)
def test_form(tile, parts, shape, pad):
    m, n, k = shape
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n + k)
    ld = (k + 15) // 16 * 16 if pad else k + (k % 16 == 0)
    x = torch.randint(-128, 128, (m, ld), generator=g, device="cuda", dtype=torch.int8)[:, :k]
    w = torch.randint(-128, 128, (n, ld), generator=g, device="cuda", dtype=torch.int8)[:, :k]
    xs, ws = torch.rand(m, generator=g, device="cuda") + 0.1, torch.rand(n, generator=g, device="cuda") + 0.1
    want = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()[None, :]
    for out in (torch.float32, torch.bfloat16):
        got = tk.product(x, xs, w, ws, dtype=out)
        bound = want.abs() * (UNIT[out] + 4 * U32) + TINY[out]
        off = (got.double() - want).abs() - bound
        assert not torch.isnan(off).any() and off.max().item() <= 0
        assert torch.equal(got, tk.product(x, xs, w, ws, dtype=out))
