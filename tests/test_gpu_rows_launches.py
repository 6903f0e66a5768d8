"""Calls of the row operators that are more blocks than one launch has (2^32 threads along an
axis): each is what the same call gives in parts.  They need much memory, and are skipped
where it is not free."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2205_04702_amd import tokens as tk  # noqa: E402
from tests import rows_reference as ref  # noqa: E402

BF16 = torch.bfloat16


def room(gigabytes):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 1e9:
        pytest.skip(f"{gigabytes} GB of free GPU memory needed")


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def test_cache_of_more_groups_than_a_launch_has():
    """2^30 groups and more: 2^24 blocks of 64."""
    room(60)
    n, dim, group = 2 ** 21 + 5, 4096, 8
    x = torch.empty((n, dim), dtype=BF16, device="cuda").normal_()
    q, s = tk.quantize(x, group)
    for i in range(0, n, 2 ** 18):
        part, scales = tk.quantize(x[i:i + 2 ** 18], group)
        assert torch.equal(q[i:i + 2 ** 18], part) and torch.equal(s[i:i + 2 ** 18], scales)


def test_lookup_of_more_rows_than_a_launch_has():
    """Rows of 513 octets are a block each: 2^24 and more of them."""
    room(160)
    n, dim = 2 ** 24 + 3, 4104
    w = torch.empty((7, dim), dtype=BF16, device="cuda").normal_()
    tok = torch.randint(-1, 7, (n,), device="cuda", dtype=torch.int32)
    rows = [0, 2 ** 23 - 1, 2 ** 23, 2 ** 24 - 1, 2 ** 24, n - 1]
    tok[torch.tensor(rows, device="cuda")] = 3
    got = tk.lookup(tok, w, 1.5, 0.1, 3, 4)
    scale = 1.5 * ref.keep_factor(0.1)
    for i in range(0, n, 2 ** 19):
        a = got[i:i + 2 ** 19]
        b = tk.lookup(tok[i:i + 2 ** 19], w, scale)
        assert torch.equal(a, torch.where(a != 0, b, torch.zeros((), dtype=BF16, device="cuda")))
        live = (b != 0).sum().item()
        assert abs((a != 0).sum().item() / live - 0.9) < 5 * (0.09 / live) ** 0.5 + 2.0 ** -17
    drop = ref.dropped_below(0.1)
    for row in rows:  # the mask is the row's own
        for octet in (0, 255, 512):
            words = ref.philox([octet, row, 4, 0], [3, 0])
            keep = torch.tensor([words[e // 2] >> (16 * (e % 2)) & 0xFFFF for e in range(8)]) >= drop
            live = w[3, octet * 8:octet * 8 + 8] != 0
            assert torch.equal((got[row, octet * 8:octet * 8 + 8] != 0).cpu(), keep & live.cpu())


def test_product_of_more_tiles_than_a_launch_has():
    """2^30 rows and more on either side: 2^24 tiles of 64 rows."""
    room(70)
    n, k = 2 ** 30 + 130, 16
    x = torch.empty((n, k), dtype=torch.int8, device="cuda")
    for i in range(0, n, 2 ** 26):
        x[i:i + 2 ** 26].random_(-128, 128)
    xs = torch.rand(n, device="cuda")
    y, ys = x[-3:].clone(), torch.rand(3, device="cuda")
    step = 2 ** 24
    got = tk.product(x, xs, y, ys)
    for i in range(0, n, step):
        assert torch.equal(got[i:i + step], tk.product(x[i:i + step], xs[i:i + step], y, ys))
    got = None
    got = tk.product(y, ys, x, xs)
    for i in range(0, n, step):
        assert torch.equal(got[:, i:i + step], tk.product(y, ys, x[i:i + step], xs[i:i + step]))
