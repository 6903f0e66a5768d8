"""Rows in 4 bits read into each type: every value that codes and scales stand for, rounded once."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2205_04702_amd import tokens as tk  # noqa: E402
from tests import scores_reference as ref  # noqa: E402
from tests.test_gpu_rows4 import BF16, F16, F32, some_rows, values  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def same(got, want):
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got, 7.0), torch.nan_to_num(want, 7.0))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_every_code_and_scale(dtype):
    """256 slots, one for each scale byte, of all codes.  Those past a type's largest number are infinite, those below
    its smallest are rounded to its subnormal numbers or to zero."""
    q, s = tk.empty_cache4(256, 64)
    code = torch.arange(64, dtype=torch.uint8) % 16
    q.copy_((code[0::2] | code[1::2] << 4).expand(256, -1))
    s.copy_(torch.arange(256, dtype=torch.uint8)[:, None].expand(-1, 2))
    got = tk.cache_read4(q, s, torch.arange(256, device="cuda"), dtype=dtype).cpu()
    # (fp32 holds all of them exactly that are below 2^128, which every type's largest number is)
    same(got, ref.values4(q.cpu(), s.cpu()).float().to(dtype))


@pytest.mark.parametrize("dim,lead,ld", [(1001, 0, 1001), (1001, 3, 1011), (1024, 0, 1024), (1024, 16, 1040), (1024, 5, 1029), (2000, 1, 2004),
                                         (40, 0, 41), (7, 0, 7), (3, 1, 5), (16, 0, 16)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_many_rows(dim, lead, ld, dtype):
    """Enough octets for the form with four per thread: rows that start at any place of a line, slots that are none."""
    n, slots = (1 << 20) // ((dim + 7) // 8) + 77, 300
    q, s = some_rows(slots, dim, dim, -130 if dtype == BF16 else -30, 125 if dtype == BF16 else 20)
    s[::7] = 255
    s[1::7] = 0
    at = torch.randint(-1, slots + 1, (n,), generator=torch.Generator().manual_seed(9))
    buf = torch.full((n * ld + lead + 8,), 9.0, device="cuda", dtype=dtype)
    out = buf[lead:lead + n * ld].view(n, ld)[:, :dim]
    got = tk.cache_read4(q, s, at.cuda(), dim, dtype, out=out).cpu()
    table = torch.cat([ref.values4(q.cpu(), s.cpu())[:, :dim].float(), torch.zeros((1, dim))]).to(dtype)
    same(got, table[torch.where((at < 0) | (at >= slots), slots, at)])
    out.fill_(9.0)
    assert (buf == 9).all()


@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("dim", [1, 31, 45, 64, 1000])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_few_rows(dim, dtype, index):
    """What was written comes back in the type that it came in; slots outside the cache are zeros."""
    slots = 50
    q, s = tk.empty_cache4(slots, dim)
    x = values(slots, dim, dim, dtype)
    tk.cache_write4(q, s, x.cuda(), torch.arange(slots, device="cuda"))
    at = torch.tensor([[0, -1, 7], [slots - 1, slots, 7]])
    out = torch.full((2, 3, dim + 2), 9.0, device="cuda", dtype=dtype)
    got = tk.cache_read4(q, s, at.to(index).cuda(), dim, dtype, out=out[:, :, 1:1 + dim]).cpu()
    want = ref.values4(*ref.quantize4(x))[at.clamp(0, slots - 1)][..., :dim].to(dtype)
    want[0, 1] = want[1, 1] = 0
    same(got, want)
    assert (out[:, :, 0] == 9).all() and (out[:, :, -1] == 9).all()
