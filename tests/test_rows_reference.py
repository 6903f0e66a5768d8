"""The references of the row operators' tests, against published values and by hand."""
import torch

from tests import rows_reference as ref


def test_philox_gives_the_published_vectors():
    """The known answers of Philox 4x32-10 published with the generator (Random123)."""
    assert ref.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert ref.philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6,
                                                             0x6D5451FD]
    assert ref.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) \
        == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_mask_by_hand():
    """The first octet of counter 0, key 0: 16 bits per column, low halves first."""
    bits = [0xE8D5, 0x6627, 0xC58D, 0xE169, 0xAC4C, 0xBC57, 0xDBD8, 0x9B00]
    for p in (0.25, 0.5, 0.75):
        want = [b >= round(65536 * p) for b in bits]
        assert ref.keep_mask(1, 8, p, 0, 0)[0].tolist() == want
    assert ref.keep_mask(1, 5, 0.75, 0, 0)[0].tolist() == [b >= 49152 for b in bits[:5]]
    assert ref.keep_factor(0.5) == 2.0 and ref.dropped_below(2.0 ** -18) == 0


def test_mask_keeps_its_share():
    """Of 32768 columns at p = 0.3 the kept are 0.7 within five standard deviations."""
    kept = ref.keep_mask(64, 512, 0.3, 7, 9).double().mean().item()
    assert abs(kept - 0.7) < 5 * (0.21 / 32768) ** 0.5


def test_grad_reference_by_hand():
    tok = torch.tensor([2, -1, 2, 0, 9])
    g = torch.tensor([[1.0], [10.0], [2.0], [4.0], [8.0]])
    total, size, count = ref.lookup_grad(tok, g, 3, scale=0.5)
    assert total.view(-1).tolist() == [2.0, 0.0, 1.5] and count.view(-1).tolist() == [1, 0, 2]


def test_e4m3_rounding_agrees_with_torch():
    x = torch.cat([torch.linspace(-448, 448, 100_001), torch.linspace(-2.0 ** -6, 2.0 ** -6, 10_001)])
    assert torch.equal(ref.round_e4m3(x.double()), x.to(torch.float8_e4m3fn).double())
