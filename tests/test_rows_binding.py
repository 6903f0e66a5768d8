"""What the row operators' binding decides before any device work."""
import pytest
import torch

from paper_2205_04702_amd import scratchpipe as sp
from paper_2205_04702_amd import tokens as tk


@pytest.mark.parametrize("dim,group", [(96, 40), (100, 30), (64, 128), (64, -8), (0, None), (0, 4)])
def test_a_cache_of_groups_that_do_not_divide_its_rows_is_refused(dim, group):
    """(96 columns in groups of 40 had been taken for two groups of 48.)"""
    with pytest.raises(sp.SPError, match="does not divide"):
        tk.empty_cache(10, dim, group, device="cpu")


@pytest.mark.parametrize("dim,group,scales", [(96, 48, 2), (96, None, 1), (96, 96, 1), (7, 7, 1), (512, 8, 64)])
def test_a_cache_has_a_scale_for_each_group(dim, group, scales):
    q, s = tk.empty_cache(10, dim, group, device="cpu")
    assert q.shape == (10, dim) and s.shape == (10, scales) and s.dtype == torch.float32
    assert q.stride(0) % 16 == 0 and q.stride(0) >= dim
