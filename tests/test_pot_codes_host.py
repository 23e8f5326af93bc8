"""Pools in 8 bits on the host: what their constructors refuse."""
import pytest
import torch

from paper_2410_01518_amd.pot import PagedPots


@pytest.mark.parametrize("codes,page,rows", [(torch.float8_e4m3fn, 16, 12), (torch.float8_e4m3fn, 16, 32), (torch.float8_e4m3fn, 48, 3), (torch.float8_e4m3fn, 37, 2), (torch.float8_e4m3fn, 16, 0),
                                             (torch.float8_e4m3fn, 16, -4), (torch.int8, 16, 16), (torch.int8, 16, 2)])
def test_scale_rows_that_there_cannot_be(codes, page, rows):
    with pytest.raises(ValueError, match="scale_rows"):
        PagedPots(2, 4, page, 100, 20, 1, 2, 1, 64, device="cpu", codes=codes, scale_rows=rows)


@pytest.mark.parametrize("codes,page,rows", [(torch.float8_e4m3fn, 16, 16), (torch.float8_e4m3fn, 48, 16), (torch.float8_e4m3fn, 37, 1), (torch.int8, 37, 1)])
def test_scales_of_a_pool(codes, page, rows):
    pool = PagedPots(2, 4, page, 100, 20, 3, 2, 1, 64, device="cpu", codes=codes, scale_rows=rows)
    assert pool.K.dtype is codes and pool.K.shape == (4, 3, 1, page, 64) and pool.K_scales.shape == (4, 3, 1, page // rows) and not pool.V_scales.any()
