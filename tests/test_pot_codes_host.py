"""Pools in 8 bits on the host: what they refuse before anything is launched."""
import pytest
import torch

from paper_2410_01518_amd.pot import PagedPots
from tests.test_paged_binding import launches  # noqa: F401  (a fixture)


@pytest.mark.parametrize("codes,page,rows", [(torch.float8_e4m3fn, 16, 12), (torch.float8_e4m3fn, 16, 32), (torch.float8_e4m3fn, 48, 3), (torch.float8_e4m3fn, 37, 2), (torch.float8_e4m3fn, 16, 0),
                                             (torch.float8_e4m3fn, 16, -4), (torch.int8, 16, 16), (torch.int8, 16, 2)])
def test_scale_rows_that_there_cannot_be(codes, page, rows):
    with pytest.raises(ValueError, match="scale_rows"):
        PagedPots(2, 4, page, 100, 20, 1, 2, 1, 64, device="cpu", codes=codes, scale_rows=rows)


@pytest.mark.parametrize("codes,page,rows", [(torch.float8_e4m3fn, 16, 16), (torch.float8_e4m3fn, 48, 16), (torch.float8_e4m3fn, 37, 1), (torch.int8, 37, 1)])
def test_scales_of_a_pool(codes, page, rows):
    pool = PagedPots(2, 4, page, 100, 20, 3, 2, 1, 64, device="cpu", codes=codes, scale_rows=rows)
    assert pool.K.dtype is codes and pool.K.shape == (4, 3, 1, page, 64) and pool.K_scales.shape == (4, 3, 1, page // rows) and not pool.V_scales.any()


def test_a_pot_whose_tokens_share_scales_is_not_distilled(launches):  # noqa: F811
    """Refused before its scores are worked out."""
    n, L, Hkv, d = 64, 2, 1, 64
    pool = PagedPots(2, 4, n, n, n, L, 2, Hkv, d, device="cpu", codes=torch.float8_e4m3fn, scale_rows=16)
    pool.lengths[0] = n
    keep, workspace = torch.full((1, L, Hkv, 20), -5, dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)
    with pytest.raises(AssertionError, match="scale per token"):
        pool.distill(0, 0, torch.zeros((1, L, 2, 3, d), dtype=torch.bfloat16), torch.zeros((1, n)), keep, workspace, k=20, T=4)
    assert launches.calls == 0 and pool.lengths[0] == n and (keep == -5).all()


@pytest.mark.parametrize("shared", [1, 2])
def test_novelty_carried_per_head_that_some_heads_share(launches, shared):  # noqa: F811
    """Rows that are compacted cannot be those of two layers, or of two heads; refused before anything is moved."""
    n, L, Hkv, d = 64, 2, 3, 64
    pool = PagedPots(2, 4, n, n, n, L, 3, Hkv, d, device="cpu", codes=torch.int8)
    pool.lengths[0] = n
    novelty = torch.zeros((1, 1, Hkv, n) if shared == 1 else (1, L, 1, n)).expand(1, L, Hkv, n)
    with pytest.raises(AssertionError, match="shared by some"):
        pool.distill(0, 0, torch.zeros((1, L, 3, 3, d), dtype=torch.bfloat16), novelty, torch.zeros((1, L, Hkv, 20), dtype=torch.int32), None, k=20, T=4)
    assert launches.calls == 0 and pool.lengths[0] == n
