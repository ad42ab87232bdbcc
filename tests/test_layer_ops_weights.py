"""Weights as strp_linear reads them (no GPU needed)."""
import pytest
import torch

from paper_2510_03246_amd import strp


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 19), (5, 8), (7, 4915), (1001, 13)])
def test_rows_begin_at_multiples_of_eight(M, K, dt):
    g = torch.Generator().manual_seed(K)
    W = torch.randn((M, K + 3), generator=g).to(dt)
    for w in (W[:, :K], W[:, 3:], W[:, :K].contiguous(), W[:, :K].t().contiguous().t(), W[:, torch.arange(0, K, 2)]):
        a = strp.aligned_rows(w)
        assert torch.equal(a, w) and a.dtype == dt
        assert a.stride(1) == 1 or a.shape[1] == 1
        assert a.stride(0) % 8 == 0 and a.stride(0) >= (a.shape[1] + 7) // 8 * 8 and a.data_ptr() % 16 == 0
        assert strp.aligned_rows(a) is a          # nothing to do a second time
        assert a.untyped_storage().nbytes() >= a.storage_offset() * a.element_size() + M * a.stride(0) * a.element_size()          # the last row's eights are there too
