"""The plain statements that the GPU tests of the few-bit calls compare with, against themselves and their bounds (no GPU)."""
import math

import pytest
import torch

import few_bits as F


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_held_value_is_the_group_by_group_one(dtype):
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(40, 128, generator=g) * 3 + torch.randn(40, 1, generator=g) * 5).to(dtype)
    x[3] = 0
    x[4, :64] = 1.5
    x[5, 7] = math.inf
    x[6, 100] = math.nan
    x[7] = torch.arange(128).to(dtype)                      # values between two codes
    held = F.held_value(x)
    for i in range(40):
        for j in range(2):
            lo, step, codes = F.quantize_group(x[i, 64 * j: 64 * j + 64])
            want = torch.tensor([lo + step * c for c in codes], dtype=torch.float64)
            assert torch.equal(held[i, 64 * j: 64 * j + 64].nan_to_num(7.0), want.nan_to_num(7.0))
            if math.isfinite(lo):
                off = (want - x[i, 64 * j: 64 * j + 64].double()).abs().max()
                assert off <= step / 2


def test_page_bytes():
    import paper_1610_02132_b200 as Q
    for dim in (64, 128, 192, 256):
        for page in (16, 48, 128):
            x = torch.zeros(page, dim, dtype=torch.bfloat16)
            assert len(F.cache_bytes(x, x)) * 3 == Q.qsgd_cache_page_bytes(page, 3, dim)
    for bad in ((15, 1, 64), (16, 0, 64), (16, 1, 96), (0, 1, 64), (2 ** 17, 1, 64), (16, 2 ** 17, 64)):
        assert Q.qsgd_cache_page_bytes(*bad) == 0
