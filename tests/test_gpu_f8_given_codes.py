"""Given codes of tokens at the limit of few rows, which both the workspace's size and the call have to place alike although the call knows the inner
dimension by whole runs of 128 only."""
import pytest
import torch

from f8_plain import BF16, F32, small_integers
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("t,n,k", [(16, 33000, 1000), (40, 5500, 1000), (1, 270000, 100), (17, 4200, 1990)])
def test_given_codes_at_the_limit_of_few_rows(t, n, k):
    g = torch.Generator().manual_seed(t)
    X, W = small_integers((t, k), g, 3), torch.randint(-3, 4, (n, k), generator=g).double()
    xc, xs = torch.empty(t, oz.f8_row_bytes(k), dtype=torch.uint8, device=DEV), torch.empty(t, oz.f8_scale_bytes(k), dtype=torch.uint8, device=DEV)
    codes, scales = torch.empty(n, oz.f8_row_bytes(k), dtype=torch.uint8, device=DEV), torch.empty(-(-n // 128), oz.f8_scale_bytes(k), dtype=torch.uint8, device=DEV)
    oz.f8_split(X.float().to(DEV), xc, xs, 1)
    oz.f8_split(W.float().to(DEV), codes, scales)
    want = (X.to(DEV) @ W.to(DEV).t()).float()
    for dt in (BF16, F32):
        Y = torch.full((t, n), 77.0, dtype=dt, device=DEV)
        oz.f8_gemm(xc, codes, scales, Y, oz.alloc_f8_workspace("gemm", t, n, k, torch.uint8), x_scales=xs)
        assert torch.equal(Y, want.to(dt))
