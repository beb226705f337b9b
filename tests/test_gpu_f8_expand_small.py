"""Values of codes under 32-bit scales: each is the product rounded once to 32 bits, also where that is subnormal."""
import pytest
import torch

from f8_plain import BF16, F16, F32, decode
from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("low,high", [(-149, -140), (-140, -118), (-30, 30), (100, 128)])
def test_expand_rounds_once(low, high, block_rows):
    n, groups = 512, 16
    g = torch.Generator().manual_seed(high)
    codes = torch.arange(256, dtype=torch.uint8).repeat(n, groups // 2)
    codes[(codes & 127) == 127] ^= 1
    rows = n // block_rows
    scales = (torch.ldexp(1.0 + torch.rand(rows, groups, generator=g).double(), torch.randint(low, high, (rows, groups), generator=g)) *
              torch.where(torch.rand(rows, groups, generator=g) < 0.5, -1.0, 1.0)).to(F32)
    want = decode(codes) * scales.double().repeat_interleave(block_rows, 0).repeat_interleave(128, 1)      # (28 bits: exact)
    for dt in (F32, BF16, F16):
        out = torch.empty(n, groups * 128, dtype=dt, device=DEV)
        oz.f8_expand(codes.to(DEV), scales.to(DEV), out, block_rows)
        assert torch.equal(out.cpu(), want.to(F32).to(dt))
