"""Products of tokens with one value far above the others, under codes that are zero there and under codes that are not: errors go by the terms of the sum, not by the largest value of a
token."""
import pytest
import torch

from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def half_step(dt):
    return torch.finfo(dt).eps / 2


# one token and two, every tile of the passes, tiles, and the product
CASES = [(1, 300, 600, 64), (2, 50, 700, 32), (2, 5000, 256, 32), (2, 5000, 1024, 128), (3, 64, 256, 64), (3, 64, 1024, 128), (5, 100, 2500, 32), (16, 500, 3000, 64), (16, 8200, 300, 128), (16, 16400, 257, 32),
         (20, 90, 1000, 32), (33, 300, 2049, 128), (40, 9000, 130, 64), (64, 60, 900, 128), (300, 2000, 200, 64), (2000, 2100, 2570, 32)]


def by_type():
    for case in CASES:
        for dt, outlier in ((F16, 1.0e4), (F16, 6.0e4), (BF16, 2.0 ** 14), (BF16, 2.0 ** 20), (BF16, 2.0 ** 24), (BF16, 2.0 ** 100), (F32, 2.0 ** 20), (F32, 2.0 ** 60)):
            if dt != F32 or oz.q4_workspace_bytes(*case, dt) == 0:     # (two slices of a row hold 2^-39 of its largest value)
                yield (*case, dt, outlier)


@pytest.mark.parametrize("t,n,k,group,dt,outlier", by_type())
def test_one_large_value_in_a_token(t, n, k, group, dt, outlier):
    """Codes and tokens are exact operands of the sums, whose products are exact and which are formed in 32 bits: a sum of `k` terms, in whatever order, is off by at most k + 8 roundings (of
    sums, and of the scales' products with them) of the sum of the terms' magnitudes, where a rounding of the matrix cores may be a cut (2^-23). Then one rounding of the result; beyond
    16 tokens of 16-bit types one of every weight too."""
    g = torch.Generator().manual_seed(t + n + k)
    c = torch.randint(-8, 8, (n, k), generator=g)
    s = ((torch.rand(n, -(-k // group), generator=g) + 0.5) * 2.0 ** -8).to(dt)
    X = torch.randn(t, k, generator=g)
    at = torch.randint(0, k, (t,), generator=g)
    at[0] = 0
    at[-1] = k - 1
    X[torch.arange(t), at] = outlier * torch.where(torch.rand(t, generator=g) < 0.5, 1.0, -1.0)
    X = X.to(dt)
    # rows without a code at any of the large values, and rows without one at a third of them
    c[0::4, at] = 0
    c[1::4, at[::3]] = 0
    room = oz.q4_row_bytes(k)
    packed = torch.nn.functional.pad(c, (0, 2 * room - k)) + 8
    codes = (packed[:, 0::2] | (packed[:, 1::2] << 4)).to(torch.uint8).to(DEV)
    Y = torch.empty(t, n, dtype=dt, device=DEV)
    oz.q4_gemm(X.to(DEV), codes, s.to(DEV), group, Y, oz.alloc_q4_workspace(t, n, k, group, dt))
    W = c.double() * s.double().repeat_interleave(group, dim=1)[:, :k]
    want, terms = X.double() @ W.t(), X.double().abs() @ W.abs().t()
    bound = (k + 8) * 2.0 ** -23 * terms + (half_step(dt) * terms if dt != F32 and t > 16 else 0.0)
    bound = bound + half_step(dt) * (want.abs() + bound)
    beyond = want.abs() + bound >= torch.finfo(dt).max     # (may be an infinity)
    got = Y.cpu().double()
    off = torch.where(beyond & ~got.isfinite() & ~got.isnan(), torch.zeros_like(want), (got - want).abs())
    assert (off <= bound).all(), f"off by up to {float((off / bound).max()):.3g} times what roundings can do"
    # where the large values meet zeros only, the result's own rounding (and the weights') is what is left, in the norm too
    quiet = want[:, 0::4]
    if quiet.numel() > 64:
        rel = float((got - want)[:, 0::4].norm() / quiet.norm())
        assert rel <= (2e-6 if dt == F32 else 1.5 * half_step(dt)), rel
