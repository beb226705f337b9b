"""What stands beyond the last position of a row of four-bit codes counts for nothing, whatever it is and however large the row's scales are."""
import pytest
import torch

from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16

# Scales with which 7 s is a value of the type and 8 s is not: the code -8 of a padding of zero bytes would be an infinity.
TOP = {F16: 8500.0, BF16: 4.5e37, F32: 4.5e37}
# Tokens that keep the results inside the type (fp16: a term is 7 * 8500 * 2^-16 = 0.9 times a normal value)
SIZE = {F16: 2.0 ** -16, BF16: 2.0 ** -20, F32: 2.0 ** -20}

# Rows that end in every part of a byte, of a piece of 16 bytes and of a group; for one token and two, passes, tiles of both sizes, and the product.
CASES = [(1, 70, 621, 32), (2, 2100, 1000, 128), (3, 50, 7, 32), (5, 100, 333, 64), (16, 300, 1, 32), (20, 100, 2500, 32), (40, 130, 77, 128),
         (300, 2000, 100, 32), (300, 2000, 101, 64), (290, 2001, 9, 32), (257, 2050, 63, 128), (64, 8200, 200, 32), (1000, 1030, 129, 64),
         (2000, 2100, 513, 64), (2000, 4130, 66, 32), (2000, 2100, 2571, 32), (4000, 300, 2001, 32)]


def fill_padding(codes, k, how):
    """A copy of the codes (n x row bytes) with other values beyond position k."""
    c = codes.clone()
    n, room = c.shape
    g = torch.Generator().manual_seed(k)
    what = {"zeros": torch.zeros(n, room, dtype=torch.uint8), "ones": torch.full((n, room), 0xFF, dtype=torch.uint8),
            "random": torch.randint(0, 256, (n, room), generator=g, dtype=torch.uint8)}[how]
    whole = (k + 1) // 2
    c[:, whole:] = what[:, whole:]
    if k % 2:
        c[:, k // 2] = (c[:, k // 2] & 15) | (what[:, k // 2] & 0xF0)
    return c


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("t,n,k,group", CASES)
def test_padding_is_ignored(t, n, k, group, dt):
    g = torch.Generator().manual_seed(t + n + k)
    c = torch.randint(-7, 8, (n, k), generator=g)
    room = oz.q4_row_bytes(k)
    c = torch.nn.functional.pad(c, (0, 2 * room - k)) + 8
    clean = (c[:, 0::2] | (c[:, 1::2] << 4)).to(torch.uint8)
    scales = (torch.rand(n, -(-k // group), generator=g) + 0.5) * 2.0 ** -10
    scales[::3] = TOP[dt]                                # every third row
    scales[1::3, -1] = TOP[dt]                           # and the last group, which the padding is in, of every third
    scales = scales.to(dt).to(DEV)
    X = (torch.randn(t, k, generator=g) * SIZE[dt] / (k ** 0.5 if dt != F16 else 1.0)).to(dt).to(DEV)
    D = (torch.randn(t, n, generator=g) * SIZE[dt] / n ** 0.5).to(dt).to(DEV)
    wf, wg = oz.alloc_q4_workspace(t, n, k, group, dt), oz.alloc_q4_workspace(t, n, k, group, dt, gradient=True)

    def results(codes):
        Y, R, W = torch.empty(t, n, dtype=dt, device=DEV), torch.empty(t, k, dtype=dt, device=DEV), torch.empty(n, k, dtype=dt, device=DEV)
        oz.q4_gemm(X, codes, scales, group, Y, wf)
        oz.q4_gemm_grad(D, codes, scales, group, R, wg)
        oz.q4_expand(codes, scales, group, W)
        return Y, R, W

    want = results(clean.to(DEV))
    assert all(w.isfinite().all() for w in want)
    for how in ("zeros", "ones", "random"):
        for got, w in zip(results(fill_padding(clean, k, how).to(DEV)), want):
            assert torch.equal(got, w), how
