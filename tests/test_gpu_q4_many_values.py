"""Weights of more values than the threads of one launch: 4194304 x 8224, 17 GB of codes, 69 GB of 16-bit weights or of a product's operand."""
import pytest
import torch

from paper_2306_11975_amd import ozimmu as oz

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16 = torch.float16
N, K, GROUP = 1 << 22, 8224, 128
PART = 1 << 18      # rows of a call that is one launch


@pytest.fixture(scope="module")
def weights():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 140 << 30:
        pytest.skip("takes 110 GB of the GPU's memory")
    g = torch.Generator(device=DEV).manual_seed(1)
    codes = torch.randint(0, 256, (N, oz.q4_row_bytes(K)), generator=g, dtype=torch.uint8, device=DEV)
    scales = (torch.rand(N, -(-K // GROUP), generator=g, device=DEV) + 0.5).to(F16)
    yield codes, scales
    del codes, scales
    torch.cuda.empty_cache()


def test_expansion_and_cut(weights):
    codes, scales = weights
    W = torch.empty(N, K, dtype=F16, device=DEV)
    W.fill_(float("nan"))
    oz.q4_expand(codes, scales, GROUP, W)
    part = torch.empty(PART, K, dtype=F16, device=DEV)
    for r in range(0, N, PART):
        oz.q4_expand(codes[r:r + PART], scales[r:r + PART], GROUP, part)
        assert torch.equal(part, W[r:r + PART]), r
    cut, s = torch.zeros_like(codes), torch.zeros_like(scales)
    oz.q4_split(W, GROUP, cut, s)
    part_cut, part_s = torch.zeros_like(codes[:PART]), torch.zeros_like(scales[:PART])
    for r in range(0, N, PART):
        oz.q4_split(W[r:r + PART], GROUP, part_cut, part_s)
        assert torch.equal(part_cut, cut[r:r + PART]) and torch.equal(part_s, s[r:r + PART]), r
    assert int(cut[-1].max()) > 0
    del W, part, cut, s, part_cut, part_s
    torch.cuda.empty_cache()


def test_product(weights):
    """1536 tokens: six tiles of 256, and in both calls whole rounds of them, so that a part of the outputs is the same tiles, and the same bits."""
    codes, scales = weights
    t = 1536
    X = torch.randn(t, K, device=DEV).to(F16)
    Y = torch.empty(t, N, dtype=F16, device=DEV)
    ws = oz.alloc_q4_workspace(t, N, K, GROUP, F16)
    assert oz.q4_workspace_bytes(t, N, K, GROUP, F16) > 0 and oz.q4_workspace_bytes(t, PART, K, GROUP, F16) > 0
    ws.fill_(0xFF)
    oz.q4_gemm(X, codes, scales, GROUP, Y, ws)
    part = torch.empty(t, PART, dtype=F16, device=DEV)
    for r in range(0, N, PART):
        oz.q4_gemm(X, codes[r:r + PART], scales[r:r + PART], GROUP, part, ws)
        assert torch.equal(part, Y[:, r:r + PART]), r
    assert Y.isfinite().all()
    del ws, Y, part
    torch.cuda.empty_cache()


def test_gradient(weights):
    """Gradients that are zero but for some rows, which 64 bits are enough to check; what of the operand was not written would be NaN."""
    codes, scales = weights
    t, rows = 64, 2048
    ws = oz.alloc_q4_workspace(t, N, K, GROUP, F16, gradient=True)
    R = torch.empty(t, K, dtype=F16, device=DEV)
    for r in (0, N // 2 - 1000, N - rows):
        ws.fill_(0xFF)
        D = torch.zeros(t, N, dtype=F16, device=DEV)
        D[:, r:r + rows] = torch.randn(t, rows, device=DEV)
        oz.q4_gemm_grad(D, codes, scales, GROUP, R, ws)
        c = torch.stack((codes[r:r + rows] & 15, codes[r:r + rows] >> 4), dim=2).view(rows, -1)[:, :K].double() - 8
        W = c * scales[r:r + rows].double().repeat_interleave(GROUP, dim=1)[:, :K]
        V = D[:, r:r + rows].double()
        want, terms = V @ W, V.abs() @ W.abs()
        half = torch.finfo(F16).eps / 2
        # a rounding of every weight, sums of `rows` terms in 32 bits, a rounding of the result
        bound = half * terms + (rows + 8) * 2.0 ** -23 * terms
        assert ((R.double() - want).abs() <= bound + half * (want.abs() + bound)).all()
    del ws, D, R
    torch.cuda.empty_cache()
