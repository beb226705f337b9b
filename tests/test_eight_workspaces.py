"""A workspace for given codes serves the call, whose inner dimension is known by whole runs of 128 only. No GPU."""
import pytest
import torch

from paper_2306_11975_amd import ozimmu as oz


@pytest.mark.parametrize("experts", [0, 5])
def test_workspace_of_given_codes_counts_whole_runs(experts):
    """About the limit of few rows, where the operator begins to need one."""
    needed = 0
    for t, k in ((1, 1), (1, 129), (16, 1000), (17, 1000), (33, 1900), (64, 8000), (200, 520), (5000, 130)):
        padded = oz.f8_row_bytes(k)
        runs = t // 16 + min(experts, t) if experts else 0.5 if t <= 16 else -(-t // 16)
        for limit in (k, padded):
            for n in range(max(1, int(2 ** 24 / runs / limit) - 2), int(2 ** 24 / runs / limit) + 3):
                if n <= 1 << 22:
                    size = oz.f8_workspace_bytes("gemm", t, n, k, torch.uint8, experts=experts)
                    assert size == oz.f8_workspace_bytes("gemm", t, n, padded, torch.uint8, experts=experts)
                    needed += size > 0
    assert needed or experts      # (over experts tiles are not shared, so given codes need none)
