"""slim_block_fp8_gemm_plan (host logic, nothing is launched): its refusals, and what it says of a layer's sizes."""
import ctypes

import pytest
import torch

from paper_2410_09615_amd import binding as B


def test_refuses():
    f, out = B.lib().slim_block_fp8_gemm_plan, (ctypes.c_int32 * 6)()
    assert f(64, 256, 4, 0, None) == B.SLIM_ERR_NULL
    for bad in ((0, 256, 4, 0), (64, 0, 4, 0), (64, (1 << 22) + 1, 4, 0), (64, 256, 0, 0), (64, 256, 4, 3), (64, 256, 4, -1)):
        assert f(*bad, out) == B.SLIM_ERR_SHAPE, bad


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,k", [(1, 1), (300, 700), (4096, 4096), (5120, 5120), (10007, 4100), (28672, 8192)])
def test_workgroups_cover_the_result(n, k, dtype):
    """Up to 64 tokens one column of workgroups, summed in binary32 whatever the type; above, tiles, in binary32 for fp32 results."""
    for m in (1, 16, 17, 48, 64, 65, 128, 333, 1000, 4096):
        p = B.slim_block_fp8_gemm_plan(n, k, m, dtype)
        few = m <= 64
        assert p["kernel"] == ("stream" if few else "tile") and p["binary32"] == (few or dtype == torch.float32)
        rows = -(-n // 64) * 64 if few else n                          # (streamed weights: whole tiles of 64 rows)
        assert p["workgroups"] == -(-rows // p["rows"]) * -(-m // p["tokens"])
        assert p["threads"] % 64 == 0 and 64 <= p["threads"] <= 512 and (not few or p["threads"] <= 64 * -(-k // 128))
