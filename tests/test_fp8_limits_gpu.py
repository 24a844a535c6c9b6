"""8-bit operators at the ends of the extents that they accept, on the GPU; rows are sampled.  Bounds as in tests/test_fp8_gpu.py."""
import numpy as np
import pytest
import torch

from oracle import ref_fp8 as rf
from oracle import ref_numpy as rn
from paper_2604_27089_amd import binding as sp
from test_fp8_gpu import EPS, check_norm_operand
from gpu_util import host_f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,C,res", [((1 << 24) + 5, 8, True), ((1 << 24) + 5, 64, False), ((1 << 22) + 1, 264, True)])
def test_norm_of_more_rows_than_one_launch_dimension_holds(T, C, res):
    """2^24 rows with 256 threads each are 2^32 threads.  Rows on either side of every 2^22, first and last: the bits of the same rows
    alone, and the oracle's values."""
    g = torch.Generator(device="cuda").manual_seed(T + C)
    x = torch.empty((T, C), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    r = torch.empty((T, C), dtype=torch.bfloat16, device="cuda").normal_(generator=g) if res else None
    w = torch.empty(C, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    h, q, qs, rstd = sp.sp_rmsnorm_fp8_fwd(x, w, EPS, res=r)
    for at in [0, *range((1 << 22) - 8, T - 16, 1 << 22), T - 16]:
        part = slice(at, at + 16)
        h2, q2, qs2, rstd2 = sp.sp_rmsnorm_fp8_fwd(x[part], w, EPS, res=None if r is None else r[part])
        assert torch.equal(h[part], h2) and torch.equal(q[part].view(torch.uint8), q2.view(torch.uint8)), at
        assert torch.equal(qs[:, part].view(torch.uint8), qs2[:, :16].view(torch.uint8)) and torch.equal(rstd[part], rstd2), at
        _, y, _ = rf.norm_fwd(host_f64(h2), None, host_f64(w), EPS, None)
        check_norm_operand(q2, qs2, y, f"rows from {at}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N", [((1 << 27) + 5, 1), ((1 << 26) + 1, 3)])
def test_product_without_contraction_of_many_rows(M, N, dtype):
    """16 rows a workgroup of 512 threads: 2^27 rows are 2^32 threads."""
    z = lambda R: torch.empty((R, 0), dtype=torch.float8_e4m3fn, device="cuda")  # noqa: E731
    e = lambda R: torch.empty((0, (R + 15) // 16 * 16), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)  # noqa: E731
    out = torch.full((M, N), 7.0, device="cuda", dtype=dtype)
    sp.sp_fp8_matmul(z(M), e(M), z(N), e(N), out=out)
    assert not out.any()
