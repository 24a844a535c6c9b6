"""8-bit operators at the ends of the extents that they accept, on the GPU; rows are sampled.  Bounds as in tests/test_fp8_gpu.py."""
import numpy as np
import pytest
import torch

from oracle import ref_fp8 as rf
from oracle import ref_numpy as rn
from paper_2604_27089_amd import binding as sp
from test_fp8_gpu import E8M0, EPS, TYPE, awkward, bits, check_norm_operand, check_operand, check_product
from gpu_util import dev_bf16, host_f64

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


# ------------------------------------------------------------------ conversion of a norm's output with values that are not finite
@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("T,C", [(1, 8), (9, 64), (37, 520), (129, 136), (300, 1000)])
def test_quant_of_the_norm_of_awkward_values(T, C, kind):
    """x * rstd * w is two multiplications in fp32, which numpy does alike, so the conversion is compared bit for bit: NaN and infinities
    in x, in rstd and in w, zeros against infinities, products that overflow or are denormal, in ragged tiles and beside finite blocks."""
    r = np.random.default_rng([T, C])
    xb, wb = awkward(T + C, T, C), bits(C, (C,))
    rstd = np.exp(r.standard_normal(T) * 8).astype(np.float32)
    if C > 16:
        wb[C - 1], wb[11] = 0x7F80, 0x7FC0
    if T > 8:
        rstd[5], rstd[6], rstd[7], rstd[T - 2] = np.inf, np.nan, 0.0, 1e38
    with np.errstate(all="ignore"):
        v = (rn.widen_bf16(xb).astype(np.float32) * rstd[:, None]) * rn.widen_bf16(wb).astype(np.float32)
    v = v.astype(np.float64)
    for rows, cols in ((True, True), (True, False), (False, True)):
        q, qs, qt, qts = sp.sp_fp8_quant(dev_bf16(xb), TYPE[kind], rows=rows, cols=cols, rstd=torch.from_numpy(rstd).cuda(), w=dev_bf16(wb))
        if rows:
            check_operand(q, qs, v, kind, "rows")
        if cols:
            check_operand(qt, qts, np.ascontiguousarray(v.T), kind, "columns")


# ------------------------------------------------------------------ product at the largest extents
def operand_on_gpu(seed, R, K, kind):
    """Any finite bytes, exponents near 127, made on the GPU: (bytes, exponents)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    b = torch.randint(0, 256, (R, K), dtype=torch.uint8, device="cuda", generator=g)
    least = 0x7F if kind == "e4m3" else 0x7C  # of the magnitudes that are not finite
    b[(b & 0x7F) >= least] = 0x38
    return b, torch.randint(124, 131, (K // 128, (R + 15) // 16 * 16), dtype=torch.uint8, device="cuda", generator=g)


def check_samples(M, N, K, kind, rows, cols):
    (a, ea), (b, eb) = operand_on_gpu(1, M, K, kind), operand_on_gpu(2, N, K, "e4m3")
    ri, ci = torch.tensor(rows, device="cuda"), torch.tensor(cols, device="cuda")
    host = lambda t: t.contiguous().cpu().numpy()  # noqa: E731
    for dtype in (torch.bfloat16, torch.float32):
        out = sp.sp_fp8_matmul(a.view(TYPE[kind]), ea.view(E8M0), b.view(TYPE["e4m3"]), eb.view(E8M0), out_dtype=dtype)
        check_product(out[ri][:, ci], host(a[ri]), host(ea[:, ri]), host(b[ci]), host(eb[:, ci]), kind, what=f"{dtype}")
        del out


@pytest.mark.parametrize("M,kind", [(1, "e4m3"), (40, "e5m2"), (300, "e4m3"), (513, "e5m2")])
def test_product_of_the_most_columns(M, kind):
    N = 1 << 22
    check_samples(M, N, 128, kind, sorted({0, M // 2, M - 1}), [0, 1, 255, 256, N // 2 - 1, N // 2, N - 257, N - 256, N - 1])


@pytest.mark.parametrize("M,N,kind", [(1, 70, "e4m3"), (300, 70, "e5m2"), (300, 1030, "e4m3")])
def test_product_of_the_longest_contraction(M, N, kind):
    check_samples(M, N, 1 << 22, kind, sorted({0, M // 2, M - 1}), [0, 1, 64, N - 1])
