"""Extents that need 2^32 threads in one dimension of a launch are refused before it: the runtime would run a part of the threads and
report no error.  Only refused calls here: the addresses stand for nothing."""
import ctypes

from paper_2604_27089_amd import binding as sp


def A(n):
    return ctypes.c_void_p(0x1000 * n)


def test_conversion():
    f = sp.lib().sp_fp8_quant
    for T, C in (((1 << 31) - 1, 8), ((1 << 30) + 1, 136), (1 << 24, 16512)):
        for seven in ([A(1), None, None, A(2), A(3), None, None], [A(1), None, None, None, None, A(2), A(3)], [A(i) for i in range(1, 8)]):
            assert f(*seven, T, C, 0, None) == sp.SP_ERR_SHAPE, (T, C)


def test_product_in_fp32():
    f = sp.lib().sp_fp8_matmul
    for M, N in (((1 << 31) - 1, 1), ((1 << 31) - 127, 128), (1 << 20, 1 << 18), (1 << 22, 1 << 16)):
        for kind in (0, 1):
            assert f(*[A(i) for i in range(1, 6)], M, N, 128, kind, 1, 0, None) == sp.SP_ERR_SHAPE, (M, N)


def test_norm_rotary_and_gate():
    L = sp.lib()
    for T in (1 << 26, (1 << 26) + 5, 1 << 32):
        assert L.sp_rmsnorm_fwd(*[A(i) for i in range(1, 5)], T, 8, 1e-5, None) == sp.SP_ERR_SHAPE
    for T, H, D in ((1 << 28, 1, 256), (1 << 25, 16, 128), (1 << 31, 32, 64)):
        assert L.sp_rope(*[A(i) for i in range(1, 5)], T, H, D, 0, None) == sp.SP_ERR_SHAPE
    for n in (1 << 35, (1 << 35) + 8, 1 << 40):
        assert L.sp_swiglu_fwd(A(1), A(2), A(3), n, None) == sp.SP_ERR_SHAPE
        assert L.sp_swiglu_bwd(*[A(i) for i in range(1, 6)], n, None) == sp.SP_ERR_SHAPE


def test_attention():
    L = sp.lib()
    B, Hq = 65535, 256  # a workgroup of 512 threads for each head of each batch entry
    assert L.sp_attn_fwd(*[A(i) for i in range(1, 6)], B, 1, Hq, Hq, 64, 0.125, None) == sp.SP_ERR_SHAPE
    assert L.sp_attn_merge(*[A(i) for i in range(1, 6)], 1, 1 << 20, 1 << 8, 64, None) == sp.SP_ERR_SHAPE
    assert L.sp_attn_merge(*[A(i) for i in range(1, 6)], 1, 1 << 20, 1 << 7, 128, None) == sp.SP_ERR_SHAPE


def test_product_past_its_largest_extents():
    f, five = sp.lib().sp_fp8_matmul, [A(i) for i in range(1, 6)]
    for M, N, K in ((4, (1 << 22) + 1, 128), (4, 4, (1 << 22) + 128), (1 << 31, 4, 128)):
        for out_type in (0, 1):
            assert f(*five, M, N, K, 0, out_type, 0, None) == sp.SP_ERR_SHAPE
        assert sp.sp_fp8_matmul_workspace_bytes(M, N, K) == 0
