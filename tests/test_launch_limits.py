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
