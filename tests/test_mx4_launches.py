"""Products of microscaled 4-bit floating point, without a GPU: sizes that no kind of tiles launches are refused as shapes before the device is asked for anything."""
import ctypes

from tests.test_mx4_rotary_abi import BIG, P, _mx4, b  # noqa: F401


def test_sizes_past_every_kind_of_tiles(b):  # noqa: F811
    L = b.lib()

    def linear(M, N):
        return L.w4a4_mx4_linear(ctypes.byref(_mx4(b, rows=M, K=32)), ctypes.byref(_mx4(b, rows=N, K=32)), None, 0, 0, P, None)

    def a16(M, N):
        return L.w4a4_mx4_linear_a16(P, 0, M, 32, ctypes.byref(_mx4(b, rows=N, K=32)), None, 0, P, None)

    # tiles of 32 x 32 from 2^22 channels on, of 256 x 256 below; 2^23 workgroups of 512 threads are 2^32 threads
    for M, N in ((1, 1 << 28), (33, 1 << 27), (1 << 10, 1 << 23), (1 << 20, 1 << 22), (BIG, 8), (1 << 30, 512), (1 << 25, (1 << 22) - 8)):
        assert linear(M, N) == -2, (M, N)
    for M, N in ((1, BIG - 7), (33, 1 << 30), (1 << 15, 1 << 21), (1 << 30, 64), (BIG, 8)):
        assert a16(M, N) == -2, (M, N)
