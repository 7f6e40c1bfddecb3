"""The largest problems that the products by expert and in 8 bits take, and the first ones that they refuse, as the header has them."""
import pytest

import api_stub

A = 0x1000          # never dereferenced: launches are lines in a log
SHAPE = -2


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    L = api_stub.build(tmp_path_factory.mktemp("limits"))
    L.stub_reset(b"", 0)
    return L


def _dx(L, R, E, K, N):
    return L.ffuse_grouped_gemm_dx(0, A, A, A, R, E, K, N, A, None)


def _dw(L, R, E, K, N):
    return L.ffuse_grouped_gemm_dw(0, A, A, A, R, E, K, N, A, None)


def _fp8(L, M, K, N):
    return L.ffuse_gemm_fp8(0, A, A, A, A, 1, M, K, N, A, None)


def _quantise(L, M, K):
    return L.ffuse_fp8_quantize(0, A, M, K, 1, 0, A, A, None)


def test_grouped(lib):
    top = 1 << 31
    for call in (_dx, _dw):
        for good, bad in (((4, 2, 1 << 20, 8), (4, 2, (1 << 20) + 8, 8)), ((4, 2, 8, 1 << 20), (4, 2, 8, (1 << 20) + 8)), ((4, 1024, 8, 8), (4, 1025, 8, 8)),
                          ((4, 1, 1 << 15, 32640), (4, 1, 1 << 15, 32648)),                  # (K + 128) N 2 against 2^31
                          ((top - 513, 1, 8, 8), (top - 512, 1, 8, 8)),
                          ((16 * 1023, 1, 1 << 20, 8), (16 * 65536, 1, 1 << 20, 8)),         # (R / 16 + E) (K / 32 + 1) against 2^31
                          ((16 * 65533, 1, 1 << 20, 8), (16 * 65534, 1, 1 << 20, 8))):
            assert call(lib, *good) == 0 and call(lib, *bad) == SHAPE, (call.__name__, good, bad)
    assert _dw(lib, 4, 511, 16384, 16384) == 0 and _dw(lib, 4, 512, 16384, 16384) == SHAPE and _dx(lib, 4, 512, 16384, 16384) == 0


def test_8_bits(lib):
    for good, bad in (((4, 1 << 20, 8), (4, (1 << 20) + 16, 8)), ((4, 16, 1 << 20), (4, 16, (1 << 20) + 8)), ((4, 16, 8), (4, 0, 8)),
                      ((4, 65536 - 128, 32760), (4, 65536 - 128, 32768)), ((0, 16, 8), (-1, 16, 8)), (((1 << 31) - 513, 16, 8), ((1 << 31) - 512, 16, 8))):
        assert _fp8(lib, *good) == 0 and _fp8(lib, *bad) == SHAPE, (good, bad)
    for good, bad in (((64 * 16382, 65408), (64 * 16383, 65408)), ((64 * 1022, 1 << 20), (64 * 1024, 1 << 20)), ((4, 1 << 20), (4, (1 << 20) + 8)), ((4, 8), (4, 0))):
        assert _quantise(lib, *good) == 0 and _quantise(lib, *bad) == SHAPE, (good, bad)
