"""The choice of a kernel for the product of 8-bit operands (a host function of sizes alone), on both sides of its lines.  No kernel is launched here."""
import pytest

from fp8_reference import kernel_of

FEW_Y, FEW_CODES, RING128, RING256 = range(4)


@pytest.mark.parametrize("N,C,K,Nout,rows8,act,want", [
    # y alone: 32 x 32 tiles up to two a CU
    (1, 16, 1024, 4096, False, "none", FEW_Y), (1, 128, 1024, 4096, False, "gelu", FEW_Y), (1, 129, 1024, 4096, False, "none", RING128),
    (1, 128, 1024, 4104, False, "none", RING128), (512, 1, 64, 32, False, "relu", FEW_Y), (513, 1, 64, 32, False, "relu", RING128),
    # 8-bit rows: 32 x 128 tiles up to one a CU, contractions of four blocks or less
    (1, 128, 512, 8192, True, "gelu", FEW_CODES), (1, 129, 512, 8192, True, "gelu", RING128), (1, 128, 512, 8200, True, "none", RING128),
    (1, 128, 520, 8192, True, "gelu", RING128), (1, 1, 8, 8, True, "none", FEW_CODES), (1, 1, 520, 8, True, "none", RING128),
    # 128 x 256 tiles: contractions of sixteen blocks or more, no activation, four rounds
    (128, 256, 2048, 512, False, "none", RING128), (128, 256, 2048, 1024, False, "none", RING256), (128, 256, 1920, 1024, False, "none", RING128),
    (128, 256, 2048, 1024, False, "gelu", RING128), (128, 256, 2048, 1024, True, "none", RING128), (128, 128, 1928, 1920, False, "none", RING256),
    (128, 128, 1928, 1792, False, "none", RING128),
    # the limits
    (4096, 32768, 32768, 32768, False, "none", RING256), (4096, 32768, 32768, 32768, True, "gelu", RING128), (1, 1 << 27, 8, 32768, False, "relu", RING128),
])
def test_kernel_of_a_product(N, C, K, Nout, rows8, act, want):
    assert kernel_of(256, N, C, K, Nout, rows8, act) == want
