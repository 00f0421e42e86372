"""Long sums in every kind of tiles of the products with blocks of 128 and of grouped rows: more stages than the scales or exponents
that a tile holds at a time, whole and with an end inside a stage.  Bars as in the tests of these products (plain 64-bit forms)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2511_05811_amd as moss
from gpu_util import to_gpu
from test_gpu_block128 import check_product, operands, values
from test_gpu_grouped import Dw, Rows

pytestmark = pytest.mark.gpu


def tile(name, *args):
    fn = getattr(moss.load(), name)
    fn.restype = C.c_int
    return fn(*(C.c_int64(a) for a in args))


@pytest.mark.parametrize("M,N,K,b_block,expected", [(33, 96, 32768 + 32, 128, 32032), (33, 96, 32768 + 32, 1, 32032), (513, 2052, 4128, 128, 64064),
                                                    (513, 2052, 8256, 1, 64064), (700, 2304, 8224, 1, 64128), (512, 4096, 4096, 128, 64128),
                                                    (640, 4096, 8224, 128, 128128), (1100, 2304, 4096 + 96, 1, 128128), (1030, 4096, 8224, 1, 128256),
                                                    (2050, 4104, 2112, 128, 128256), (4000, 4104, 4128, 128, 256256), (3000, 3080, 4128, 1, 256256)])
def test_block_products(M, N, K, b_block, expected):
    assert tile("moss_internal_gemm_block_tile", M, N, K, b_block, N) == expected
    a, a_s, b, b_s = operands(M, N, K, b_block, M + N + K)
    got = moss.gemm_fp8_block128(*(to_gpu(t) for t in (a, a_s, b, b_s)), out_dtype=torch.float32)
    check_product(got, values(a, a_s, 1), values(b, b_s, b_block))


@pytest.mark.parametrize("sizes,N,K,expected", [([3, 0, 1, 70, 33], 264, 32768 + 32, 32032), ([3, 0, 100, 1, 20, 61, 64, 2] * 4, 768, 8224, 64128),
                                                ([128, 0, 1, 256, 515, 0, 0], 2560, 8224, 128128), ([0, 1, 130, 37] * 10, 4104, 4128, 128256),
                                                ([0, 1, 256, 1703, 400, 633, 7], 2056, 8192, -128256)])
def test_grouped_rows(sizes, N, K, expected):
    p = Rows(np.concatenate([[0], np.cumsum(sizes)]), N, K)
    assert tile("moss_internal_gemm_grouped_tile", p.R, N, K, p.G, 1, N) == expected
    p.check(moss.gemm_fp8_mx_grouped(**p.args(out_dtype=torch.float32)))


@pytest.mark.parametrize("sizes,M,N,expected", [([32, 6208, 0, 32] + [32] * 36, 264, 136, 128128), ([32, 6016, 0, 32, 64, 32, 0, 64], 520, 1672, 128256),
                                                ([32, 8160, 0, 32, 0, 0], 1120, 1672, 256256)])
def test_grouped_weight_gradients(sizes, M, N, expected):
    p = Dw(np.concatenate([[0], np.cumsum(sizes)]), M, N)
    assert tile("moss_internal_gemm_grouped_dw_tile", p.R, M, N, p.G) == expected
    p.check(moss.gemm_fp8_mx_grouped_dw(**p.args()))
