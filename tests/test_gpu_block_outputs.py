"""Outputs of the products with blocks of 128 in every kind of wide tiles: rows further apart than they are wide, BF16 and FP32, sums on top
of what is there."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2511_05811_amd as moss
from gpu_util import dev, to_gpu
from test_gpu_block128 import check_product, operands, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,b_block,expected", [(512, 4096, 1024, 128, 64128), (900, 1288, 288, 1, 64128), (651, 4032, 1216, 128, 128128),
                                                    (2304, 1280, 288, 1, 128128), (2050, 4104, 288, 128, 128256), (2050, 4104, 288, 1, 128256),
                                                    (4000, 10008, 672, 128, 256256), (8000, 3208, 160, 1, 256256)])
def test_wider_outputs_and_sums(M, N, K, b_block, expected):
    tile = moss.load().moss_internal_gemm_block_tile
    tile.restype = C.c_int
    assert tile(*(C.c_int64(v) for v in (M, N, K, b_block, N + 8))) == expected
    a, a_s, b, b_s = operands(M, N, K, b_block, M + N + K)
    A, B = values(a, a_s, 1), values(b, b_s, b_block)
    d = [to_gpu(t) for t in (a, a_s, b, b_s)]
    for dtype in (torch.bfloat16, torch.float32):
        wide = torch.full((M, N + 8), 7.0, device=dev(), dtype=dtype)
        got = moss.gemm_fp8_block128(*d, out=wide[:, :N])
        check_product(got, A, B)
        assert bool((wide[:, N:] == 7.0).all())
    base = wide[:, :N].flip(1).clone()
    wide[:, :N] = base
    check_product(moss.gemm_fp8_block128(*d, out=wide[:, :N], accumulate=True), A, B, base.double().cpu().numpy())
    assert bool((wide[:, N:] == 7.0).all())
