"""A scale that is NaN or infinite shows in every output that it scales and in no other, whichever kind of tiles a product takes: a step
that has diverged looks the same at every size."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2511_05811_amd as moss
from gpu_util import dev, to_gpu
from test_gpu_block128 import operands

pytestmark = pytest.mark.gpu

# every kind of tiles: M, N, K, rows of b per scale, tile
KINDS = [(33, 96, 160, 128, 32032), (33, 96, 160, 1, 32032), (17, 520, 2016, 128, 32032), (17, 520, 2016, 1, 32032), (1100, 1288, 96, 128, 64064),
         (1100, 1288, 96, 1, 64064), (2048, 1001, 1056, 128, 64064), (2048, 1001, 1056, 1, 64064), (512, 4096, 1024, 128, 64128), (900, 1288, 288, 1, 64128),
         (651, 4032, 1216, 128, 128128), (2304, 1280, 288, 1, 128128), (2050, 4104, 288, 128, 128256), (2050, 4104, 288, 1, 128256),
         (4000, 10008, 672, 128, 256256), (8000, 3208, 160, 1, 256256)]


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("M,N,K,b_block,expected", KINDS)
def test_it_shows_in_what_it_scales(M, N, K, b_block, expected, value):
    tile = moss.load().moss_internal_gemm_block_tile
    tile.restype = C.c_int
    assert tile(*(C.c_int64(v) for v in (M, N, K, b_block, N))) == expected
    a, a_s, b, b_s = (to_gpu(t) for t in operands(M, N, K, b_block, M + N + K))
    want = moss.gemm_fp8_block128(a, a_s, b, b_s)
    assert bool(torch.isfinite(want).all())
    blocks = a_s.shape[1]
    # one block of K of every fifth row, each time another one
    rows = torch.arange(4, M, 5, device=dev())
    bad = a_s.clone()
    bad[rows, rows % blocks] = value
    got = moss.gemm_fp8_block128(a, bad, b, b_s)
    hit = torch.zeros(M, dtype=torch.bool, device=dev())
    hit[rows] = True
    assert not bool(torch.isfinite(got[hit]).any())
    assert torch.equal(got[~hit], want[~hit])
    # the same of every third scale of b
    of_b = torch.arange(0, b_s.shape[0], 3, device=dev())
    bad = b_s.clone()
    bad[of_b, of_b % blocks] = value
    got = moss.gemm_fp8_block128(a, a_s, b, bad)
    hit = torch.zeros(b_s.shape[0], dtype=torch.bool, device=dev())
    hit[of_b] = True
    hit = hit.repeat_interleave(b_block)[:N]
    assert not bool(torch.isfinite(got[:, hit]).any())
    assert torch.equal(got[:, ~hit], want[:, ~hit])


@pytest.mark.parametrize("M,N,K,b_block,expected", KINDS)
def test_a_block_of_zeros_shows_it_too(M, N, K, b_block, expected):
    """Codes that are all zeros times an infinite scale are no zeros; times a finite one, however large, they are."""
    a, a_s, b, b_s = operands(M, N, K, b_block, M + N + K)
    a[:, :128] = 0
    a_s[1::2, 0] = np.float32(3e38)
    d = [to_gpu(t) for t in (a, a_s, b, b_s)]
    want = moss.gemm_fp8_block128(*d)
    assert bool(torch.isfinite(want).all())
    d[1][2::5, 0] = float("inf")
    got = moss.gemm_fp8_block128(*d)
    hit = torch.zeros(M, dtype=torch.bool, device=dev())
    hit[2::5] = True
    assert not bool(torch.isfinite(got[hit]).any())
    assert torch.equal(got[~hit], want[~hit])
