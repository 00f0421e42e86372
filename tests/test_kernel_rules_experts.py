"""Which tiles a product with blocks of 128 or of grouped rows takes: the rules behind the entry points, asked on the host (256 compute
units are assumed where there is no GPU)."""
import ctypes as C

import pytest

import paper_2511_05811_amd as moss


@pytest.fixture(scope="module")
def L():
    lib = moss.load()
    if lib.moss_device_cu_count() not in (0, 256):
        pytest.skip("the sizes below are those of 256 compute units")
    return lib


def ask(fn, *args):
    fn.restype = C.c_int
    return fn(*(C.c_int64(a) for a in args))


@pytest.mark.parametrize("M,N,K,block,row", [(1, 4096, 4096, 32032, 32032), (600, 520, 128, 32032, 32032), (512, 4096, 1024, 64128, 64128),
                                             (651, 4032, 1216, 128128, 128128), (2050, 4104, 288, 128256, 128256), (8000, 3200, 160, 128256, 256256),
                                             (8192, 11008, 4096, 256256, 256256), (4553, 1792, 2048, 128256, 128256)])
def test_block_products_take_larger_tiles_the_larger_they_are(L, M, N, K, block, row):
    assert ask(L.moss_internal_gemm_block_tile, M, N, K, 128, N) == block
    assert ask(L.moss_internal_gemm_block_tile, M, N, K, 1, N) == row


@pytest.mark.parametrize("M,N,K,ld,tile", [(8192, 11008, 96, 11008, 64064), (8192, 11004, 4096, 11008, 64064), (8192, 11008, 4096, 11012, 64064),
                                           (8192, 1, 4096, 8, 32032), (16, 4096, 64, 4096, 32032), (512, 1001, 1024, 1001, 32032),
                                           (1152, 3968, 32, 3968, 64064), (256, 4100, 512, 4100, 64064), (1, 11001, 96, 11001, 32032)])
def test_block_products_that_the_wide_tiles_cannot_take(L, M, N, K, ld, tile):
    assert ask(L.moss_internal_gemm_block_tile, M, N, K, 128, ld) == ask(L.moss_internal_gemm_block_tile, M, N, K, 1, ld) == tile


@pytest.mark.parametrize("rows,N,K,groups,tile", [(4, 384, 2432, 64, 32032), (32, 11008, 4096, 8, 32032), (1003, 768, 1184, 32, 64128),
                                                  (1024, 2560, 1280, 8, 128128), (1500, 5888, 288, 40, 128256), (800, 2056, 512, 12, -128256),
                                                  (5003, 2056, 1152, 7, -256256), (16608, 11008, 4096, 8, -256256)])
def test_grouped_rows_take_larger_tiles_the_more_rows_a_group_has(L, rows, N, K, groups, tile):
    assert ask(L.moss_internal_gemm_grouped_tile, rows, N, K, groups, 1, N) == tile


@pytest.mark.parametrize("N,K,a_e,ld", [(11008, 4096, 0, 11008), (11004, 4096, 1, 11008), (11008, 96, 1, 11008), (11008, 4096, 1, 11012)])
def test_grouped_rows_that_only_the_small_tiles_take(L, N, K, a_e, ld):
    assert ask(L.moss_internal_gemm_grouped_tile, 16608, N, K, 8, a_e, ld) == 128128


def test_grouped_rows_in_large_tiles_only_with_whole_stages(L):
    assert ask(L.moss_internal_gemm_grouped_tile, 16608, 11008, 4096, 8, 1, 11008) < 0 < ask(L.moss_internal_gemm_grouped_tile, 16608, 11008, 4064, 8, 1, 11008)


@pytest.mark.parametrize("rows,M,N,groups,tile", [(1728, 392, 264, 32, 128128), (64, 4096, 4096, 2, 128128), (2016, 1000, 1001, 32, 128128),
                                                  (2048, 520, 1672, 8, 128256), (672, 1120, 1672, 6, 256256), (16608, 4096, 4096, 8, 256256)])
def test_weight_gradients_take_larger_tiles_the_more_there_are(L, rows, M, N, groups, tile):
    assert ask(L.moss_internal_gemm_grouped_dw_tile, rows, M, N, groups) == tile
