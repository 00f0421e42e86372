"""Every tile that a product with blocks of 128 or of grouped rows can take, at sizes that end inside it: against plain 64-bit forms
(bars as in the tests of these products), run to run, on two streams at once and in replayed graphs."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2511_05811_amd as moss
from gpu_util import dev, to_gpu
from test_gpu_block128 import check_product, operands, values
from test_gpu_grouped import Dw, Rows, SENTINEL

pytestmark = pytest.mark.gpu


def tile(name, *args):
    fn = getattr(moss.load(), name)
    fn.restype = C.c_int
    return fn(*(C.c_int64(a) for a in args))


def again(call, want):
    """The same bits from two streams at once and from every replay of a graph."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got += [call(torch.full_like(want, SENTINEL)) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    out = torch.full_like(want, SENTINEL)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for _ in range(3):
        out.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("M,N,K,b_block,expected", [(33, 96, 160, 128, 32032), (512, 4096, 1024, 128, 64128), (900, 1288, 288, 1, 64128),
                                                    (651, 4032, 1216, 128, 128128), (2304, 1280, 288, 1, 128128),
                                                    (2050, 4104, 288, 128, 128256), (2050, 4104, 288, 1, 128256),
                                                    (4000, 10008, 672, 128, 256256), (8000, 3208, 160, 1, 256256)])
def test_block_products(M, N, K, b_block, expected):
    assert tile("moss_internal_gemm_block_tile", M, N, K, b_block, N) == expected
    a, a_s, b, b_s = operands(M, N, K, b_block, M + N + K)
    d = [to_gpu(t) for t in (a, a_s, b, b_s)]
    got = moss.gemm_fp8_block128(*d)
    check_product(got, values(a, a_s, 1), values(b, b_s, b_block))
    again(lambda out: moss.gemm_fp8_block128(*d, out=out), got)


@pytest.mark.parametrize("sizes,N,K,expected", [([3, 0, 1, 70, 33], 264, 416, 32032), ([3, 0, 100, 1, 20, 61, 64, 2] * 4, 768, 1184, 64128),
                                                ([128, 0, 1, 256, 515, 0, 0], 2560, 1184, 128128),
                                                ([0, 1, 130, 37] * 10, 5888, 288, 128256), ([64, 0, 1, 127, 200, 8] * 2, 2056, 512, -128256),
                                                ([0, 1, 256, 2303, 700, 1733, 10], 2056, 1152, -256256)])
def test_grouped_rows(sizes, N, K, expected):
    p = Rows(np.concatenate([[0], np.cumsum(sizes)]), N, K)
    assert tile("moss_internal_gemm_grouped_tile", p.R, N, K, p.G, 1, N) == expected
    args = p.args()
    got = moss.gemm_fp8_mx_grouped(**args)
    p.check(got)
    again(lambda out: moss.gemm_fp8_mx_grouped(out=out, **args), got)


@pytest.mark.parametrize("sizes,M,N,expected", [([32, 0, 64, 160] * 7, 392, 264, 128128), ([0, 96, 1120, 32, 0, 512, 256, 32], 520, 1672, 128256),
                                                ([0, 32, 288, 0, 320, 32], 1120, 1672, 256256)])
def test_grouped_weight_gradients(sizes, M, N, expected):
    p = Dw(np.concatenate([[0], np.cumsum(sizes)]), M, N)
    assert tile("moss_internal_gemm_grouped_dw_tile", p.R, M, N, p.G) == expected
    args = p.args()
    got = moss.gemm_fp8_mx_grouped_dw(out_dtype=torch.float32, **args)
    p.check(got)
    again(lambda out: moss.gemm_fp8_mx_grouped_dw(out=out, **args), got)


# 128 x 128, 128 x 256 and 256 x 256 outputs at a time; groups that end inside a stage, before and behind rows of no group
@pytest.mark.parametrize("sizes,M,N", [([96, 160, 0, 64], 392, 264), ([96, 1120, 32, 0, 512, 224], 520, 1672), ([32, 288, 320, 32], 1120, 1672)])
def test_rows_of_other_groups_may_hold_anything(sizes, M, N):
    """What lies outside a group, NaN codes and exponents among it, is no part of its gradient."""
    p = Dw(64 + np.concatenate([[0], np.cumsum(sizes)]), M, N, R=64 + sum(sizes) + 96)
    args = p.args()
    want = moss.gemm_fp8_mx_grouped_dw(out_dtype=torch.float32, **args)
    p.check(want)
    for g in range(p.G):
        first, end = (int(v) for v in p.offsets[g:g + 2])
        poisoned = dict(args)
        for name, unit, value in (("a_q", 1, 0x7F), ("b_q", 1, 0xFF), ("a_e", 32, 255), ("b_e", 32, 255)):
            t = args[name].clone()
            t[:, :first // unit] = value
            t[:, end // unit:] = value
            poisoned[name] = t
        assert torch.equal(moss.gemm_fp8_mx_grouped_dw(out_dtype=torch.float32, **poisoned)[g], want[g])


@pytest.mark.parametrize("M,N,K,b_block", [(512, 4096, 1024, 128), (900, 1288, 288, 1), (651, 4032, 1216, 128), (2304, 1280, 288, 1), (2050, 4104, 288, 128),
                                           (2050, 4104, 288, 1), (4000, 10008, 672, 128), (8000, 3208, 160, 1)])
def test_a_scale_that_is_not_finite_stays_in_its_rows(M, N, K, b_block):
    a, a_s, b, b_s = (to_gpu(t) for t in operands(M, N, K, b_block, M + N + K))
    want = moss.gemm_fp8_block128(a, a_s, b, b_s)
    rows, blocks = torch.arange(M, device=dev()) % 5 == 4, torch.arange(b_s.shape[0], device=dev()) % 7 == 3
    columns = blocks.repeat_interleave(b_block)[:N]
    a_s[rows], b_s[blocks] = float("inf"), float("inf")
    got = moss.gemm_fp8_block128(a, a_s, b, b_s)
    assert torch.equal(got[~rows][:, ~columns], want[~rows][:, ~columns])


@pytest.mark.parametrize("M,N,K", [(1152, 1000, 32), (1100, 1288, 96), (257, 4100, 512), (2048, 1001, 1056)])
@pytest.mark.parametrize("b_block", [1, 128])
def test_block_products_of_odd_sizes(M, N, K, b_block):
    """64 x 64 outputs at a time, a fragment per wave"""
    assert tile("moss_internal_gemm_block_tile", M, N, K, b_block, N) == 64064
    a, a_s, b, b_s = operands(M, N, K, b_block, M + N + K)
    d = [to_gpu(t) for t in (a, a_s, b, b_s)]
    A, B = values(a, a_s, 1), values(b, b_s, b_block)
    got = moss.gemm_fp8_block128(*d)
    check_product(got, A, B)
    again(lambda out: moss.gemm_fp8_block128(*d, out=out), got)
    wide = torch.full((M, N + 3), 7.0, device=dev())
    out = moss.gemm_fp8_block128(*d, out=wide[:, :N])
    check_product(out, A, B)
    base = out.double().cpu().numpy()
    check_product(moss.gemm_fp8_block128(*d, out=wide[:, :N], accumulate=True), A, B, base)
    assert bool((wide[:, N:] == 7.0).all())


# sizes that go to every kind of tiles; offsets that decrease, lie outside and are no multiples of 32
@pytest.mark.parametrize("R,N,K,G,expected", [(107, 264, 416, 5, 32032), (1004, 768, 1184, 32, 64128), (900, 2560, 1184, 7, 128128), (1680, 5888, 288, 40, 128256),
                                              (800, 2056, 512, 12, -128256), (5003, 2056, 1152, 7, -256256)])
def test_wrong_offsets_write_nothing_outside(R, N, K, G, expected):
    assert tile("moss_internal_gemm_grouped_tile", R, N, K, G, 1, N) == expected
    p = Rows([0] * G + [R], N, K)
    wide = torch.full((R + 128, N), SENTINEL, device=dev(), dtype=torch.bfloat16)
    held = wide[0, 0].item()
    rng = np.random.default_rng(R)
    for offsets in (rng.integers(-2 ** 31, 2 ** 31, G + 1), rng.integers(-50, R + 50, G + 1), np.linspace(R, 0, G + 1)):
        moss.gemm_fp8_mx_grouped(**p.args(out=wide[64:64 + R], offsets=to_gpu(offsets.astype(np.int32))))
        torch.cuda.synchronize()
        assert bool((wide[:64] == held).all()) and bool((wide[64 + R:] == held).all())


@pytest.mark.parametrize("R,M,N,G,expected", [(1792, 392, 264, 28, 128128), (2048, 520, 1672, 8, 128256), (672, 1120, 1672, 6, 256256)])
def test_wrong_offsets_of_weight_gradients_write_nothing_outside(R, M, N, G, expected):
    assert tile("moss_internal_gemm_grouped_dw_tile", R, M, N, G) == expected
    p = Dw([0] * G + [R], M, N)
    wide = torch.full((G + 2, M, N), SENTINEL, device=dev())
    rng = np.random.default_rng(R)
    for offsets in (rng.integers(-2 ** 31, 2 ** 31, G + 1), rng.integers(-50, R + 50, G + 1), np.linspace(R, 0, G + 1)):
        moss.gemm_fp8_mx_grouped_dw(**p.args(out=wide[1:1 + G], offsets=to_gpu(offsets.astype(np.int32))))
        torch.cuda.synchronize()
        assert bool((wide[0] == SENTINEL).all()) and bool((wide[-1] == SENTINEL).all())
        assert bool((wide[1:1 + G] != SENTINEL).all())
