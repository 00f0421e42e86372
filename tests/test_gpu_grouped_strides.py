"""Strides and accumulation of the grouped products in every kind of tiles: weights of one stacked transposed matrix (dX) and weights apart
from each other, scales inside states, rows of the output further apart than they are wide, sums on top of what is there, rows of no
group ahead of, between and behind the groups' own.  Bars as in the tests of these products (plain 64-bit forms)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2511_05811_amd as moss
from gpu_util import dev, to_gpu
from test_gpu_grouped import Dw, Rows, SENTINEL

pytestmark = pytest.mark.gpu


def tile(name, *args):
    fn = getattr(moss.load(), name)
    fn.restype = C.c_int
    return fn(*(C.c_int64(a) for a in args))


# sizes of groups, N, K, tile (rows * 1000 + columns, the large-tile kernel's with a minus); behind them eleven rows of no group
KINDS = [([3, 0, 1, 70, 33], 264, 416, 32032), ([3, 0, 100, 1, 20, 61, 64, 2] * 4, 768, 1184, 64128), ([128, 0, 1, 256, 515, 0, 0], 2560, 1184, 128128),
         ([0, 1, 130, 37] * 10, 5888, 288, 128256), ([64, 0, 1, 127, 200, 8] * 2, 2056, 512, -128256),
         ([0, 1, 256, 2303, 700, 1733, 10], 2056, 1152, -256256)]


def problem(sizes, N, K, expected):
    offsets = 5 + np.concatenate([[0], np.cumsum(sizes)])
    p = Rows(offsets, N, K, R=int(offsets[-1]) + 6)
    assert tile("moss_internal_gemm_grouped_tile", p.R, N, K, p.G, 1, N + 8) == expected
    return p


def stacked(p):
    """The weights as the transposed codes of one matrix [G N x K] hold them: row n of all groups side by side"""
    t = to_gpu(np.ascontiguousarray(p.b.transpose(1, 0, 2)).reshape(p.N, p.G * p.K))
    return t.view(p.N, p.G, p.K).permute(1, 0, 2)


def apart(p):
    """Rows 16 bytes, groups two rows further apart than they are long; NaN codes in between"""
    t = torch.full((p.G, p.N + 2, p.K + 16), 0x7F, dtype=torch.uint8, device=dev())
    t[:, :p.N, :p.K] = to_gpu(p.b)
    return t[:, :p.N, :p.K]


def in_states(p):
    states = torch.full((p.G, 12), float("nan"), device=dev())
    states[:, 1] = to_gpu(p.b_s)
    return states[:, 1]


@pytest.mark.parametrize("weights", [stacked, apart])
@pytest.mark.parametrize("sizes,N,K,expected", KINDS)
def test_rows(sizes, N, K, expected, weights):
    p = problem(sizes, N, K, expected)
    args = p.args(b_q=weights(p), b_s=in_states(p))
    assert args["b_q"].stride(1) != K and args["b_s"].stride(0) == 12
    for dtype in (torch.bfloat16, torch.float32):
        wide = torch.full((p.R, N + 8), SENTINEL, device=dev(), dtype=dtype)
        held = wide[0, 0].item()
        p.check(moss.gemm_fp8_mx_grouped(out=wide[:, :N], **args), untouched=held)
        assert bool((wide[:, N:] == held).all())


@pytest.mark.parametrize("sizes,N,K,expected", KINDS)
def test_rows_that_accumulate(sizes, N, K, expected):
    p = problem(sizes, N, K, expected)
    typical = float(np.abs(p.A[p.offsets[-1] - 8:p.offsets[-1]] @ p.B[-1].T).mean()) + 1.0
    base = torch.randn((p.R, N), generator=torch.Generator().manual_seed(K)) * typical
    wide = torch.full((p.R, N + 8), SENTINEL, device=dev())
    wide[:, :N] = base.to(dev())
    got = moss.gemm_fp8_mx_grouped(out=wide[:, :N], accumulate=True, **p.args(b_q=stacked(p), b_s=in_states(p)))
    p.check(got, base=base.double().numpy())
    for rows in (slice(0, p.offsets[0]), slice(p.offsets[-1], p.R)):
        assert torch.equal(got[rows].cpu(), base[rows])
    assert bool((wide[:, N:] == SENTINEL).all())


@pytest.mark.parametrize("sizes,N,K,expected", KINDS)
def test_rows_of_a_group_that_takes_them_all(sizes, N, K, expected):
    """One group from the first row to the last, and groups that end with the array"""
    R = sum(sizes)
    for offsets in ([0] * (len(sizes) - 1) + [0, R], np.concatenate([[0], np.cumsum(sizes)])):
        p = Rows(offsets, N, K, R=R)
        p.check(moss.gemm_fp8_mx_grouped(**p.args(b_q=stacked(p), b_s=in_states(p))))


DW_KINDS = [([32, 0, 64, 160] * 7, 392, 264, 128128), ([0, 96, 1120, 32, 0, 512, 256, 32], 520, 1672, 128256), ([0, 32, 288, 0, 320, 32], 1120, 1672, 256256)]


@pytest.mark.parametrize("sizes,M,N,expected", DW_KINDS)
def test_weight_gradients_that_accumulate(sizes, M, N, expected):
    offsets = 32 + np.concatenate([[0], np.cumsum(sizes)])
    p = Dw(offsets, M, N, R=int(offsets[-1]) + 96)
    assert tile("moss_internal_gemm_grouped_dw_tile", p.R, M, N, p.G) == expected
    typical = float(np.abs(p.A[:, 32:96] @ p.B[:, 32:96].T).mean())
    base = torch.randn((p.G, M, N), generator=torch.Generator().manual_seed(N)) * typical
    around = torch.full((p.G + 2, M, N), SENTINEL, device=dev())
    around[1:-1] = base.to(dev())
    got = moss.gemm_fp8_mx_grouped_dw(out=around[1:-1], accumulate=True, **p.args())
    p.check(got, base=base.double().numpy())
    for g in range(p.G):
        if p.offsets[g] == p.offsets[g + 1]:
            assert torch.equal(got[g].cpu(), base[g])
    assert bool((around[0] == SENTINEL).all()) and bool((around[-1] == SENTINEL).all())
    p.check(moss.gemm_fp8_mx_grouped_dw(out_dtype=torch.bfloat16, **p.args()))
