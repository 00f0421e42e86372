"""Operands and outputs that reach beyond 2^32 bytes, and as many groups as there can be: parts of the results against plain forms of
those parts, or against the same call on a small copy of them."""
import numpy as np
import pytest
import torch

import paper_2511_05811_amd as moss
import reference64 as ref
from gpu_util import dev, to_gpu
from test_gpu_block128 import check_product, operands, values
from test_gpu_grouped import Dw, Rows, norms, within

pytestmark = pytest.mark.gpu


def random_codes(*shape):
    c = torch.randint(0, 256, shape, dtype=torch.uint8, device=dev(), generator=torch.Generator(dev()).manual_seed(sum(shape)))
    return c.masked_fill_((c & 0x7F) == 0x7F, 0x38)


def pieces(n):
    """A few rows at both ends and around the middle."""
    return [slice(0, 3), slice(n // 2 - 1, n // 2 + 2), slice(n - 3, n)]


def test_quantizer():
    rows, cols = 540672, 4096
    x = torch.randn((rows, cols), dtype=torch.bfloat16, device=dev(), generator=torch.Generator(dev()).manual_seed(1))
    assert x.numel() * 2 > 1 << 32
    both, alone = moss.quant_block128(x, moss.MOSS_Q_ROW | moss.MOSS_Q_COL), moss.quant_block128(x)
    for first in (0, 270336, rows - 128):
        part = moss.quant_block128(x[first:first + 128], moss.MOSS_Q_ROW | moss.MOSS_Q_COL)
        here = slice(first, first + 128)
        for got in (both, alone):
            assert torch.equal(got["q_row"][here], part["q_row"]) and torch.equal(got["s_row"][here], part["s_row"])
        assert torch.equal(both["q_col"][:, here], part["q_col"]) and torch.equal(both["s_col"][:, first // 128], part["s_col"][:, 0])


@pytest.mark.parametrize("b_block", [1, 128])
def test_block_product(b_block):
    """rows of a beyond 2^32 bytes, then an output beyond them"""
    for M, N, K in ((1056777, 72, 4096), (33000, 66000, 160)):
        _, a_s, _, b_s = operands(M, N, 32, b_block, 3)
        blocks = (K + 127) // 128
        a, b = random_codes(M, K), random_codes(N, K)
        a_s, b_s = to_gpu(np.repeat(a_s, blocks, 1)), to_gpu(np.repeat(b_s, blocks, 1))
        got = moss.gemm_fp8_block128(a, a_s, b, b_s)
        assert max(a.numel(), got.numel() * 2) > 1 << 32
        B = values(b.cpu().numpy(), b_s.cpu().numpy(), b_block)
        for rows in pieces(M):
            check_product(got[rows], values(a[rows].cpu().numpy(), a_s[rows].cpu().numpy(), 1), B)
        del got, a, b


def test_grouped_rows():
    for R, N, K, G in ((1056777, 72, 4096, 3), (66000, 33000, 512, 3)):
        a, a_e, b = random_codes(R, K), torch.randint(100, 128, (R, K // 32), dtype=torch.uint8, device=dev()), random_codes(G, N, K)
        a_s, b_s = torch.full((1,), 0.5, device=dev()), torch.tensor([1.0, 2.0, 0.25], device=dev())
        offsets = torch.tensor([0, R // 2, R // 2 + 1, R], dtype=torch.int32, device=dev())
        got = moss.gemm_fp8_mx_grouped(a, a_e, a_s, b, b_s, offsets)
        assert max(a.numel(), got.numel() * 2) > 1 << 32
        B = [ref.decode(b[g].cpu()) * float(b_s[g]) for g in range(G)]
        for rows in pieces(R):
            for r in range(rows.start, rows.stop):
                g = int((offsets[1:] <= r).sum())
                A = ref.mx_values(a[r:r + 1].cpu(), a_e[r:r + 1].cpu()) * 0.5
                within(got[r:r + 1], A @ B[g].T, norms(A, B[g]))
        del got, a, b


def test_grouped_weight_gradients():
    """an output beyond 2^32 bytes, then operands beyond them"""
    for M, N, R, offsets in ((8192, 8200, 2048, list(range(0, 2048 + 1, 64))), (4104, 136, 1056768, [0, 528384, 528416, 1056768])):
        G = len(offsets) - 1
        a, b = random_codes(M, R), random_codes(N, R)
        a_e, b_e = (torch.randint(100, 128, (n, R // 32), dtype=torch.uint8, device=dev()) for n in (M, N))
        one, off = torch.ones(1, device=dev()), torch.tensor(offsets, dtype=torch.int32, device=dev())
        got = moss.gemm_fp8_mx_grouped_dw(a, a_e, one, b, b_e, one, off, out_dtype=torch.bfloat16)
        assert max(a.numel(), got.numel() * 2) > 1 << 32
        for g in (0, 1, G - 1):
            part = slice(offsets[g], offsets[g + 1])
            e = slice(part.start // 32, part.stop // 32)
            B = ref.mx_values(b[:, part].cpu().contiguous(), b_e[:, e].cpu().contiguous())
            for rows in pieces(M):
                A = ref.mx_values(a[rows, part].cpu().contiguous(), a_e[rows, e].cpu().contiguous())
                within(got[g, rows], A @ B.T, norms(A, B))
        del got, a, b


def test_rows_of_experts():
    T, k, E, cols = 270400, 2, 8, 4096
    generator = torch.Generator(dev()).manual_seed(5)
    x = torch.randn((T, cols), dtype=torch.bfloat16, device=dev(), generator=generator)
    experts = torch.rand((T, E), device=dev(), generator=generator).topk(k, 1)[1].int()
    weights = torch.rand((T, k), device=dev(), generator=generator)
    plan = moss.expert_plan(experts, E)
    y, _ = moss.expert_dispatch_bf16(x, plan)
    assert y.numel() * 2 > 1 << 32
    out = moss.expert_combine_bf16(y, plan, weights)
    d_y, d_w, _ = moss.expert_combine_bf16_backward(x, y, plan, weights)
    kept = y.clone()
    in_place, d_w2, _ = moss.expert_combine_bf16_backward(x, kept, plan, weights, d_y=kept)
    assert torch.equal(in_place, d_y) and torch.equal(d_w2, d_w)
    for t in pieces(T):
        for j in range(k):
            rows = plan["row_of"][t, j].long()
            assert torch.equal(plan["source"][rows], (torch.arange(t.start, t.stop, device=dev()) * k + j).int())
            assert torch.equal(y[rows], x[t])
            assert torch.equal(d_y[rows], (weights[t, j, None] * x[t].float()).bfloat16())
        want = sum(weights[t, j, None].double() * x[t].double() for j in range(k))
        assert bool(((out[t].double() - want).abs() <= want.abs() * 2.0 ** -8 + 2.0 ** -22 * x[t].double().abs()).all())
        dot = (x[t].double() ** 2).sum(1, keepdim=True).expand(-1, k)          # (cols products in FP32: each step rounds at most 2^-24)
        assert bool(((d_w[t].double() - dot).abs() <= dot * cols * 2.0 ** -24).all())


def test_as_many_groups_as_there_can_be():
    for N, K in ((72, 96), (1544, 256), (264, 512)):
        p = Rows(np.arange(0, 2 * 1024 + 1, 2), N, K)
        p.check(moss.gemm_fp8_mx_grouped(**p.args()))
    p = Dw(np.arange(0, 32 * 1024 + 1, 32), 72, 136)
    p.check(moss.gemm_fp8_mx_grouped_dw(**p.args()))
