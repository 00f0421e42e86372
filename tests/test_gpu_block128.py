"""GPU parity of the quantizers and products with an FP32 scale per block of 128 against plain 64-bit forms.

Quantizers: bit for bit (scales, codes).  Products: the bar of the block-scaled GEMM tests, |err| <= 3e-4 |a_row| |b_row| for the
matrix unit's sums (runs of 16 products in a window some 14 bits below the largest: 16 * 2^-14 of the largest of a run at the very most,
1e-3, and a third of that over a whole row), plus half a step of BF16, 2^-8 |y| at most."""
import numpy as np
import pytest
import torch

import moss_inputs as mi
import paper_2511_05811_amd as moss
import reference64 as ref
from gpu_util import assert_same_bits, bf16_to_gpu, dev, to_gpu, u8

pytestmark = pytest.mark.gpu
ROW, COL = moss.MOSS_Q_ROW, moss.MOSS_Q_COL


def bf16_bits(rows, cols, seed):
    return mi.heavy_tailed_activation(rows, cols, seed=seed)


def check_quant(bits, flags, pad=0):
    rows, cols = bits.shape
    wide = np.full((rows, cols + pad), 0x7F7F, np.uint16)           # (a large finite value where nothing may be read)
    wide[:, :cols] = bits
    got = moss.quant_block128(bf16_to_gpu(wide)[:, :cols], flags)
    torch.cuda.synchronize()
    x = mi.bf16_bits_to_f32(bits)
    for flag, q, s, y in ((ROW, "q_row", "s_row", x), (COL, "q_col", "s_col", np.ascontiguousarray(x.T))):
        if not flags & flag:
            assert got[q] is None and got[s] is None
            continue
        want_q, want_s = ref.quant_block(y, 1, 128)
        assert_same_bits(got[s].cpu().numpy(), want_s, s)
        assert_same_bits(u8(got[q]), want_q, q)


@pytest.mark.parametrize("rows,cols", [(1, 32), (17, 96), (3, 128), (257, 160), (1333, 1056), (40, 11008)])
@pytest.mark.parametrize("pad", [0, 24])
def test_row_groups(rows, cols, pad):
    check_quant(bf16_bits(rows, cols, rows + cols), ROW, pad)


@pytest.mark.parametrize("rows,cols", [(32, 32), (96, 160), (128, 128), (160, 416), (2016, 96), (64, 4128)])
@pytest.mark.parametrize("flags", [COL, ROW | COL])
@pytest.mark.parametrize("pad", [0, 64])
def test_column_groups(rows, cols, flags, pad):
    check_quant(bf16_bits(rows, cols, rows * 3 + cols), flags, pad)


@pytest.mark.parametrize("name", sorted(mi.adversarial_activations()))
def test_adversarial_activations(name):
    check_quant(mi.adversarial_activations()[name], ROW | COL)
    check_quant(mi.adversarial_activations()[name], ROW)


@pytest.mark.parametrize("rows,cols", [(1, 32), (100, 96), (128, 128), (160, 416), (512, 1056)])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("transpose", [False, True])
def test_weight_blocks(rows, cols, bf16, transpose):
    if transpose and rows % 32:
        pytest.skip("transposed codes come in multiples of 32 rows")
    w = mi.config4_weights(rows, cols, seed=rows)
    w[: rows // 2, :32] = 0.0
    w[:, cols // 2:] *= np.float32(2.0 ** -130)                      # subnormal blocks, reciprocals beyond FP32
    if bf16:
        w = mi.bf16_bits_to_f32(mi.f32_to_bf16_bits(w))
    t = to_gpu(w).to(torch.bfloat16) if bf16 else to_gpu(w)
    q, s, q_t, s_t = moss.quant_block128_weight(t, want_transpose=transpose)
    torch.cuda.synchronize()
    want_q, want_s = ref.quant_block(w, 128, 128)
    assert_same_bits(s.cpu().numpy(), want_s, "s")
    assert_same_bits(u8(q), want_q, "q")
    if transpose:
        assert_same_bits(s_t.cpu().numpy(), np.ascontiguousarray(want_s.T), "s_t")
        assert_same_bits(u8(q_t), np.ascontiguousarray(want_q.T), "q_t")
    else:
        assert q_t is None and s_t is None


def operands(M, N, K, b_block, seed):
    rng = np.random.default_rng(seed)
    def codes(n):
        c = rng.integers(0, 256, size=(n, K), dtype=np.uint8)
        c[(c & 0x7F) == 0x7F] = 0x38
        return c
    KB, NB = -(-K // 128), -(-N // b_block)
    a, b = codes(M), codes(N)
    a_s = np.exp(rng.uniform(-6, 2, (M, KB))).astype(np.float32)
    b_s = np.exp(rng.uniform(-6, 2, (NB, KB))).astype(np.float32)
    return a, a_s, b, b_s


def values(q, s, block):
    v = ref.decode(torch.from_numpy(q))
    return v * ref.spread(ref.spread(s.astype(np.float64), v.shape[0], 0, block), v.shape[1], 1)


def check_product(got, A, B, base=None):
    want = A @ B.T + (0 if base is None else base)
    bar = 3e-4 * np.outer(np.linalg.norm(A, axis=1), np.linalg.norm(B, axis=1)) + 1e-30
    if base is not None:
        bar = bar + 2.0 ** -23 * np.abs(want) + 2.0 ** -24 * np.abs(base)
    bf16 = got.dtype == torch.bfloat16
    err = np.abs(got.double().cpu().numpy() - want)
    if bf16:
        bar = bar * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    assert (err <= bar).all(), float((err / bar).max())


@pytest.mark.parametrize("M,N,K", [(1, 1, 32), (5, 3, 64), (16, 16, 128), (33, 95, 160), (17, 520, 2016), (200, 136, 96), (257, 129, 416),
                                   (130, 260, 1024), (64, 512, 4128), (1024, 1030, 640), (2050, 2042, 288), (1333, 4096, 544), (300, 700, 8224)])
@pytest.mark.parametrize("b_block", [1, 128])
def test_products_at_every_edge(M, N, K, b_block):
    a, a_s, b, b_s = operands(M, N, K, b_block, M + N + K)
    A, B = values(a, a_s, 1), values(b, b_s, b_block)
    d = [to_gpu(t) for t in (a, a_s, b, b_s)]
    check_product(moss.gemm_fp8_block128(*d), A, B)
    check_product(moss.gemm_fp8_block128(*d, out_dtype=torch.float32), A, B)
    base = torch.randn((M, N), generator=torch.Generator().manual_seed(K)).mul_(float(np.abs(A @ B.T).mean()))
    wide = torch.full((M, N + 8), 7.0, device=dev())
    wide[:, :N] = base.to(dev())
    out = moss.gemm_fp8_block128(*d, out=wide[:, :N], accumulate=True)
    check_product(out, A, B, base.double().numpy())
    assert bool((wide[:, N:] == 7.0).all())


# large tiles: whole and ragged K, edges inside a fragment, a tile of one row, more tiles than compute units
@pytest.mark.parametrize("M,N,K", [(600, 520, 128), (513, 1032, 160), (1, 300000, 256), (2050, 4104, 288), (300, 1000, 8224), (4353, 4096, 640), (2048, 4096, 1024)])
@pytest.mark.parametrize("b_block", [1, 128])
def test_products_in_large_tiles(M, N, K, b_block):
    a, a_s, b, b_s = operands(M, N, K, b_block, M + N + K)
    A, B = values(a, a_s, 1), values(b, b_s, b_block)
    d = [to_gpu(t) for t in (a, a_s, b, b_s)]
    check_product(moss.gemm_fp8_block128(*d), A, B)
    wide = torch.full((M, N + 8), 7.0, device=dev())
    out = moss.gemm_fp8_block128(*d, out=wide[:, :N])
    check_product(out, A, B)
    base = out.double().cpu().numpy()
    check_product(moss.gemm_fp8_block128(*d, out=wide[:, :N], accumulate=True), A, B, base)
    assert bool((wide[:, N:] == 7.0).all())


def test_blocks_of_zeros_and_scales_of_any_size():
    """A block that is all zeros adds nothing whatever its scale; scales from 2^-100 to 2^100 keep their products."""
    M, N, K = 70, 90, 640
    a, a_s, b, b_s = operands(M, N, K, 1, 5)
    a[:, 128:256] = 0
    a_s[:, 1] = np.float32(3e38)
    a_s[:, 2] *= np.float32(2.0 ** 100); b_s[:, 2] *= np.float32(2.0 ** -100)
    got = moss.gemm_fp8_block128(*(to_gpu(t) for t in (a, a_s, b, b_s)), out_dtype=torch.float32)
    check_product(got, values(a, a_s, 1), values(b, b_s, 1))


def test_linear_layer():
    """Forward and both gradients of a linear layer, as the recipe goes: each from what the quantizers made."""
    T, n_in, n_out = 160, 416, 288
    x, w = bf16_bits(T, n_in, 1), mi.config4_weights(n_out, n_in, seed=2)
    dy = mi.f32_to_bf16_bits(np.random.default_rng(3).standard_normal((T, n_out)).astype(np.float32) * np.float32(1e-3))
    qx, qdy = moss.quant_block128(bf16_to_gpu(x), ROW | COL), moss.quant_block128(bf16_to_gpu(dy), ROW | COL)
    wq, ws, wq_t, ws_t = moss.quant_block128_weight(to_gpu(w), want_transpose=True)
    v = lambda q, s, block=1: values(u8(q), s.cpu().numpy(), block)
    check_product(moss.gemm_fp8_block128(qx["q_row"], qx["s_row"], wq, ws), v(qx["q_row"], qx["s_row"]), v(wq, ws, 128))
    check_product(moss.gemm_fp8_block128(qdy["q_row"], qdy["s_row"], wq_t, ws_t), v(qdy["q_row"], qdy["s_row"]), v(wq_t, ws_t, 128))
    dw = moss.gemm_fp8_block128(qdy["q_col"], qdy["s_col"], qx["q_col"], qx["s_col"], out_dtype=torch.float32)
    check_product(dw, v(qdy["q_col"], qdy["s_col"]), v(qx["q_col"], qx["s_col"]))
    # and the whole against the layer without quantization.  A code is within half a step of its value, 2^-4 of it, or, below 2^-6,
    # within 2^-10 of its scale; independent errors of a row of products add up by their squares, so that 8 times the root of their
    # sum is never reached by chance
    X, W = mi.bf16_bits_to_f32(x).astype(np.float64), w.astype(np.float64)
    def err(t, s, q):
        return np.abs(t) * 2.0 ** -4 + 2.0 ** -10 * np.asarray(s, np.float64)
    ex = err(X, ref.spread(qx["s_row"].cpu().numpy(), n_in, 1), None)
    ew = err(W, ref.spread(ref.spread(ws.cpu().numpy(), n_out, 0), n_in, 1), None)
    y = moss.gemm_fp8_block128(qx["q_row"], qx["s_row"], wq, ws, out_dtype=torch.float32).double().cpu().numpy()
    bound = 8 * np.sqrt((ex ** 2) @ (W ** 2).T + (X ** 2) @ (ew ** 2).T + (ex ** 2) @ (ew ** 2).T)
    assert (np.abs(y - X @ W.T) <= bound).all()


def test_graph_replays_and_streams():
    M, N, K = 96, 256, 416
    a, a_s, b, b_s = (to_gpu(t) for t in operands(M, N, K, 128, 9))
    x = bf16_to_gpu(bf16_bits(M, N, 4))
    q = {k: torch.empty_like(v) for k, v in moss.quant_block128(x, ROW | COL).items()}
    out = torch.empty((M, N), dtype=torch.bfloat16, device=dev())
    want = [moss.gemm_fp8_block128(a, a_s, b, b_s), moss.quant_block128(x, ROW | COL)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        moss.gemm_fp8_block128(a, a_s, b, b_s, out=out)
        moss.quant_block128(x, ROW | COL, out=q)
    for _ in range(3):
        out.zero_()
        for t in q.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and all(torch.equal(q[k], want[1][k]) for k in q)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got += [moss.gemm_fp8_block128(a, a_s, b, b_s) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[0]) for g in got)


def test_refusals():
    x = torch.zeros((64, 96), dtype=torch.bfloat16, device=dev())
    with pytest.raises(moss.MossError):
        moss.quant_block128(x[:33], COL)
    with pytest.raises(moss.MossError):
        moss.quant_block128(x[:, :40], ROW)
    with pytest.raises(moss.MossError):
        moss.quant_block128(x, 0)
    with pytest.raises(AssertionError):
        moss.quant_block128(x.float())
    with pytest.raises(AssertionError):
        moss.quant_block128(x.t())
    with pytest.raises(AssertionError):
        moss.quant_block128(x, out=dict(q_row=torch.empty((64, 64), dtype=torch.uint8, device=dev())))
    with pytest.raises(moss.MossError):
        moss.quant_block128_weight(torch.zeros((40, 32), device=dev()), want_transpose=True)
    a, a_s, b, b_s = (to_gpu(t) for t in operands(32, 64, 256, 128, 1))
    with pytest.raises(AssertionError):
        moss.gemm_fp8_block128(a, a_s[:, :1], b, b_s)
    with pytest.raises(AssertionError):
        moss.gemm_fp8_block128(a, a_s, b, torch.zeros((3, 2), device=dev()))
    with pytest.raises(moss.MossError):
        moss.gemm_fp8_block128(a, a_s, b, b_s, accumulate=True)      # into BF16
    with pytest.raises(AssertionError):
        moss.gemm_fp8_block128(a.cpu(), a_s, b, b_s)


@pytest.mark.parametrize("flags", [ROW, COL, ROW | COL])
def test_every_magnitude_as_the_largest_of_a_group(flags):
    """All finite BF16 magnitudes, subnormals and zero among them, each the largest of a group of rows and of one of columns."""
    top = np.arange(0x7F80, dtype=np.uint16)                         # a group each: [255 x 128] of them
    bits = np.zeros((255 * 128, 128), np.uint16)
    small = np.random.default_rng(1).random((255 * 128, 128)) * mi.bf16_bits_to_f32(top.reshape(-1, 1))
    bits[:] = np.minimum(mi.f32_to_bf16_bits(small.astype(np.float32)) & 0x7FFF, top[:, None])
    bits[np.arange(bits.shape[0]), np.arange(bits.shape[0]) % 128] = top
    bits[1::2] ^= 0x8000
    check_quant(bits, flags & ROW or flags)
    if flags & COL:
        check_quant(np.ascontiguousarray(bits.T), flags)
