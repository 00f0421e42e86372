"""GPU parity of the grouped products of a layer of experts against plain 64-bit forms.  The bar is that of the block-scaled GEMM
tests: 3e-4 |a_row| |b_row| for the matrix unit's sums, half a step of BF16 (2^-8 |y| at most) where the output is BF16, half a step of
FP32 for what is accumulated into."""
import numpy as np
import pytest
import torch

import paper_2511_05811_amd as moss
import reference64 as ref
from gpu_util import dev, to_gpu

pytestmark = pytest.mark.gpu
SENTINEL = 12345.0


def codes(rng, shape):
    c = rng.integers(0, 256, size=shape, dtype=np.uint8)
    c[(c & 0x7F) == 0x7F] = 0x38
    return c


def exps(rng, shape):
    return rng.integers(100, 128, size=shape, dtype=np.uint8)


def within(got, want, bar, base=None):
    if base is not None:
        want = want + base
        bar = bar + 2.0 ** -23 * np.abs(want) + 2.0 ** -24 * np.abs(base)
    if got.dtype == torch.bfloat16:
        bar = bar * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= bar + 1e-30).all(), float((err / (bar + 1e-30)).max())


def norms(A, B):
    return 3e-4 * np.outer(np.linalg.norm(A, axis=1), np.linalg.norm(B, axis=1))


class Rows:
    """Operands of a grouped product and what it gives."""

    def __init__(self, offsets, N, K, R=None, seed=0, unit=False, one_scale=False):
        rng = np.random.default_rng(seed + N + K)
        self.offsets, self.G = np.asarray(offsets, np.int32), len(offsets) - 1
        self.R = int(self.offsets[-1] if R is None else R)
        self.N, self.K = N, K
        self.a, self.b = codes(rng, (self.R, K)), codes(rng, (self.G, N, K))
        self.ae = None if unit else exps(rng, (self.R, K // 32))
        self.a_s = np.array([0.37], np.float32)
        self.b_s = rng.uniform(0.5, 2.0, 1 if one_scale else self.G).astype(np.float32)
        t = lambda x: None if x is None else torch.from_numpy(x)
        self.A = ref.mx_values(t(self.a), t(self.ae)) * np.float64(self.a_s[0])
        self.B = [ref.decode(t(self.b[g])) * np.float64(self.b_s[g if self.b_s.size > 1 else 0]) for g in range(self.G)]

    def args(self, **other):
        d = dict(a_q=to_gpu(self.a), a_e=None if self.ae is None else to_gpu(self.ae), a_s=to_gpu(self.a_s), b_q=to_gpu(self.b), b_s=to_gpu(self.b_s),
                 offsets=to_gpu(self.offsets))
        d.update(other)
        return d

    def check(self, got, base=None, untouched=None):
        """base: what was accumulated into; untouched: what rows of no group hold"""
        there = np.zeros(self.R, bool)
        for g in range(self.G):
            rows = slice(self.offsets[g], self.offsets[g + 1])
            there[rows] = True
            if rows.start < rows.stop:
                within(got[rows], self.A[rows] @ self.B[g].T, norms(self.A[rows], self.B[g]), None if base is None else base[rows])
        if untouched is not None:
            assert bool((got[torch.from_numpy(~there).to(dev())] == untouched).all())


GROUPS = {
    "one": [0, 77], "one_row": [0, 1], "single_rows": [0, 1, 2, 3, 4], "empty_ones": [0, 0, 40, 40, 41, 41], "ragged": [0, 3, 131, 260, 261, 500],
    "starts_late": [16, 40, 90], "many": list(range(0, 131)), "aligned": [0, 128, 128, 384, 640], "skewed": [0, 2, 1200, 1203],
}


@pytest.mark.parametrize("name", sorted(GROUPS))
@pytest.mark.parametrize("N,K", [(1, 32), (40, 96), (129, 160), (264, 1024), (96, 4128)])
def test_rows_of_every_layout(name, N, K):
    offsets = GROUPS[name]
    p = Rows(offsets, N, K, R=offsets[-1] + 5, unit=name == "many" and K == 32, one_scale=name == "aligned")
    for dtype in (torch.bfloat16, torch.float32):
        wide = torch.full((p.R, N + 8), SENTINEL, device=dev(), dtype=dtype)
        held = wide[0, 0].item()
        got = moss.gemm_fp8_mx_grouped(**p.args(out=wide[:, :N]))
        p.check(got, untouched=held)
        assert bool((wide[:, N:] == held).all())
    base = torch.randn((p.R, N), generator=torch.Generator().manual_seed(K)) * float(np.abs(p.A @ p.B[0].T).mean())
    got = moss.gemm_fp8_mx_grouped(**p.args(out=base.to(dev()), accumulate=True))
    p.check(got, base=base.double().numpy())


# rows per expert from few to many, each of which gets another tile
@pytest.mark.parametrize("per,N,K", [(2, 2048, 512), (40, 1024, 1024), (90, 1152, 640), (300, 1000, 1056), (700, 2304, 768), (1500, 1536, 512)])
def test_sizes_in_earnest(per, N, K):
    rng = np.random.default_rng(per)
    sizes = rng.integers(0, 2 * per + 1, 6)
    p = Rows(np.concatenate([[0], np.cumsum(sizes)]), N, K, R=int(sizes.sum()) + 3, seed=per)
    got = moss.gemm_fp8_mx_grouped(**p.args(out=torch.full((p.R, N), SENTINEL, device=dev())))
    p.check(got, untouched=SENTINEL)
    p.check(moss.gemm_fp8_mx_grouped(**p.args()))


def test_weights_of_one_stacked_matrix_and_scales_inside_states():
    """dX: the transposed codes of one matrix [E N x K], a view per expert, and the scales where the optimizer keeps them."""
    E, N, K = 5, 96, 160
    p = Rows([0, 30, 30, 200, 201, 333], N, K)
    stacked = to_gpu(np.ascontiguousarray(p.b.transpose(1, 0, 2)).reshape(N, E * K))
    view = stacked.view(N, E, K).permute(1, 0, 2)
    states = torch.zeros((E, 48), dtype=torch.uint8, device=dev())
    scales = states.view(torch.float32)[:, 1]
    scales.copy_(to_gpu(p.b_s))
    p.check(moss.gemm_fp8_mx_grouped(**p.args(b_q=view, b_s=scales)))


def test_a_weight_shared_by_all_groups_and_views_of_groups():
    p = Rows([0, 10, 90], 72, 256)
    shared = to_gpu(p.b)[:1].expand(2, -1, -1)
    p.B = [p.B[0], p.B[0] / np.float64(p.b_s[0]) * np.float64(p.b_s[1])]
    p.check(moss.gemm_fp8_mx_grouped(**p.args(b_q=shared)))


def test_offsets_that_leave_the_rows_stay_inside():
    """Offsets are not known on the host; beyond the rows they count as their end, below zero as their start."""
    p = Rows([0, 64, 128], 64, 256)
    wide = torch.full((p.R + 64, p.N), SENTINEL, device=dev())
    got = moss.gemm_fp8_mx_grouped(**p.args(out=wide[:p.R], offsets=to_gpu(np.array([-50, 64, 1 << 30], np.int32))))
    p.check(got)
    assert bool((wide[p.R:] == SENTINEL).all())
    got = moss.gemm_fp8_mx_grouped(**p.args(out=wide, a_q=torch.cat([to_gpu(p.a), to_gpu(p.a)[:64]]), a_e=torch.cat([to_gpu(p.ae), to_gpu(p.ae)[:64]]),
                                            offsets=to_gpu(np.array([-9, -5, -1], np.int32))))
    assert bool((got[p.R:] == SENTINEL).all())


class Dw:
    def __init__(self, offsets, M, N, R=None, seed=0):
        rng = np.random.default_rng(seed + M + N)
        self.offsets, self.G = np.asarray(offsets, np.int32), len(offsets) - 1
        self.R, self.M, self.N = int(self.offsets[-1] if R is None else R), M, N
        self.a, self.b = codes(rng, (M, self.R)), codes(rng, (N, self.R))
        self.ae, self.be = exps(rng, (M, self.R // 32)), exps(rng, (N, self.R // 32))
        self.a_s, self.b_s = np.array([0.3], np.float32), np.array([1.9], np.float32)
        t = torch.from_numpy
        self.A, self.B = ref.mx_values(t(self.a), t(self.ae)) * np.float64(self.a_s[0]), ref.mx_values(t(self.b), t(self.be)) * np.float64(self.b_s[0])

    def args(self, **other):
        d = {k: to_gpu(v) for k, v in dict(a_q=self.a, a_e=self.ae, a_s=self.a_s, b_q=self.b, b_e=self.be, b_s=self.b_s, offsets=self.offsets).items()}
        d.update(other)
        return d

    def check(self, got, base=None):
        for g in range(self.G):
            part = slice(self.offsets[g], self.offsets[g + 1])
            A, B = self.A[:, part], self.B[:, part]
            within(got[g], A @ B.T, norms(A, B), None if base is None else base[g])


DW_GROUPS = {
    "one": [0, 96], "shortest": [0, 32], "empty_ones": [0, 0, 64, 64, 96, 96], "ragged": [0, 32, 160, 416, 448, 1184], "starts_late": [32, 64, 256],
    "many": list(range(0, 32 * 70, 32)), "aligned": [0, 128, 128, 512, 640], "long": [0, 64, 6240, 6272],
}


@pytest.mark.parametrize("name", sorted(DW_GROUPS))
@pytest.mark.parametrize("M,N", [(1, 1), (40, 33), (160, 264)])
def test_weight_gradients_of_every_layout(name, M, N):
    offsets = DW_GROUPS[name]
    p = Dw(offsets, M, N, R=offsets[-1] + 64)
    p.check(moss.gemm_fp8_mx_grouped_dw(**p.args()))
    p.check(moss.gemm_fp8_mx_grouped_dw(**p.args(out_dtype=torch.bfloat16)))
    base = torch.randn((p.G, M, N), generator=torch.Generator().manual_seed(N)) * float(np.abs(p.A @ p.B.T).mean())
    got = moss.gemm_fp8_mx_grouped_dw(**p.args(out=base.to(dev()), accumulate=True))
    p.check(got, base=base.double().numpy())


def test_weight_gradients_in_earnest():
    p = Dw([0, 992, 992, 1504, 4128], 520, 1096)
    p.check(moss.gemm_fp8_mx_grouped_dw(**p.args()))
    p = Dw([0, 256, 768, 1024], 1024, 512)
    p.check(moss.gemm_fp8_mx_grouped_dw(**p.args(out_dtype=torch.bfloat16)))


def test_graph_replays_with_other_offsets():
    """The offsets are read when the kernel runs: a replay takes what they hold then."""
    p, q = Rows([0, 40, 100, 160], 200, 256), Rows([0, 100, 100, 160], 200, 256)
    d = Dw([0, 32, 96, 160], 72, 104)
    args, dargs = p.args(), d.args()
    out, dw = torch.empty((160, 200), dtype=torch.bfloat16, device=dev()), torch.empty((3, 72, 104), device=dev())
    moss.gemm_fp8_mx_grouped(out=out, **args), moss.gemm_fp8_mx_grouped_dw(out=dw, **dargs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moss.gemm_fp8_mx_grouped(out=out, **args)
        moss.gemm_fp8_mx_grouped_dw(out=dw, **dargs)
    for offsets in (p.offsets, q.offsets, p.offsets):
        args["offsets"].copy_(torch.from_numpy(offsets))
        out.zero_(), dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        p.offsets = offsets
        p.check(out)
        d.check(dw)


def test_refusals():
    p = Rows([0, 32, 64], 64, 128)
    bad = [dict(offsets=to_gpu(p.offsets).long()), dict(offsets=to_gpu(p.offsets)[:2]), dict(a_s=to_gpu(p.b_s)), dict(b_s=torch.ones(3, device=dev())),
           dict(a_q=to_gpu(p.a)[:, :96]), dict(b_q=to_gpu(p.b).transpose(1, 2)), dict(out=torch.empty((63, 64), device=dev()))]
    for other in bad:
        with pytest.raises(AssertionError):
            moss.gemm_fp8_mx_grouped(**p.args(**other))
    wide = torch.zeros((2, 64, 136), dtype=torch.uint8, device=dev())
    for other in (dict(accumulate=True), dict(b_q=wide[:, :, :128]), dict(out=torch.empty((64, 64), device=dev(), dtype=torch.float16))):
        with pytest.raises(moss.MossError):
            moss.gemm_fp8_mx_grouped(**p.args(**other))
    d = Dw([0, 32, 64], 64, 96)
    for other in (dict(offsets=to_gpu(d.offsets).long()), dict(a_e=to_gpu(d.ae)[:, :1]), dict(b_e=None), dict(out=torch.empty((2, 64, 64), device=dev()))):
        with pytest.raises((AssertionError, AttributeError)):
            moss.gemm_fp8_mx_grouped_dw(**d.args(**other))
    with pytest.raises(moss.MossError):
        moss.gemm_fp8_mx_grouped_dw(**d.args(out_dtype=torch.bfloat16, accumulate=True))
