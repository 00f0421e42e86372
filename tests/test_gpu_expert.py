"""The rows' way to the experts and back against plain forms: the plan assignment by assignment, copies bit for bit, sums and gradients in
64 bits, and all operators of a layer of experts together."""
import numpy as np
import pytest
import torch

import paper_2511_05811_amd as moss
import reference64 as ref
from gpu_util import dev, to_gpu

pytestmark = pytest.mark.gpu


def route(T, k, E, seed, distinct=True, drop=0.0):
    rng = np.random.default_rng(seed)
    if distinct:
        e = np.argsort(rng.random((T, E)), axis=1)[:, :k]
    else:
        e = np.minimum(rng.geometric(0.3, (T, k)) - 1, E - 1)
    e = e.astype(np.int32)
    e[rng.random((T, k)) < drop] = rng.choice([-1, E, 2 ** 31 - 1, -2 ** 31])
    return e


def bf16(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16)


def same_plan(plan, experts, E, multiple):
    row_of, source, offsets = ref.plan(experts, E, multiple, plan["source"].numel())
    assert plan["offsets"].tolist() == offsets
    assert plan["source"].tolist() == source
    assert plan["row_of"].flatten().tolist() == row_of


@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 4, 4), (1, 2, 64), (5, 3, 1024), (63, 1, 2), (64, 2, 8), (65, 2, 7), (333, 8, 129), (2048, 2, 64),
                                   (5000, 4, 16)])
@pytest.mark.parametrize("multiple", [1, 32, 128])
def test_plan(T, k, E, multiple):
    for distinct, drop in ((True, 0.0), (False, 0.1), (False, 1.0)):
        if distinct and k > E:
            continue
        experts = route(T, k, E, T + k, distinct, drop)
        plan = moss.expert_plan(to_gpu(experts), E, multiple=multiple)
        assert plan["source"].numel() == moss.expert_rows(T, k, E, multiple)
        same_plan(plan, experts, E, multiple)


@pytest.mark.parametrize("T,k,E", [(9001, 2, 64), (70000, 2, 256), (200000, 1, 1024), (40000, 8, 3)])
def test_plan_of_many_tokens(T, k, E):
    experts = route(T, k, E, 3, distinct=False, drop=0.05)
    same_plan(moss.expert_plan(to_gpu(experts), E, multiple=32), experts, E, 32)


def test_plan_with_more_rows_than_needed():
    experts = route(40, 2, 8, 1)
    plan = moss.expert_plan(to_gpu(experts), 8, multiple=32, rows=1024)
    same_plan(plan, experts, 8, 32)


def make(T, k, E, C, multiple=32, drop=0.0, distinct=True, seed=0):
    experts = route(T, k, E, seed, distinct, drop)
    plan = moss.expert_plan(to_gpu(experts), E, multiple=multiple)
    row_of, source, _ = ref.plan(experts, E, multiple, plan["source"].numel())
    return plan, np.array(row_of).reshape(T, k), np.array(source)


def padded(t, pad):
    """t as a view of a wider tensor whose other columns are large"""
    if not pad:
        return t.to(dev())
    wide = torch.full((t.shape[0], t.shape[1] + pad), 1e30, dtype=t.dtype, device=dev())
    wide[:, :t.shape[1]] = t.to(dev())
    return wide[:, :t.shape[1]]


CASES = [(1, 1, 1, 8, 1), (1, 2, 64, 4096, 32), (7, 3, 5, 24, 32), (64, 2, 8, 256, 32), (65, 1, 3, 520, 1), (130, 4, 16, 1032, 128), (257, 2, 8, 2056, 32),
         (33, 9, 12, 4104, 32), (1000, 2, 64, 768, 32)]


@pytest.mark.parametrize("T,k,E,C,multiple", CASES)
@pytest.mark.parametrize("pad", [0, 8])
@pytest.mark.parametrize("drop", [0.0, 0.3, 1.0])
def test_dispatch_combine_and_gradients(T, k, E, C, multiple, pad, drop):
    plan, row_of, source = make(T, k, E, C, multiple, drop, distinct=drop == 0.0, seed=T)
    R = len(source)
    x, y, d_out = bf16((T, C), 1), bf16((R, C), 2), bf16((T, C), 3, 1e-3)
    w = torch.rand((T, k), generator=torch.Generator().manual_seed(4)) + 0.1
    there, at = row_of >= 0, np.maximum(row_of, 0)
    filled, tok = source >= 0, np.maximum(source, 0) // k
    X, Y, D, W = (t.double().numpy() for t in (x, y, d_out, w))

    rows, top = moss.expert_dispatch_bf16(padded(x, pad), plan)
    want = torch.where(torch.from_numpy(filled)[:, None], x[torch.from_numpy(tok)], torch.zeros((), dtype=torch.bfloat16))
    assert torch.equal(rows.cpu(), want)
    assert top.to(torch.int16).view(torch.bfloat16).item() == want.abs().max().item()

    # rows without an assignment are not read: whatever they hold does not show
    held = y.clone()
    held[torch.from_numpy(~filled)] = float("nan")
    back = np.where(there[..., None], Y[at], 0.0)
    for weights in (w, None):
        out = moss.expert_combine_bf16(padded(held, pad), plan, None if weights is None else weights.to(dev()))
        terms = back * (W[..., None] if weights is not None else 1.0)
        want = terms.sum(1)
        # k products and k - 1 sums in FP32, each half a step of at most the sum of magnitudes, then half a step of BF16
        bar = 2 * k * 2.0 ** -24 * np.abs(terms).sum(1)
        bar = bar * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
        assert (np.abs(out.double().cpu().numpy() - want) <= bar).all()

    d_y, d_w, d_top = moss.expert_combine_bf16_backward(padded(d_out, pad), padded(y, pad), plan, w.to(dev()))
    want = torch.where(torch.from_numpy(filled)[:, None], (w.flatten()[torch.from_numpy(np.maximum(source, 0))][:, None] * d_out.float()[torch.from_numpy(tok)]),
                       torch.zeros(())).to(torch.bfloat16)         # (one product in 32 bits, one rounding)
    assert torch.equal(d_y.cpu(), want)
    assert d_top.to(torch.int16).view(torch.bfloat16).item() == want.abs().max().item()
    terms = D[:, None] * back
    # products of BF16 are exact in FP32; a sum of C of them in any order is off by at most C - 1 half steps of the sum of magnitudes
    assert (np.abs(d_w.double().cpu().numpy() - terms.sum(2)) <= C * 2.0 ** -24 * np.abs(terms).sum(2)).all()
    assert bool((d_w.cpu()[torch.from_numpy(~there)] == 0).all())


def test_gradients_against_differences():
    """combine is linear in y and in the weights, dispatch in x: differences of the 64-bit forms are the gradients."""
    T, k, E, C = 6, 2, 4, 16
    plan, row_of, source = make(T, k, E, C, 1, seed=5)
    y, d_out = bf16((len(source), C), 1), bf16((T, C), 2)
    w = torch.rand((T, k), generator=torch.Generator().manual_seed(3))
    loss = lambda y, w: float(((y[row_of] * w[..., None]).sum(1) * d_out.double().numpy()).sum())
    Y, W = y.double().numpy(), w.double().numpy()
    d_y, d_w, _ = moss.expert_combine_bf16_backward(d_out.to(dev()), y.to(dev()), plan, w.to(dev()))
    h = 2.0 ** -10
    for got, arg in ((d_y, 0), (d_w, 1)):
        got = got.double().cpu().numpy()
        for at in np.ndindex(got.shape):
            a, b = [Y.copy(), W.copy()], [Y.copy(), W.copy()]
            a[arg][at] += h
            b[arg][at] -= h
            slope = (loss(*a) - loss(*b)) / (2 * h)
            # (the slope of a linear function is exact up to rounding in 64 bits)
            assert abs(slope - got[at]) <= 2.0 ** -8 * abs(slope) + 1e-5
    x = bf16((T, C), 4)
    d_rows = bf16((len(source), C), 5)
    d_x = moss.expert_combine_bf16(d_rows.to(dev()), plan).double().cpu().numpy()
    X = x.double().numpy()
    way = lambda x: float((x[source // k] * d_rows.double().numpy()).sum())
    for at in np.ndindex(X.shape):
        a, b = X.copy(), X.copy()
        a[at] += h
        b[at] -= h
        slope = (way(a) - way(b)) / (2 * h)
        assert abs(slope - d_x[at]) <= 2.0 ** -8 * abs(slope) + 1e-5


def test_entries_outside_their_range_count_as_dropped():
    T, k, E, C = 20, 2, 4, 64
    plan, row_of, source = make(T, k, E, C, 32, seed=7)
    R = len(source)
    plan["row_of"][3, 1] = R
    plan["row_of"][4, 0] = -7
    for t, j in ((3, 1), (4, 0)):
        plan["source"][row_of[t, j]] = T * k + 5
        row_of[t, j] = -1
    x, y = bf16((T, C), 1), bf16((R, C), 2)
    rows, _ = moss.expert_dispatch_bf16(x.to(dev()), plan)
    want = torch.zeros((R, C), dtype=torch.bfloat16)
    for t in range(T):
        for j in range(k):
            if row_of[t, j] >= 0:
                want[row_of[t, j]] = x[t]
    assert torch.equal(rows.cpu(), want)
    out = moss.expert_combine_bf16(y.to(dev()), plan)
    back = np.where((row_of >= 0)[..., None], y.double().numpy()[np.maximum(row_of, 0)], 0.0)
    want = back.sum(1)
    assert (np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * np.abs(back).sum(1)).all()
    w = torch.ones((T, k), device=dev())
    _, d_w, _ = moss.expert_combine_bf16_backward(x.to(dev()), y.to(dev()), plan, w)
    assert d_w[3, 1].item() == 0.0 and d_w[4, 0].item() == 0.0


class Layer:
    """A layer of experts on the library: forward and backward of tokens through gate, up and down projections with SwiGLU in between,
    every product in FP8, every intermediate result kept for the comparison."""

    def __init__(self, T, k, E, hidden, ffn, seed):
        gen = torch.Generator().manual_seed(seed)
        rnd = lambda *s, scale=1.0: torch.randn(s, generator=gen).mul_(scale).to(dev())
        self.T, self.k, self.E, self.hidden, self.ffn = T, k, E, hidden, ffn
        self.x, self.d_out = rnd(T, hidden).to(torch.bfloat16), rnd(T, hidden, scale=1e-3).to(torch.bfloat16)
        self.experts = to_gpu(route(T, k, E, seed))
        self.w = torch.rand((T, k), generator=gen).to(dev()) + 0.1
        self.weights = {}
        for name, n, kk in (("gate", ffn, hidden), ("up", ffn, hidden), ("down", hidden, ffn)):
            states = torch.zeros((E, 48), dtype=torch.uint8, device=dev())
            q, q_t = torch.empty((E, n, kk), dtype=torch.uint8, device=dev()), torch.empty((E, kk, n), dtype=torch.uint8, device=dev())
            for e in range(E):
                moss.weight_autoscale_init(rnd(n, kk, scale=0.05), states[e], wq=q[e], wq_t=q_t[e])
            self.weights[name] = (q, q_t, states.view(torch.float32)[:, 1])

    def step(self):
        both = moss.MOSS_Q_ROW | moss.MOSS_Q_COL
        r = {}
        plan = r["plan"] = moss.expert_plan(self.experts, self.E)
        off = plan["offsets"]
        fwd = lambda q, name: moss.gemm_fp8_mx_grouped(q["q_row"], q["e_row"], q["s"], self.weights[name][0], self.weights[name][2], off)
        bwd = lambda q, name, **kw: moss.gemm_fp8_mx_grouped(q["q_row"], q["e_row"], q["s"], self.weights[name][1], self.weights[name][2], off, **kw)
        dw = lambda a, b: moss.gemm_fp8_mx_grouped_dw(a["q_col"], a["e_col"], a["s"], b["q_col"], b["e_col"], b["s"], off)
        quant = lambda t, word: moss.quant_act_2level_given_max(t, word, both)
        r["rows"], word = moss.expert_dispatch_bf16(self.x, plan)
        r["q_rows"] = quant(r["rows"], word)
        r["gate"], r["up"] = fwd(r["q_rows"], "gate"), fwd(r["q_rows"], "up")
        r["h"], word = moss.swiglu_bf16(r["gate"], r["up"])
        r["q_h"] = quant(r["h"], word)
        r["y"] = fwd(r["q_h"], "down")
        r["out"] = moss.expert_combine_bf16(r["y"], plan, self.w)
        r["d_y"], r["d_w"], word = moss.expert_combine_bf16_backward(self.d_out, r["y"], plan, self.w)
        r["q_dy"] = quant(r["d_y"], word)
        r["d_h"], r["dw_down"] = bwd(r["q_dy"], "down"), dw(r["q_dy"], r["q_h"])
        r["d_gate"], r["d_up"], wg, wu = moss.swiglu_bf16_backward(r["gate"], r["up"], r["d_h"])
        r["q_dg"], r["q_du"] = quant(r["d_gate"], wg), quant(r["d_up"], wu)
        r["dw_gate"], r["dw_up"] = dw(r["q_dg"], r["q_rows"]), dw(r["q_du"], r["q_rows"])
        d_rows = bwd(r["q_dg"], "gate", out_dtype=torch.float32)
        r["d_rows"] = bwd(r["q_du"], "up", out=d_rows, accumulate=True).to(torch.bfloat16)
        r["d_x"] = moss.expert_combine_bf16(r["d_rows"], plan)
        return r


def test_a_layer_of_experts_together():
    """Every product of the layer against the 64-bit product of the operands that it was given, by the bars of each; the whole against
    the layer without FP8: codes are within 2^-4 of their values (or 2^-9 of the largest of their group of 32 below the normal range), so the
    relative error of a product of sums of independent errors stays below 4 * sqrt(2) * 2^-4 = 0.36 in the 2-norm; two layers
    one behind the other and SwiGLU's slope (at most 1.1 of each factor) below three times that."""
    L = Layer(T=130, k=2, E=4, hidden=256, ffn=416, seed=11)
    r = L.step()
    off = r["plan"]["offsets"].tolist()
    assert off[-1] == r["rows"].shape[0]
    val = lambda q, side: ref.mx_values(q["q_" + side], q["e_" + side]) * q["s"].double().item()

    def rows_product(got, q, name, which):
        A = val(q, "row")
        for e in range(L.E):
            B = ref.decode(L.weights[name][which][e]) * L.weights[name][2][e].double().item()
            part = slice(off[e], off[e + 1])
            want = A[part] @ B.T
            bar = 3e-4 * np.outer(np.linalg.norm(A[part], axis=1), np.linalg.norm(B, axis=1)) + 2.0 ** -8 * np.abs(want) + 1e-30
            assert (np.abs(got[part].double().cpu().numpy() - want) <= bar * (1 + 2.0 ** -8)).all(), name
    rows_product(r["gate"], r["q_rows"], "gate", 0)
    rows_product(r["up"], r["q_rows"], "up", 0)
    rows_product(r["y"], r["q_h"], "down", 0)
    rows_product(r["d_h"], r["q_dy"], "down", 1)
    for got, a, b in (("dw_down", "q_dy", "q_h"), ("dw_gate", "q_dg", "q_rows"), ("dw_up", "q_du", "q_rows")):
        A, B = val(r[a], "col"), val(r[b], "col")
        for e in range(L.E):
            part = slice(off[e], off[e + 1])
            bar = 3e-4 * np.outer(np.linalg.norm(A[:, part], axis=1), np.linalg.norm(B[:, part], axis=1)) + 1e-30
            assert (np.abs(r[got][e].double().cpu().numpy() - A[:, part] @ B[:, part].T) <= bar).all(), got

    # without FP8
    x = L.x.double().cpu().requires_grad_(True)
    w = L.w.double().cpu().requires_grad_(True)
    W = {n: (torch.from_numpy(ref.decode(L.weights[n][0])) * L.weights[n][2].double().cpu()[:, None, None]).requires_grad_(True) for n in L.weights}
    out = torch.zeros_like(x)
    experts = L.experts.cpu().long()
    for j in range(L.k):
        e = experts[:, j]
        g = torch.einsum("tc,tfc->tf", x, W["gate"][e])
        u = torch.einsum("tc,tfc->tf", x, W["up"][e])
        out = out + w[:, j:j + 1] * torch.einsum("tf,tcf->tc", torch.nn.functional.silu(g) * u, W["down"][e])
    out.backward(L.d_out.double().cpu())
    far = lambda got, want: float((got.double().cpu() - want).norm() / want.norm())
    for name, got, want in (("out", r["out"], out.detach()), ("d_x", r["d_x"], x.grad), ("d_w", r["d_w"], w.grad), ("dw_gate", r["dw_gate"], W["gate"].grad),
                            ("dw_up", r["dw_up"], W["up"].grad), ("dw_down", r["dw_down"], W["down"].grad)):
        print(f"[layer of experts] {name}: {far(got, want):.3e}", flush=True)
        assert far(got, want) <= 3 * 0.36, name


def test_a_layer_of_experts_in_a_graph():
    L = Layer(T=70, k=2, E=8, hidden=128, ffn=256, seed=3)
    names = ("out", "d_x", "d_w", "dw_gate", "dw_up", "dw_down", "rows", "d_y")
    want = {n: t.clone() for n, t in L.step().items() if n in names}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = L.step()
    other = to_gpu(route(70, 2, 8, 99))
    first = L.experts.clone()
    for k in range(4):
        L.experts.copy_(other if k == 1 else first)
        for n in names:
            r[n].zero_()
        graph.replay()
        torch.cuda.synchronize()
        expect = want
        if k == 1:
            expect = {n: t.clone() for n, t in L.step().items() if n in names}
        for n in names:
            assert torch.equal(r[n], expect[n]), (k, n)


def test_refusals():
    experts = to_gpu(route(8, 2, 4, 0))
    with pytest.raises(AssertionError):
        moss.expert_plan(experts.long(), 4)
    for bad in (dict(n_experts=0), dict(n_experts=4, multiple=0), dict(n_experts=1025), dict(n_experts=4, multiple=4097), dict(n_experts=4, rows=32),
                dict(n_experts=4, rows=1000)):
        with pytest.raises(moss.MossError):
            moss.expert_plan(experts, **bad)
    plan = moss.expert_plan(experts, 4)
    R = plan["source"].numel()
    x, y = torch.zeros((8, 64), dtype=torch.bfloat16, device=dev()), torch.zeros((R, 64), dtype=torch.bfloat16, device=dev())
    w = torch.ones((8, 2), device=dev())
    for call in (lambda: moss.expert_dispatch_bf16(x[:7], plan), lambda: moss.expert_dispatch_bf16(x.float(), plan), lambda: moss.expert_combine_bf16(y[1:], plan),
                 lambda: moss.expert_combine_bf16(y, plan, w.half()), lambda: moss.expert_combine_bf16_backward(x, y[:, :32], plan, w),
                 lambda: moss.expert_combine_bf16_backward(x, y, plan, w[:, :1])):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(moss.MossError):
        moss.expert_dispatch_bf16(x[:, :12], plan)
