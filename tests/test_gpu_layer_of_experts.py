"""A layer of experts, forward and backward, step by step: what each operator gave against the 64-bit form of its operands as they were,
the gradients of the tokens and of the routing weights among them, and the whole against the layer without FP8 within what the codes
can be off by."""
import numpy as np
import pytest
import torch

import paper_2511_05811_amd as moss
import reference64 as ref
from test_gpu_expert import Layer

pytestmark = pytest.mark.gpu

# (the second: more experts than some have tokens for, a width that ends inside a stage)
SIZES = [dict(T=130, k=2, E=4, hidden=256, ffn=416, seed=11), dict(T=61, k=3, E=16, hidden=160, ffn=320, seed=5)]


def f64(t):
    return t.double().cpu().numpy()


def rows_of(q):
    return ref.mx_values(q["q_row"], q["e_row"]) * q["s"].double().item()


def bf16_of(got, want, bar):
    """within `bar` ahead of one rounding to BF16 (half a step is 2^-8 of the value at most)"""
    err = np.abs(f64(got) - want)
    assert (err <= bar * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want) + 1e-37).all(), float((err / (bar + 2.0 ** -8 * np.abs(want) + 1e-37)).max())


@pytest.mark.parametrize("size", SIZES)
def test_every_step_from_what_it_was_given(size):
    L = Layer(**size)
    r = L.step()
    row_of, source, off = (r["plan"][n].cpu().numpy() for n in ("row_of", "source", "offsets"))
    x, d_out, w = f64(L.x), f64(L.d_out), f64(L.w)
    there = source >= 0
    assert sorted(source[there]) == list(range(L.T * L.k)) and (row_of.reshape(-1)[source[there]] == np.flatnonzero(there)).all()

    rows = f64(r["rows"])
    assert (rows[there] == x[source[there] // L.k]).all() and (rows[~there] == 0).all()

    # the quantizers that take their maximum from the step before, against those that look for it
    for name, q in (("rows", "q_rows"), ("h", "q_h"), ("d_y", "q_dy"), ("d_gate", "q_dg"), ("d_up", "q_du")):
        again = moss.quant_act_2level(r[name], moss.MOSS_Q_ROW | moss.MOSS_Q_COL)
        assert all(torch.equal(r[q][n], again[n]) for n in again), name

    # SwiGLU: FP32 inside, 2^-20 of each factor for its exponential, quotient and products
    g, u, d_h = f64(r["gate"]), f64(r["up"]), f64(r["d_h"])
    sig = 1 / (1 + np.exp(-g))
    bf16_of(r["h"], g * sig * u, 2.0 ** -20 * np.abs(g * u))
    bf16_of(r["d_up"], d_h * g * sig, 2.0 ** -20 * np.abs(d_h * g))
    bf16_of(r["d_gate"], d_h * u * sig * (1 + g * (1 - sig)), 2.0 ** -20 * np.abs(d_h * u) * (1 + np.abs(g)))

    # weighted sum and its gradients: k products in FP32; C products and their sum, each within C steps of 2^-24
    y = f64(r["y"])[row_of]                                                      # [T, k, C]
    bf16_of(r["out"], (w[..., None] * y).sum(1), 2.0 ** -22 * np.abs(w[..., None] * y).sum(1))
    d_y = f64(r["d_y"])
    want = w[..., None] * d_out[:, None]
    bf16_of(r["d_y"][torch.from_numpy(row_of.astype(np.int64).reshape(-1)).to(r["d_y"].device)], want.reshape(-1, L.hidden), 0 * want.reshape(-1, L.hidden))
    assert (d_y[~there] == 0).all()
    dots = d_out[:, None] * y
    assert (np.abs(f64(r["d_w"]) - dots.sum(-1)) <= L.hidden * 2.0 ** -24 * np.abs(dots).sum(-1)).all()

    # gradient of the experts' rows: two products, the second on top of the first in FP32, then one rounding
    dg, du = rows_of(r["q_dg"]), rows_of(r["q_du"])
    for e in range(L.E):
        part = slice(off[e], off[e + 1])
        if off[e] == off[e + 1]:
            continue
        both, bar = 0.0, 0.0
        for A, name in ((dg[part], "gate"), (du[part], "up")):
            B = ref.decode(L.weights[name][1][e]) * L.weights[name][2][e].double().item()
            product = A @ B.T
            both = both + product
            bar = bar + 3e-4 * np.outer(np.linalg.norm(A, axis=1), np.linalg.norm(B, axis=1)) + 2.0 ** -23 * np.abs(product)
        bf16_of(r["d_rows"][part], both, bar + 2.0 ** -23 * np.abs(both))
    assert (f64(r["d_rows"])[~there] == 0).all()

    # and of the tokens: the sum over their choices
    back = f64(r["d_rows"])[row_of]
    bf16_of(r["d_x"], back.sum(1), 2.0 ** -22 * np.abs(back).sum(1))


@pytest.mark.parametrize("size", SIZES)
def test_the_whole_without_fp8(size, monkeypatch):
    """Micro-scales rounded up, so that no code is clipped (rounded to the nearest, as is the default, they clip what lies up to sqrt(2) above
    448: single codes are off by 0.29 then, and all of a tensor by 0.07 to 0.11 in the 2-norm).  A code is within e = 2^-4 of its value
    (what lies below the normal range is within 2^-18 of the largest of its group, which no norm sees); the weights are the codes' own values on both sides.  Errors of independent codes add up by their squares, those that stem from
    the same codes (gate and up, of x) directly, SwiGLU's slopes are at most 1.1 of the relative error of each factor.  In units of e: gate 1, up 1,
    h 1.1 + 1 = 2.1, y behind its codes sqrt(2.1^2 + 1) = 2.3; d_h 1 (of d_y), d_gate sqrt(2.1^2 + 1) = 2.3, behind its codes 2.5, d_x 2.5, and the weight
    gradients with the codes of their other factor sqrt(2.5^2 + 1) = 2.7 at most.  2.7 * 2^-4 = 0.17, and 0.01 for the roundings to BF16.
    A term left out, of gate or of up, is an error of 0.5 to 0.7."""
    quantizer = moss.quant_act_2level_given_max
    monkeypatch.setattr(moss, "quant_act_2level_given_max", lambda t, word, flags: quantizer(t, word, flags | moss.MOSS_EXP_CEIL))
    L = Layer(**size)
    r = L.step()
    x = L.x.double().cpu().requires_grad_(True)
    w = L.w.double().cpu().requires_grad_(True)
    W = {n: (torch.from_numpy(ref.decode(L.weights[n][0])) * L.weights[n][2].double().cpu()[:, None, None]).requires_grad_(True) for n in L.weights}
    experts = L.experts.cpu().long()
    out = torch.zeros_like(x)
    for j in range(L.k):
        for e in range(L.E):
            t = (experts[:, j] == e).nonzero()[:, 0]
            g, u = x[t] @ W["gate"][e].T, x[t] @ W["up"][e].T
            out = out.index_add(0, t, w[t, j:j + 1] * ((torch.nn.functional.silu(g) * u) @ W["down"][e].T))
    out.backward(L.d_out.double().cpu())
    for name, want in (("out", out.detach()), ("d_x", x.grad), ("d_w", w.grad), ("dw_gate", W["gate"].grad), ("dw_up", W["up"].grad),
                       ("dw_down", W["down"].grad)):
        far = float((r[name].double().cpu() - want).norm() / want.norm())
        assert far <= 0.18, (name, far)
