"""FP8 products with a scale per block of 128, and the products of a layer of experts, as cases that can be timed and compared.

Five operators:

  block_quant   the quantizers of the recipe with one FP32 scale per 128 elements: activations and gradients (`weight` False) in
                groups along the columns (the inner dimension of Y and dX) and / or along the rows (that of dW, stored transposed),
                weights in blocks of 128 x 128, with or without the transposed codes that dX needs.
  block_gemm    the product of such operands: forward and dX (a scale per row of a and per block of the weight), or dW (`dw`: a
                scale per row of both).
  grouped       the products of E experts with their rows, as many as routing gave each: forward, or dX (`view`: the weights are
                taken from the transposed codes of one stacked matrix).
  grouped_dw    the weight gradients of E experts: sums over each expert's rows.
  experts       the rows' way to the experts and back, as a training step goes through it: plan, dispatch, weighted combination,
                and the gradients of both.

The layer sizes are those of a LLaMA-7B block (hidden 4096, FFN 11008), of its small test version (hidden 256, FFN 512) and of the
single-linear configuration (1024 -> 1024).

`own` False computes the plain form: elementary torch operations in 32 bits, rounded once.
"""
import math

import torch

own = False

DEV = "cuda:0"
F32, F64, BF16, FP8 = torch.float32, torch.float64, torch.bfloat16, torch.float8_e4m3fn
FLT_MAX = torch.finfo(torch.float32).max


def listed():
    return [
        # the input of a projection at 8192 tokens, for forward and weight gradient at once
        dict(name="quant_both", kind="block_quant", weight=False, rows=8192, cols=4096, pad=0, row=True, col=True),
        # an FFN weight after an optimizer step, from FP32 masters
        dict(name="quant_weight", kind="block_quant", weight=True, rows=11008, cols=4096, bf16=False, transpose=True),
        # generation for a handful of sequences: every weight is read for few rows
        dict(name="gemm_generate", kind="block_gemm", M=17, N=11008, K=4096, dw=False),
        # the gate projection of the benchmark's batch
        dict(name="gemm_ffn", kind="block_gemm", M=8192, N=11008, K=4096, dw=False),
        # weight gradient of the output projection over 2016 tokens (the sum ends inside a block)
        dict(name="gemm_dw", kind="block_gemm", M=4096, N=4096, K=2016, dw=True),
        # experts of the small block: latency and launches count
        dict(name="grouped_small", kind="grouped", tokens=64, k=2, E=8, N=512, K=256, multiple=32, view=False),
        # generation: 16 sequences, two experts each, no padding between the experts' rows
        dict(name="grouped_generate", kind="grouped", tokens=16, k=2, E=8, N=11008, K=4096, multiple=1, view=False),
        # a training batch of 8192 tokens through the experts' up projection (the largest)
        dict(name="grouped_train", kind="grouped", tokens=8192, k=2, E=8, N=11008, K=4096, multiple=32, view=False),
        # weight gradients of many narrow experts over a short batch: sums of a few dozen rows
        dict(name="grouped_dw_short", kind="grouped_dw", tokens=512, k=2, E=32, M=1024, N=1024, multiple=32),
        # weight gradients of 8 experts over the benchmark's batch
        dict(name="grouped_dw_train", kind="grouped_dw", tokens=8192, k=2, E=8, M=4096, N=4096, multiple=32),
        # the small block's tokens to 8 experts and back
        dict(name="experts_small", kind="experts", tokens=64, k=2, E=8, cols=256, multiple=32),
        # 8192 tokens of hidden size 4096 to 64 experts and back
        dict(name="experts_train", kind="experts", tokens=8192, k=2, E=64, cols=4096, multiple=32),
    ]


def _between(rng, lo, hi, step):
    """a multiple of `step` between lo and hi, spread over the logarithm"""
    v = math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["block_quant", "block_gemm", "block_gemm", "grouped", "grouped", "grouped_dw", "experts"])
    # layer widths are nearly always multiples of 128; the library takes multiples of 32
    step = 128 if rng.random() < 0.75 else 32
    most = 16384 * 11008 * 4096
    if kind == "block_quant":
        if rng.random() < 0.4:
            return dict(kind=kind, weight=True, rows=_between(rng, 256, 11008, 32), cols=_between(rng, 256, 4096, 32),
                        bf16=rng.random() < 0.5, transpose=rng.random() < 0.7)
        row = rng.random() < 0.8
        col = not row or rng.random() < 0.6
        rows = _between(rng, 32, 16384, 32) if col else _between(rng, 1, 16384, 1)
        return dict(kind=kind, weight=False, rows=rows, cols=_between(rng, 256, 11008, 32), pad=64 if rng.random() < 0.2 else 0, row=row, col=col)
    if kind == "block_gemm":
        if rng.random() < 0.4:
            M, N = _between(rng, 256, 11008, step), _between(rng, 256, 4096, step)
            return dict(kind=kind, M=M, N=N, K=_between(rng, 32, 8192, 32), dw=True)
        N, K = _between(rng, 256, 11008, step), _between(rng, 256, 4096, step)
        return dict(kind=kind, M=_between(rng, 1, 16384, 1), N=N, K=K, dw=False)
    E = rng.choice([4, 8, 16, 32, 64])
    k = rng.choice([1, 2, 2, 4])
    if kind == "experts":
        cols = _between(rng, 256, 8192, 8)
        tokens = _between(rng, 1, min(8192, 8192 * 2 * 4096 // (k * cols)), 1)
        return dict(kind=kind, tokens=tokens, k=k, E=E, cols=cols, multiple=rng.choice([1, 32, 32, 128]))
    tokens = _between(rng, 1, 16384 // k, 1)
    N = _between(rng, 256, 11008, step)
    K = _between(rng, 256, max(256, min(4096, 8 * 11008 * 4096 // (E * N))), step)
    if kind == "grouped":
        return dict(kind=kind, tokens=tokens, k=k, E=E, N=N, K=K, multiple=rng.choice([1, 32, 32, 128]), view=rng.random() < 0.3)
    return dict(kind=kind, tokens=tokens, k=k, E=E, M=N, N=min(K, 4096), multiple=rng.choice([32, 32, 128]))


# ---- inputs

def _normal(gen, shape, scale=1.0):
    return torch.randn(shape, generator=gen, device=DEV, dtype=F32).mul_(scale)


def _activation(gen, rows, cols, scale=1.0):
    """N(0, 1) with 8 channels x 20: the outlier channels that activations of a trained model show"""
    x = _normal(gen, (rows, cols), scale)
    x[:, torch.randperm(cols, generator=gen, device=DEV)[:8]] *= 20.0
    return x


def _blocks(n):
    return (n + 127) // 128


def _scale_of(amax):
    """amax / 448 rounded to 32 bits, 1 for a group of zeros"""
    return torch.where(amax > 0, (amax.double() / 448.0).float(), 1.0)


def _codes(x, s):
    """E4M3 values of x (32 bits) under the scales s, spread to its shape: x * fl(1 / s), rounded to nearest even, at most 448"""
    inv = (1.0 / s.double()).clamp(max=FLT_MAX).float()
    return (x * inv).clamp_(-448.0, 448.0).to(FP8)


def _in_groups(x):
    """[rows x cols] in groups of 128 along the columns: values, one scale per group"""
    rows, cols = x.shape
    n = _blocks(cols)
    wide = torch.nn.functional.pad(x, (0, n * 128 - cols)) if cols % 128 else x
    s = _scale_of(wide.view(rows, n, 128).abs().amax(2))
    return _codes(x, s.repeat_interleave(128, 1)[:, :cols]), s


def _in_blocks(w):
    """[rows x cols] in blocks of 128 x 128: values, one scale per block"""
    rows, cols = w.shape
    r, c = _blocks(rows), _blocks(cols)
    wide = torch.nn.functional.pad(w, (0, c * 128 - cols, 0, r * 128 - rows))
    s = _scale_of(wide.view(r, 128, c, 128).abs().amax(3).amax(1))
    return _codes(w, s.repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :cols]), s


def _two_level(x):
    """[rows x cols] with one FP32 scale and a power of two per 32 columns: codes, exponent bytes, scale"""
    amax = x.abs().amax()
    s = _scale_of(amax)
    g = x.view(x.shape[0], -1, 32).abs().amax(2)
    e = torch.where(g > 0, torch.log2(g.double() / amax.double()).round().clamp(-127, 0), -127.0).float()
    q = _codes(x * torch.exp2(-e.clamp(min=-100.0)).repeat_interleave(32, 1), s)
    return q.view(torch.uint8), (e + 127).to(torch.uint8), s.view(1)


def _per_tensor(w):
    s = _scale_of(w.abs().amax())
    return _codes(w, s).view(torch.uint8), s


def _routing(case, gen):
    """k different experts for every token, some more popular than others"""
    T, E = case["tokens"], case["E"]
    liking = _normal(gen, (T, E)) + _normal(gen, (1, E), 0.5)
    weight, experts = torch.topk(torch.softmax(liking, 1), case["k"], 1)
    return experts.to(torch.int32), weight / weight.sum(1, keepdim=True)


def _capacity(case):
    """rows that the experts' assignments take at most, each expert's filled up to the multiple"""
    n, m = case["tokens"] * case["k"], case["multiple"]
    return (n + min(case["E"], n) * (m - 1)) // m * m


def _plan(case, experts):
    """Where every assignment (token, choice) goes: its row, the assignment of every row (-1: padding), where the experts' rows
    start.  Assignments of an expert in order, the experts one after the other, each filled up to the multiple, the last to the end."""
    E, m, R = case["E"], case["multiple"], _capacity(case)
    flat = experts.reshape(-1).long()
    there = (flat >= 0) & (flat < E)
    key = torch.where(there, flat, E)
    order = torch.sort(key, stable=True)[1]
    counts = (key[:, None] == torch.arange(E, device=DEV)).sum(0)
    padded = (counts + m - 1) // m * m
    start, before = padded.cumsum(0) - padded, counts.cumsum(0) - counts
    row = torch.empty_like(flat)
    of = key[order].clamp(max=E - 1)
    row[order] = start[of] + torch.arange(flat.numel(), device=DEV) - before[of]
    row = torch.where(there, row, -1)
    source = torch.full((R + 1,), -1, device=DEV, dtype=torch.int64)
    source[torch.where(there, row, R)] = torch.arange(flat.numel(), device=DEV)
    offsets = torch.cat([start, torch.full((1,), R, device=DEV)])
    return row.view(experts.shape).int(), source[:R].int(), offsets.int()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind = case["kind"]
    st = dict(case=case)
    if kind == "block_quant":
        if case["weight"]:
            st["x"] = _normal(gen, (case["rows"], case["cols"]), 0.02).to(BF16 if case["bf16"] else F32)
        else:
            wide = _activation(gen, case["rows"], case["cols"] + case["pad"]).to(BF16)
            st["x"] = wide[:, :case["cols"]]
    elif kind == "block_gemm":
        M, N, K = case["M"], case["N"], case["K"]
        if case["dw"]:
            a, b = _normal(gen, (M, K), 1e-3), _activation(gen, K, N).t().contiguous()
            b_q, b_s = _in_groups(b.to(BF16).float())
        else:
            a, b = _activation(gen, M, K), _normal(gen, (N, K), 0.02)
            b_q, b_s = _in_blocks(b)
        a_q, a_s = _in_groups(a.to(BF16).float())
        st.update(a_q=a_q.view(torch.uint8), a_s=a_s, b_q=b_q.view(torch.uint8), b_s=b_s)
    else:
        experts, weight = _routing(case, gen)
        row, source, offsets = _plan(case, experts)
        if kind == "experts":
            x = _activation(gen, case["tokens"], case["cols"]).to(BF16)
            R = source.numel()
            st.update(experts=experts, weight=weight, x=x, y=_normal(gen, (R, case["cols"])).to(BF16),
                      d_out=_normal(gen, x.shape, 1e-3).to(BF16), d_rows=_normal(gen, (R, case["cols"]), 1e-3).to(BF16))
            return st
        st["offsets"], st["sizes"] = offsets, (offsets[1:] - offsets[:-1]).tolist()
        filled = (source >= 0)[:, None]
        E = case["E"]
        if kind == "grouped":
            x = torch.where(filled, _activation(gen, source.numel(), case["K"]), 0.0).to(BF16).float()
            st["a_q"], st["a_e"], st["a_s"] = _two_level(x)
            made = [_per_tensor(_normal(gen, (case["N"], case["K"]), 0.02)) for _ in range(E)]
            b_q = torch.stack([q for q, _ in made])
            if case["view"]:        # one matrix of [N x E K] bytes, an expert's columns side by side
                b_q = b_q.permute(1, 0, 2).contiguous().permute(1, 0, 2)
            st.update(b_q=b_q, b_s=torch.stack([s for _, s in made]))
        else:
            dy = torch.where(filled, _normal(gen, (source.numel(), case["M"]), 1e-3), 0.0).to(BF16).float()
            x = torch.where(filled, _activation(gen, source.numel(), case["N"]), 0.0).to(BF16).float()
            st["a_q"], st["a_e"], st["a_s"] = _two_level(dy.t().contiguous())
            st["b_q"], st["b_e"], st["b_s"] = _two_level(x.t().contiguous())
    return st


# ---- the operators

def _values(q, t):
    return q.view(FP8).to(t)


def _grouped_values(q, s, t):
    """codes of [rows x K] with a scale per row and 128 columns"""
    return _values(q, t) * s.to(t).repeat_interleave(128, 1)[:, :q.shape[1]]


def _blocked_values(q, s, t):
    return _values(q, t) * s.to(t).repeat_interleave(128, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]


def _exponent_values(q, e, t):
    return _values(q, t) * torch.exp2(e.to(t) - 127.0).repeat_interleave(32, 1)


def _run_quant(st):
    case, x = st["case"], st["x"]
    if own:
        import paper_2511_05811_amd as moss
        if case["weight"]:
            q, s, q_t, s_t = moss.quant_block128_weight(x, want_transpose=case["transpose"])
            return (q.view(FP8), s, q_t.view(FP8), s_t) if case["transpose"] else (q.view(FP8), s)
        r = moss.quant_block128(x, (moss.MOSS_Q_ROW if case["row"] else 0) | (moss.MOSS_Q_COL if case["col"] else 0))
        return (((r["q_row"].view(FP8), r["s_row"]) if case["row"] else ()) + ((r["q_col"].view(FP8), r["s_col"]) if case["col"] else ()))
    x = x.float()
    if case["weight"]:
        q, s = _in_blocks(x)
        return (q, s, q.view(torch.uint8).t().contiguous().view(FP8), s.t().contiguous()) if case["transpose"] else (q, s)
    return (_in_groups(x) if case["row"] else ()) + (_in_groups(x.t().contiguous()) if case["col"] else ())


def _run_block_gemm(st):
    if own:
        import paper_2511_05811_amd as moss
        return moss.gemm_fp8_block128(st["a_q"], st["a_s"], st["b_q"], st["b_s"])
    a = _grouped_values(st["a_q"], st["a_s"], F32)
    b = (_grouped_values if st["case"]["dw"] else _blocked_values)(st["b_q"], st["b_s"], F32)
    return (a @ b.t()).to(BF16)


def _run_grouped(st):
    if own:
        import paper_2511_05811_amd as moss
        return moss.gemm_fp8_mx_grouped(st["a_q"], st["a_e"], st["a_s"], st["b_q"], st["b_s"], st["offsets"])
    a = _exponent_values(st["a_q"], st["a_e"], F32).split(st["sizes"])
    s = (st["a_s"] * st["b_s"]).split(1)
    return torch.cat([(x @ _values(w, F32).t()) * f for x, w, f in zip(a, st["b_q"], s)]).to(BF16)


def _run_grouped_dw(st):
    if own:
        import paper_2511_05811_amd as moss
        return moss.gemm_fp8_mx_grouped_dw(st["a_q"], st["a_e"], st["a_s"], st["b_q"], st["b_e"], st["b_s"], st["offsets"], out_dtype=BF16)
    a = _exponent_values(st["a_q"], st["a_e"], F32).split(st["sizes"], 1)
    b = _exponent_values(st["b_q"], st["b_e"], F32).split(st["sizes"], 1)
    return (torch.stack([x @ y.t() for x, y in zip(a, b)]) * (st["a_s"] * st["b_s"])).to(BF16)


def _word(bits):
    """a maximum word as the value that it holds"""
    return bits.to(torch.int16).view(BF16)


def _experts_in(st, t):
    """the plan, and every result of the step in type t, from the definition"""
    case, x, w = st["case"], st["x"].to(t), st["weight"].to(t)
    row, source, offsets = _plan(case, st["experts"])
    filled, token = (source >= 0)[:, None], (source.clamp(min=0) // case["k"]).long()
    there, at = (row >= 0)[..., None], row.clamp(min=0).long()
    rows = torch.where(filled, x[token], 0.0)
    back = torch.where(there, st["y"].to(t)[at], 0.0)
    out = (back * w[..., None]).sum(1)
    d_out = st["d_out"].to(t)
    d_y = torch.where(filled, w.reshape(-1)[source.clamp(min=0).long()][:, None] * d_out[token], 0.0)
    d_w = (d_out[:, None] * back).sum(2)
    d_x = torch.where(there, st["d_rows"].to(t)[at], 0.0).sum(1)
    return row, source, offsets, rows, out, d_y, d_w, d_x


def _run_experts(st):
    if own:
        import paper_2511_05811_amd as moss
        plan = moss.expert_plan(st["experts"], st["case"]["E"], multiple=st["case"]["multiple"])
        rows, top = moss.expert_dispatch_bf16(st["x"], plan)
        out = moss.expert_combine_bf16(st["y"], plan, st["weight"])
        d_y, d_w, d_top = moss.expert_combine_bf16_backward(st["d_out"], st["y"], plan, st["weight"])
        d_x = moss.expert_combine_bf16(st["d_rows"], plan)
        return plan["row_of"], plan["source"], plan["offsets"], rows, _word(top), out, d_y, d_w, _word(d_top), d_x
    row, source, offsets, rows, out, d_y, d_w, d_x = _experts_in(st, F32)
    rows, d_y = rows.to(BF16), d_y.to(BF16)
    return row, source, offsets, rows, rows.abs().amax().view(1), out.to(BF16), d_y, d_w, d_y.abs().amax().view(1), d_x.to(BF16)


_RUN = dict(block_quant=_run_quant, block_gemm=_run_block_gemm, grouped=_run_grouped, grouped_dw=_run_grouped_dw, experts=_run_experts)


def run(state):
    return _RUN[state["case"]["kind"]](state)


# ---- what the paths cannot do without

def work(case):
    kind = case["kind"]
    if kind == "block_quant":
        n = case["rows"] * case["cols"]
        if case["weight"]:
            return dict(bytes=n * ((2 if case["bf16"] else 4) + 1 + case["transpose"]), flops=3 * n)
        out = case["row"] + case["col"]
        return dict(bytes=n * (2 + out) + 4 * n // 128 * out, flops=3 * n * out)
    if kind == "block_gemm":
        M, N, K = case["M"], case["N"], case["K"]
        scales = M * _blocks(K) + (N if case["dw"] else _blocks(N)) * _blocks(K)
        return dict(bytes=(M + N) * K + 4 * scales + 2 * M * N, flops=2 * M * N * K)
    n, E = case["tokens"] * case["k"], case["E"]
    if kind == "grouped":
        N, K = case["N"], case["K"]
        return dict(bytes=n * K * 33 // 32 + min(E, n) * N * K + 2 * n * N, flops=2 * n * N * K)
    if kind == "grouped_dw":
        M, N = case["M"], case["N"]
        return dict(bytes=n * (M + N) * 33 // 32 + 2 * E * M * N, flops=2 * n * M * N)
    C, T = case["cols"], case["tokens"]
    # dispatch: x in, rows out; combine: rows in, out; its gradient: d_out and y in, d_y out; that of dispatch: rows in, d_x out
    return dict(bytes=2 * C * (4 * T + 5 * n) + 24 * n, flops=7 * n * C)


# ---- from the definitions, in 64 bits

def _exact_codes(x, dim_rows, dim_cols):
    """E4M3 values and scales of x in blocks of dim_rows x dim_cols.  The scale is amax / 448 in 32 bits and a value is rounded
    from the product of x and the scale's reciprocal in 32 bits, so both are followed step by step in 64."""
    rows, cols = x.shape
    r, c = -(-rows // dim_rows), -(-cols // dim_cols)
    wide = torch.zeros(r * dim_rows, c * dim_cols, device=x.device, dtype=F64)
    wide[:rows, :cols] = x
    tiles = wide.view(r, dim_rows, c, dim_cols)
    top = tiles.abs().amax((1, 3))
    s = torch.where(top > 0, top / 448.0, 1.0).float().double()
    inv = (1.0 / s).clamp(max=FLT_MAX).float().double()
    y = (tiles * inv[:, None, :, None]).float().double().clamp(-448.0, 448.0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(y / step) * step).view(r * dim_rows, c * dim_cols)[:rows, :cols], s


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "block_quant":
        x = st["x"].double()
        if case["weight"]:
            q, s = _exact_codes(x, 128, 128)
            return (q, s, q.t(), s.t()) if case["transpose"] else (q, s)
        return (_exact_codes(x, 1, 128) if case["row"] else ()) + (_exact_codes(x.t(), 1, 128) if case["col"] else ())
    if kind == "block_gemm":
        spread = lambda s, n, k: s.double().repeat_interleave(128, 1)[:, :k].repeat_interleave(n // s.shape[0] if n == s.shape[0] else 128, 0)[:n]
        decoded = lambda q: q.view(FP8).double()
        M, N, K = case["M"], case["N"], case["K"]
        a, b = decoded(st["a_q"]) * spread(st["a_s"], M, K), decoded(st["b_q"])
        b = b * spread(st["b_s"], N, K)
        return a @ b.t()
    if kind == "experts":
        return _exact_experts(st)
    power = lambda e: torch.pow(2.0, e.double() - 127.0).unsqueeze(2).expand(-1, -1, 32).flatten(1)
    a = st["a_q"].view(FP8).double() * power(st["a_e"])
    ends = st["offsets"].tolist()
    if kind == "grouped":
        out = torch.zeros(a.shape[0], case["N"], device=DEV, dtype=F64)
        for g in range(case["E"]):
            out[ends[g]:ends[g + 1]] = a[ends[g]:ends[g + 1]] @ st["b_q"][g].contiguous().view(FP8).double().t() * (st["a_s"].double() * st["b_s"][g].double())
        return out
    b = st["b_q"].view(FP8).double() * power(st["b_e"])
    out = torch.zeros(case["E"], case["M"], case["N"], device=DEV, dtype=F64)
    for g in range(case["E"]):
        out[g] = a[:, ends[g]:ends[g + 1]] @ b[:, ends[g]:ends[g + 1]].t() * (st["a_s"].double() * st["b_s"].double())
    return out


def _exact_experts(st):
    """Assignment by assignment on the host for the plan, then row by row of the definitions in 64 bits."""
    case = st["case"]
    T, k, E, m, R = case["tokens"], case["k"], case["E"], case["multiple"], _capacity(case)
    lists = [[] for _ in range(E)]
    for a, e in enumerate(st["experts"].reshape(-1).tolist()):
        if 0 <= e < E:
            lists[e].append(a)
    source, offsets = [], []
    for mine in lists:
        offsets.append(len(source))
        source += mine + [-1] * (-len(mine) % m)
    source += [-1] * (R - len(source))
    offsets.append(R)
    row = [-1] * (T * k)
    for r, a in enumerate(source):
        if a >= 0:
            row[a] = r
    put = lambda v: torch.tensor(v, device=DEV, dtype=torch.int32)
    x, y, w, d_out, d_rows = (st[n].double() for n in ("x", "y", "weight", "d_out", "d_rows"))
    src = put(source).long()
    filled = (src >= 0).nonzero().flatten()
    asg = src[filled]
    rows, d_y = torch.zeros(R, x.shape[1], device=DEV, dtype=F64), torch.zeros(R, x.shape[1], device=DEV, dtype=F64)
    rows[filled] = x[asg // k]
    d_y[filled] = w.flatten()[asg, None] * d_out[asg // k]
    out, d_x = torch.zeros_like(x), torch.zeros_like(x)
    out.index_add_(0, asg // k, w.flatten()[asg, None] * y[filled])
    d_x.index_add_(0, asg // k, d_rows[filled])
    d_w = torch.zeros(T * k, device=DEV, dtype=F64)
    d_w[asg] = (d_out[asg // k] * y[filled]).sum(1)
    return (put(row).view(T, k), put(source), put(offsets), rows, rows.abs().amax().view(1), out, d_y, d_w.view(T, k), d_y.abs().amax().view(1), d_x)
