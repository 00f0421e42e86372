"""The native calls for blocks of 128 and for experts give what their Python code gives: outputs, returned objects and refusals."""
import pytest
import torch

import paper_2511_05811_amd as moss
from test_gpu_calls import both, same

ROW, COL = moss.MOSS_Q_ROW, moss.MOSS_Q_COL


@pytest.fixture
def data():
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    r = lambda *s, k=1.0: torch.randn(*s, generator=gen, device="cuda:0") * k
    d = dict(x=r(64, 256).bfloat16(), wide=r(64, 320).bfloat16()[:, :256], w=r(3, 96, 256, k=0.02), weights=r(64, 2).abs())
    d["experts"] = torch.randint(0, 3, (64, 2), generator=gen, device="cuda:0", dtype=torch.int32)
    d["plan"] = moss.expert_plan(d["experts"], 3)
    d["y"] = r(d["plan"]["source"].numel(), 256).bfloat16()
    d["q"] = moss.quant_act_2level(d["y"], ROW | COL)
    d["wq"] = torch.randint(0, 120, (3, 96, 256), generator=gen, device="cuda:0", dtype=torch.uint8)
    d["ws"] = r(3).abs()
    return d


def grouped(d, **kw):
    a = dict(a_q=d["q"]["q_row"], a_e=d["q"]["e_row"], a_s=d["q"]["s"], b_q=d["wq"], b_s=d["ws"], offsets=d["plan"]["offsets"])
    a.update(kw)
    return moss.gemm_fp8_mx_grouped(**a)


def grouped_dw(d, **kw):
    q = d["q"]
    a = dict(a_q=q["q_col"], a_e=q["e_col"], a_s=q["s"], b_q=q["q_col"][:96], b_e=q["e_col"][:96], b_s=q["s"], offsets=d["plan"]["offsets"])
    a.update(kw)
    return moss.gemm_fp8_mx_grouped_dw(**a)


def blocks(d, rows=False, **kw):
    a = moss.quant_block128(d["x"])
    b = moss.quant_block128(d["y"]) if rows else dict(zip(("q_row", "s_row"), moss.quant_block128_weight(d["w"][0])))
    return moss.gemm_fp8_block128(a["q_row"], a["s_row"], b["q_row"], b["s_row"], **kw)


CALLS = {
    "rows": lambda d: moss.quant_block128(d["x"]),
    "both groupings, strided": lambda d: moss.quant_block128(d["wide"], ROW | COL),
    "outputs given": lambda d: moss.quant_block128(d["x"], ROW | COL, out=dict(moss.quant_block128(d["x"], ROW | COL))),
    "an output of another shape": lambda d: moss.quant_block128(d["x"], ROW, out=dict(q_row=torch.zeros(64, 128, dtype=torch.uint8, device="cuda:0"))),
    "no grouping": lambda d: moss.quant_block128(d["x"], 0),
    "another flag": lambda d: moss.quant_block128(d["x"], ROW | 8),
    "float32": lambda d: moss.quant_block128(d["x"].float()),
    "one row": lambda d: moss.quant_block128(d["wide"][:1]),
    "odd width": lambda d: moss.quant_block128(d["x"][:, :40]),
    "on the host": lambda d: moss.quant_block128(d["x"].cpu()),
    "block product": lambda d: blocks(d),
    "block product, a scale per row": lambda d: blocks(d, rows=True),
    "block product into float32": lambda d: blocks(d, out_dtype=torch.float32),
    "block product into a view": lambda d: blocks(d, out=torch.zeros(64, 128, dtype=torch.bfloat16, device="cuda:0")[:, :96]),
    "block product that accumulates": lambda d: blocks(d, out=torch.ones(64, 96, device="cuda:0"), accumulate=True),
    "block product that accumulates BF16": lambda d: blocks(d, accumulate=True),
    "block product into float16": lambda d: blocks(d, out=torch.ones(64, 96, device="cuda:0").half()),
    "block product into another shape": lambda d: blocks(d, out=torch.ones(64, 95, device="cuda:0")),
    "grouped": lambda d: grouped(d),
    "grouped, without exponents": lambda d: grouped(d, a_e=None),
    "grouped, one scale": lambda d: grouped(d, b_s=d["q"]["s"]),
    "grouped, strided scales": lambda d: grouped(d, b_s=torch.ones(3, 12, device="cuda:0")[:, 1]),
    "grouped, a view of weights": lambda d: grouped(d, b_q=d["wq"].permute(1, 0, 2).contiguous().permute(1, 0, 2)),
    "grouped, transposed weights": lambda d: grouped(d, b_q=d["wq"].transpose(1, 2)),
    "grouped, int64 offsets": lambda d: grouped(d, offsets=d["plan"]["offsets"].long()),
    "grouped, too few offsets": lambda d: grouped(d, offsets=d["plan"]["offsets"][:3]),
    "grouped into float32": lambda d: grouped(d, out_dtype=torch.float32),
    "grouped that accumulates": lambda d: grouped(d, out=torch.ones(d["y"].shape[0], 96, device="cuda:0"), accumulate=True),
    "grouped that accumulates BF16": lambda d: grouped(d, accumulate=True),
    "weight gradients": lambda d: grouped_dw(d),
    "weight gradients in BF16": lambda d: grouped_dw(d, out_dtype=torch.bfloat16),
    "weight gradients that accumulate": lambda d: grouped_dw(d, out=torch.ones(3, 256, 96, device="cuda:0"), accumulate=True),
    "weight gradients into another shape": lambda d: grouped_dw(d, out=torch.ones(3, 96, 256, device="cuda:0")),
    "weight gradients without exponents": lambda d: grouped_dw(d, a_e=None),
    "plan": lambda d: moss.expert_plan(d["experts"], 3),
    "plan, rows given": lambda d: moss.expert_plan(d["experts"], 3, 64, 512),
    "plan, too few rows": lambda d: moss.expert_plan(d["experts"], 3, 32, 32),
    "plan, no experts": lambda d: moss.expert_plan(d["experts"], 0),
    "plan, int64": lambda d: moss.expert_plan(d["experts"].long(), 3),
    "plan, too many experts": lambda d: moss.expert_plan(d["experts"], 5000),
    "dispatch": lambda d: moss.expert_dispatch_bf16(d["wide"], d["plan"]),
    "dispatch, outputs given": lambda d: moss.expert_dispatch_bf16(d["x"], d["plan"], torch.zeros_like(d["y"]), torch.zeros(1, dtype=torch.int32, device="cuda:0")),
    "dispatch of too few tokens": lambda d: moss.expert_dispatch_bf16(d["x"][:63], d["plan"]),
    "dispatch without a plan": lambda d: moss.expert_dispatch_bf16(d["x"], None),
    "dispatch of float32": lambda d: moss.expert_dispatch_bf16(d["x"].float(), d["plan"]),
    "dispatch, odd width": lambda d: moss.expert_dispatch_bf16(d["x"][:, :12], d["plan"]),
    "combine": lambda d: moss.expert_combine_bf16(d["y"], d["plan"], d["weights"]),
    "combine without weights": lambda d: moss.expert_combine_bf16(d["y"], d["plan"]),
    "combine, output given": lambda d: moss.expert_combine_bf16(d["y"], d["plan"], d["weights"], torch.zeros(64, 320, dtype=torch.bfloat16, device="cuda:0")[:, :256]),
    "combine, weights of another type": lambda d: moss.expert_combine_bf16(d["y"], d["plan"], d["weights"].bfloat16()),
    "combine of too few rows": lambda d: moss.expert_combine_bf16(d["y"][:-1], d["plan"]),
    "gradient of combine": lambda d: moss.expert_combine_bf16_backward(d["wide"], d["y"], d["plan"], d["weights"]),
    "gradient of combine, outputs given": lambda d: moss.expert_combine_bf16_backward(
        d["x"], d["y"], d["plan"], d["weights"], torch.zeros_like(d["y"]), torch.zeros(64, 2, device="cuda:0"), torch.zeros(1, dtype=torch.int32, device="cuda:0")),
    "gradient of combine, another stride": lambda d: moss.expert_combine_bf16_backward(
        d["x"], d["y"], d["plan"], d["weights"], torch.zeros(d["y"].shape[0], 320, dtype=torch.bfloat16, device="cuda:0")[:, :256]),
    "gradient of combine without weights": lambda d: moss.expert_combine_bf16_backward(d["x"], d["y"], d["plan"], None),
}


def test_plain_arguments_are_what_the_native_calls_take():
    """On the CPU nothing is plain: every function answers None, and the Python code refuses."""
    from paper_2511_05811_amd import binding
    binding._bind_calls()
    if not binding._calls:
        pytest.fail("_moss_calls has not been built for this torch")
    x, i = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 2, dtype=torch.int32)
    assert binding._calls.quant_block128(x, ROW, None) is None
    assert binding._calls.expert_plan(i, 4, 32, None) is None
    assert binding._calls.expert_combine_bf16(x, dict(row_of=i, source=i[:, 0]), None, None) is None


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CALLS))
def test_native_and_python_calls_agree(monkeypatch, data, name):
    native, python = both(monkeypatch, lambda: CALLS[name](data))
    torch.cuda.synchronize()
    same(native, python)


WEIGHT_CALLS = {
    "weight": lambda w: moss.quant_block128_weight(w),
    "transposed": lambda w: moss.quant_block128_weight(w, True),
    "BF16": lambda w: moss.quant_block128_weight(w.bfloat16(), want_transpose=True),
    "outputs given": lambda w: moss.quant_block128_weight(w, True, *moss.quant_block128_weight(w * 2, True)),
    "the transposed output alone asks for it": lambda w: moss.quant_block128_weight(w, wq_t=torch.zeros(256, 288, dtype=torch.uint8, device="cuda:0")),
    "an output of another shape": lambda w: moss.quant_block128_weight(w, wq=torch.zeros(288, 128, dtype=torch.uint8, device="cuda:0")),
    "a view": lambda w: moss.quant_block128_weight(w[:, :128]),
    "float16": lambda w: moss.quant_block128_weight(w.half()),
    "odd height": lambda w: moss.quant_block128_weight(w[:40], True),
    "odd width": lambda w: moss.quant_block128_weight(w[:, :40].contiguous()),
    "on the host": lambda w: moss.quant_block128_weight(w.cpu()),
    "three dimensions": lambda w: moss.quant_block128_weight(w.view(3, 96, 256)),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(WEIGHT_CALLS))
def test_native_and_python_calls_agree_on_weights(monkeypatch, name):
    w = torch.randn(288, 256, generator=torch.Generator("cuda:0").manual_seed(2), device="cuda:0")
    native, python = both(monkeypatch, lambda: WEIGHT_CALLS[name](w))
    torch.cuda.synchronize()
    same(native, python)
