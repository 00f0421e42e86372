"""Tensors of one call that lie on different GPUs are refused before anything is launched: no kernel writes into another device's memory."""
import pytest
import torch

import paper_2511_05811_amd as moss

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")]
BOTH = moss.MOSS_Q_ROW | moss.MOSS_Q_COL


@pytest.mark.parametrize("name,shape,dtype", [("q_row", (64, 128), torch.uint8), ("s_row", (64, 1), torch.float32), ("q_col", (128, 64), torch.uint8),
                                              ("s_col", (128, 1), torch.float32)])
def test_outputs_of_the_block_quantizer(name, shape, dtype):
    x = torch.ones((64, 128), dtype=torch.bfloat16, device="cuda:0")
    far = torch.full(shape, 7, dtype=dtype, device="cuda:1")
    with pytest.raises(AssertionError):
        moss.quant_block128(x, BOTH, out={name: far})
    assert bool((far == 7).all())


def test_a_call_on_the_device_that_is_not_current():
    x = torch.ones((64, 128), dtype=torch.bfloat16, device="cuda:1")
    with pytest.raises(AssertionError):
        moss.quant_block128(x, BOTH)
    with torch.cuda.device(1):
        q = moss.quant_block128(x, BOTH)
        assert q["q_row"].device == x.device and bool((q["s_row"] > 0).all())
