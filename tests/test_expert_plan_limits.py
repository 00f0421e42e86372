"""How many rows the plan gives an expert, up to the most that its 32-bit rows can count (asked on the host, no GPU needed)."""
import ctypes as C

import pytest

import paper_2511_05811_amd as moss

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("multiple", [1, 3, 7, 32, 100, 4095, 4096])
def test_rows_of_one_expert_with_all_assignments(multiple):
    L = moss.load()
    filled = L.moss_internal_expert_filled
    filled.restype, filled.argtypes = C.c_int64, [C.c_int64, C.c_int64]
    largest = MOST // multiple * multiple                       # what one expert's rows may come to at most
    for total in (0, 1, multiple, multiple + 1, largest - multiple + 1, largest - 1, largest):
        want = -(-total // multiple) * multiple
        assert filled(total, multiple) == want
        if total:
            assert want == L.moss_expert_rows(total, 1, 1, multiple) <= MOST
