"""Results of the matrix instructions that are inline assembly, for which the compiler keeps no distance: in the kernels with blocks of 128
and of grouped rows nothing touches the vector registers of a result, spills among it, before two further matrix instructions have been issued
(the unit takes them one after the other) or its wait states have passed (looked for in assembly built from source here, no GPU
needed)."""
import os
import re
import subprocess

import pytest

from paper_2511_05811_amd import build

# wait states (of four clocks) behind which a result may be touched: the instruction's passes of four clocks, 8 for 16 x 16 x 128 and 16 for
# 32 x 32 x 64, and four more
STATES = {"16x16": 8 + 4, "32x32": 16 + 4}


def vector_registers(token):
    m = re.fullmatch(r"v\[(\d+):(\d+)\]", token)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.fullmatch(r"v(\d+)", token)
    return {int(m[1])} if m else set()


def too_early(lines):
    """Lines of a kernel that touch a result too early, as the text goes, and the number of matrix instructions"""
    found, under_way, count = [], [], 0
    for line in lines:
        op = line.split()[0]
        tokens = line[len(op):].replace(",", " ").split()
        if not op.startswith("v_mfma"):
            touched = set().union(*(vector_registers(t) for t in tokens)) if tokens else set()
            found += [(line, u["by"]) for u in under_way if u["result"] & touched]
            nop = re.match(r"s_nop (\d+)", line)
            for u in under_way:
                u["states"] += int(nop[1]) + 1 if nop else 1
        else:
            count += 1
            operands = set().union(*(vector_registers(t) for t in tokens[1:3] + tokens[4:6]))
            found += [(line, u["by"]) for u in under_way if u["result"] & operands]
            for u in under_way:
                u["behind"] += 1
            result = vector_registers(tokens[0])
            under_way = [u for u in under_way if u["result"] != result]
            under_way.append(dict(result=result, behind=0, states=0, by=line, needs=STATES["32x32" if "32x32" in op else "16x16"]))
        under_way = [u for u in under_way if u["behind"] < 2 and u["states"] < u["needs"]]
    return found, count


@pytest.mark.parametrize("source", ["moss_gemm_block.hip", "moss_gemm_grouped.hip"])
def test_results_are_left_alone_until_they_are_there(source):
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    res = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + flags + ["-I", build.INCLUDE, "-S", "--offload-device-only", "-o", "-",
                          os.path.join(build.CSRC, source)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    kernels, at = {}, None
    for line in res.stdout.splitlines():
        name = re.match(r"(_Z\w+):", line)
        if name:
            at = kernels.setdefault(name[1], [])
        line = line.split(";")[0].strip()
        if at is not None and line and not line.startswith(".") and not line.endswith(":"):
            at.append(line)
    total = 0
    for name, lines in kernels.items():
        found, count = too_early(lines)
        assert not found, (name, found[:3])
        total += count
    assert total > 100


def test_a_result_touched_too_early_is_found():
    product = "v_mfma_f32_16x16x128_f8f6f4 v[{}:{}], v[40:47], v[48:55], 0"
    one, two, three = (product.format(4 * i, 4 * i + 3) for i in range(3))
    for touch in ("v_fma_f32 v30, v1, v31, v30", "scratch_store_dword off, v2, off offset:4", "v_mov_b32_e32 v3, 0"):
        assert too_early([one, two, touch])[0] and too_early([one, "s_nop 10", touch])[0]
        assert not too_early([one, two, three, touch])[0] and not too_early([one, "s_nop 7", "s_nop 3", touch])[0]
    assert too_early([one, two.replace("v[40:47]", "v[0:7]")])[0]
