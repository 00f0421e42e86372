"""Wait states around the copies into LDS, which are inline assembly, in the kernels with blocks of 128 and of grouped rows: these keep
some of their scalar values in lanes of vector registers, and a scalar register that a vector instruction has written takes five wait states until
a memory instruction may read it (looked for in assembly built from source here, no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2511_05811_amd import build


@pytest.mark.parametrize("source", ["moss_gemm_block.hip", "moss_gemm_grouped.hip"])
def test_addresses_of_copies_are_there_in_time(source):
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    res = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + flags + ["-I", build.INCLUDE, "-S", "--offload-device-only", "-o", "-",
                          os.path.join(build.CSRC, source)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    lines = [l.split(";")[0].strip() for l in res.stdout.splitlines()]
    lines = [l for l in lines if l and not l.startswith(".") and not l.endswith(":")]
    copies = 0
    for i, line in enumerate(lines):
        if not line.startswith("global_load_" + "lds"):
            continue
        copies += 1
        first, last = (int(v) for v in re.search(r"s\[(\d+):(\d+)\]", line).groups())
        states = 0
        for before in reversed(lines[max(0, i - 8):i]):
            if states >= 5 or before.startswith("s_endpgm"):
                break
            wrote = re.match(r"v_read(?:first)?lane_b32 s(\d+)", before)
            assert not (wrote and first <= int(wrote[1]) <= last), (before, line, states)
            nop = re.match(r"s_nop (\d+)", before)
            states += int(nop[1]) + 1 if nop else 1
    assert copies > 100
