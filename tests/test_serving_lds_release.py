"""The serving kernels whose LDS is refilled behind hand-written barriers: at each barrier a wave's reads of LDS have returned (the others may
refill what it read), and, where the refill is a transfer from memory to LDS, the wave's transfers have arrived (the others will read them).
Checked in the machine code of the source, over all paths."""
import os
import re
import subprocess

import pytest

from paper_2407_02891_amd import build as hip_build
from tests.test_lds_release import _kernels, _outstanding


def _memory(body):
    """The same for vector memory: its instructions and waits in the place of LDS's."""
    out = []
    for number, line in body:
        if re.match(r"(global|buffer|flat)_", line):
            line = "ds_of " + line
        elif line.startswith("ds_"):
            line = "v_of " + line
        elif line.startswith("s_waitcnt"):
            m = re.search(r"vmcnt\((\d+)\)", line)
            line = f"s_waitcnt lgkmcnt({m[1]})" if m else "s_nop 0"
        out.append((number, line))
    return out


def test_the_translation_itself():
    def most(*lines):
        return list(_outstanding(_memory(list(enumerate(lines)))).values())

    load = "global_load_lds_dwordx4 v[0:1], off"
    assert most(load, "s_waitcnt lgkmcnt(0)", "s_barrier") == [1]
    assert most(load, "s_waitcnt vmcnt(0) lgkmcnt(0)", "s_barrier") == [0]
    assert most("ds_read_b128 v[0:3], v4", "s_barrier") == [0]
    assert most(load, load, "s_waitcnt vmcnt(1)", "s_barrier") == [1]


@pytest.mark.parametrize("source,kernel,count,transfers", [("bcq_attend_chunk.hip", "bcq_attend_chunk_kernel", 18, True),
                                                          ("bcq_lora.hip", "bcq_lora_many_kernel", 8, False)])
def test_reads_and_transfers_are_over_at_barriers(tmp_path, source, kernel, count, transfers):
    out = tmp_path / "out.s"
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-fPIC", "-shared")]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + flags + ["--cuda-device-only", "-S", os.path.join(hip_build.CSRC, source), "-o", str(out)],
                   check=True, stderr=subprocess.DEVNULL)
    bodies = {k: body for k, body in _kernels(out.read_text()).items() if kernel in k}
    assert len(bodies) == count
    for name, body in bodies.items():
        reads = _outstanding(body)
        assert len(reads) >= 2 and not any(reads.values()), (name, reads)
        if transfers:
            assert any("load_lds" in line for _, line in body)
            arrived = _outstanding(_memory(body))
            assert not any(arrived.values()), (name, arrived)
