"""The attention kernels keep a few scalar values in the lanes of a vector register (never in memory, which the build refuses): outside their
loop over the keys, in the machine code."""
import os
import re
import subprocess

import pytest

from paper_2407_02891_amd import build as hip_build
from tests.test_lds_release import _kernels


def _loop(lines):
    """The smallest of the loops that hold the most matrix instructions."""
    at = {line[:-1]: i for i, line in enumerate(lines) if line.endswith(":")}
    loops = []
    for i, line in enumerate(lines):
        m = re.match(r"s_c?branch\w* (\.L\w+)", line)
        if m and at.get(m[1], len(lines)) < i:
            loops.append((sum("mfma" in x for x in lines[at[m[1]]:i]), at[m[1]] - i, at[m[1]], i))
    return lines[max(loops)[2]:max(loops)[3]] if loops else []


def _reloads(lines, of):
    kept = {m[1] for x in lines if (m := re.match(r"v_writelane_b32 (v\d+)", x))}
    return sum(1 for x in of if (m := re.match(r"v_readlane_b32 s\d+, (v\d+), \d+", x)) and m[1] in kept)


def test_the_count_itself():
    body = ["v_writelane_b32 v9, s3, 0", ".L1:", "v_mfma x", "v_readlane_b32 s4, v9, 0", "v_readlane_b32 s4, v8, 0", ".L2:", "v_add x", "s_cbranch_scc1 .L2",
            "s_cbranch_scc1 .L1", "v_readlane_b32 s4, v9, 0"]
    assert len(_loop(body)) == 7 and _reloads(body, _loop(body)) == 1


@pytest.mark.parametrize("source,kernel", [("bcq_attend.hip", "bcq_attend_stream_kernel"), ("bcq_attend_chunk.hip", "bcq_attend_chunk_kernel")])
def test_no_scalar_comes_back_in_the_loop_over_keys(tmp_path, source, kernel):
    out = tmp_path / "out.s"
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-fPIC", "-shared")]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + flags + ["--cuda-device-only", "-S", os.path.join(hip_build.CSRC, source), "-o", str(out)],
                   check=True, stderr=subprocess.DEVNULL)
    bodies = {k: [line for _, line in body] for k, body in _kernels(out.read_text()).items() if kernel in k}
    assert bodies
    for name, lines in bodies.items():
        loop = _loop(lines)
        assert sum("mfma" in x for x in loop) >= 20, name
        assert _reloads(lines, loop) == 0, name
