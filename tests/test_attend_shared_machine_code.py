"""Attention with shared prefixes in the machine code of its source: its waves' reads of LDS and transfers to it are over at each barrier that others refill or
read behind, over all paths, and its tiles' loop over keys brings no scalar back from a lane."""
import os
import re
import subprocess

import pytest

from paper_2407_02891_amd import build as hip_build
from tests.test_lds_release import _kernels, _outstanding
from tests.test_serving_spills import _reloads


@pytest.fixture(scope="module")
def bodies(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "out.s"
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-fPIC", "-shared")]
    source = os.path.join(hip_build.CSRC, "bcq_attend_shared.hip")
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + flags + ["--cuda-device-only", "-S", source, "-o", str(out)], check=True,
                   stderr=subprocess.DEVNULL)
    found = {k: body for k, body in _kernels(out.read_text()).items() if "bcq_attend_shared_kernel" in k}
    assert len(found) == 32   # dimensions, types, addressings, and who lays the lines out
    return found


def _loops(lines):
    """The loops of 20 matrix instructions and more, with transfers to LDS, that hold no other such loop, as (first, last) lines."""
    at = {line[:-1]: i for i, line in enumerate(lines) if line.endswith(":")}
    loops = set()
    for i, line in enumerate(lines):
        m = re.match(r"s_c?branch\w* (\.L\w+)", line)
        if m and at.get(m[1], len(lines)) < i and sum("mfma" in x for x in lines[at[m[1]]:i]) >= 20 and any("load_lds" in x for x in lines[at[m[1]]:i]):
            loops.add((at[m[1]], i))
    return [a for a in loops if not any(b != a and a[0] <= b[0] and b[1] <= a[1] for b in loops)]


def _transfers(body):
    """{line of an s_barrier: whether a transfer from memory to LDS may be on its way there}, over all paths.  Vector memory returns in order, so the last
    transfer has arrived once a wait leaves no more than what was issued behind it."""
    blocks, order = {"": []}, [""]
    for number, line in body:
        if line.endswith(":"):
            order.append(line[:-1])
            blocks[order[-1]] = []
        else:
            blocks[order[-1]].append((number, line))
    none = 64                                              # (no wait counts that far)
    entry, at, work = {"": none}, {}, [""]                 # fewest operations behind the last transfer
    while work:
        block = work.pop()
        behind, falls, to = entry[block], True, []
        for number, line in blocks[block]:
            op, _, rest = line.partition(" ")
            if re.match(r"(global|buffer|flat)_", op):
                behind = 0 if "lds" in op or " lds" in rest else min(behind + 1, none)
            elif op == "s_waitcnt" and (m := re.search(r"vmcnt\((\d+)\)", rest)) and int(m[1]) <= behind:
                behind = none
            elif op == "s_barrier":
                at[number] = at.get(number, False) or behind < none
            elif op.startswith("s_cbranch"):
                to.append((rest.strip(), behind))
            elif op in ("s_branch", "s_endpgm"):
                to += [(rest.strip(), behind)] if op == "s_branch" else []
                falls = False
                break
        if falls and block != order[-1]:
            to.append((order[order.index(block) + 1], behind))
        for target, count in to:
            if entry.get(target, none + 1) > count:
                entry[target] = count
                work.append(target)
    return at


def test_the_transfers_themselves():
    def on_their_way(*lines):
        return list(_transfers(list(enumerate(lines))).values())

    load, store, barrier = "global_load_lds_dwordx4 v[0:1], off", "global_store_dwordx4 v[0:1], v[2:5], off", "s_barrier"
    assert on_their_way(load, barrier) == [True] and on_their_way(store, barrier) == [False]
    assert on_their_way(load, store, "s_waitcnt vmcnt(1)", barrier) == [False] and on_their_way(store, load, "s_waitcnt vmcnt(1)", barrier) == [True]
    assert on_their_way(store, "s_cbranch_scc0 .L1", load, ".L1:", "s_waitcnt lgkmcnt(0)", barrier) == [True]
    assert on_their_way(".L1:", barrier, load, "s_branch .L1") == [True] and on_their_way(".L1:", "s_waitcnt vmcnt(0)", barrier, load, "s_branch .L1") == [False]


def test_the_loops_themselves():
    many = ["global_load_lds_dwordx4 x"] + ["v_mfma x"] * 20
    body = [".L0:", ".L1:"] + many + ["s_cbranch_scc1 .L1", ".L2:"] + many + ["v_readlane x", "s_branch .L2", ".L3:", "v_mfma x", "s_branch .L3", "s_cbranch_scc0 .L0"]
    assert sorted(_loops(body)) == [(1, 23), (24, 47)]


def test_reads_and_transfers_are_over_at_barriers(bodies):
    for name, body in bodies.items():
        reads = _outstanding(body)
        assert len(reads) >= 2 and not any(reads.values()), (name, reads)
        assert any("load_lds" in line for _, line in body)
        on_their_way = _transfers(body)
        assert not any(on_their_way.values()), (name, on_their_way)


def test_no_scalar_comes_back_in_the_tiles_loop_over_keys(bodies):
    for name, body in bodies.items():
        lines = [line for _, line in body]
        assert _loops(lines), name
        for first, last in _loops(lines):
            assert _reloads(lines, lines[first:last]) == 0, (name, first, last)
