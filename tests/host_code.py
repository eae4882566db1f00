"""Parts of a kernel's source that compute nothing but numbers, compiled for the CPU as they stand."""
import os
import re
import subprocess

from paper_2407_02891_amd import build as hip_build

HEAD = """
#include <cstdio>
#include <cstdlib>
#include <algorithm>
#define __device__
#define __forceinline__ inline
using std::max;
using std::min;
typedef long long i64;
struct { unsigned x; } threadIdx;
#define CHECK(...) do { if (!(__VA_ARGS__)) { std::printf("line %d: " #__VA_ARGS__ "\\n", __LINE__); std::exit(1); } } while (0)
"""


def part(source, begins):
    """The definition in a file of csrc/ that has a line which begins so (its template<> line too), up to its closing brace in the first column."""
    text = open(os.path.join(hip_build.CSRC, source)).read()
    found = re.findall(rf"^((?:template <[^\n]*\n)?{re.escape(begins)}.*?^}};?\n|constexpr [^\n]*{re.escape(begins)}[^\n]*;[^\n]*\n)", text, re.M | re.S)
    assert len(found) == 1, (source, begins, len(found))
    return found[0]


def run(folder, *code):
    """What a program of these parts prints; a CHECK that fails ends it."""
    source, program = str(folder / "program.cpp"), str(folder / "program")
    with open(source, "w") as f:
        f.write(HEAD + "\n".join(code))
    # (-fwrapv: what the GPU does with a sum beyond 32 bits)
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-fwrapv", source, "-o", program], check=True)
    done = subprocess.run([program], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stdout + done.stderr
    return done.stdout
