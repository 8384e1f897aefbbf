"""Loads from memory to LDS (csrc/attend.h) as they are built: the wait states that the hardware asks for.  No GPU needed."""
import os
import re
import subprocess

from paper_2202_01085_amd import build

# values that differ from lane to lane on paper, so that every scalar operand comes from a v_readfirstlane right before the load
SOURCE = """
#include "attend.h"
extern "C" __global__ void probe(const char *p, const int *from, int stride, float *out) {
    __shared__ __attribute__((aligned(1024))) short t[8192];
    const int w = from[threadIdx.x], x = from[threadIdx.x + 64], y = from[threadIdx.x + 128];
    const u32x4 buffer = buffer_of(p + w, x);
    to_lds(buffer, 16 * threadIdx.x, lds_address(t) + 1024 * (w & 1));
    to_lds(buffer, 16 * threadIdx.x + stride, lds_address(t) + 1024 * (x & 1));
    to_lds(p + 16 * threadIdx.x, lds_address(t) + 1024 * (y & 1));
    word_to_lds((const float *)p + threadIdx.x, lds_address(t) + 1024 * (from[threadIdx.x + 192] & 1));
    arrived();
    __syncthreads();
    out[threadIdx.x] = t[threadIdx.x];
}
""".replace("#include \"attend.h\"\n", "#include \"attend.h\"\nusing namespace f3m;\n")


def scalars(text):
    """numbers of the scalar registers that operands name"""
    got = set()
    for one, lo, hi in re.findall(r"\bs(\d+)\b|\bs\[(\d+):(\d+)\]", text):
        got |= {int(one)} if one else set(range(int(lo), int(hi) + 1))
    return got


def check(assembly):
    """(loads to LDS, faults) of an assembly listing: wait states counted back from each load, in one run of instructions"""
    states = []         # of each instruction so far: what it writes (a set of scalar registers, "m0"), by a vector unit or not, its states
    loads, faults = 0, []
    for line in assembly.splitlines():
        line = line.split(";")[0].split("//")[0].strip()
        if re.match(r"^[\w.$]+:", line):       # a label: what comes before is not known; its instructions stay, as they fall through
            continue
        m = re.match(r"([sv]_\w+|ds_\w+|global_\w+|buffer_\w+|flat_\w+)\s*(.*)", line)
        if not m:
            continue
        op, rest = m.groups()
        if re.match(r"(buffer|global)_load_(lds_\w+|\w+.*\blds\b)", line):
            loads += 1
            since = 0
            reads = scalars(rest)
            for name, writes, count in reversed(states):
                if since < 1 and "m0" in writes:
                    faults.append("m0: " + line)
                if since < 5 and name.startswith("v_") and writes & reads:
                    faults.append("%s: %s" % (name, line))
                since += count
                if since >= 5:
                    break
        first = rest.split(",")[0]
        writes = {"m0"} if first.strip() == "m0" else scalars(first) if op.startswith(("s_", "v_")) and not op.startswith(("s_waitcnt", "s_nop", "s_cbranch", "s_cmp")) else set()
        states.append((op, writes, int(rest) + 1 if op == "s_nop" else 1))
    return loads, faults


def test_the_check_itself():
    assert check("s_mov_b32 m0, s3\n buffer_load_dwordx4 v6, s[4:7], s2 offen lds")[1]
    assert check("s_mov_b32 m0, s3\n global_load_lds_dword v[8:9], off")[1]
    assert check("v_readfirstlane_b32 s5, v5\n s_mov_b32 m0, s3\n s_nop 2\n buffer_load_dwordx4 v6, s[4:7], s2 offen lds")[1]
    assert check("v_readfirstlane_b32 s2, v5\n s_mov_b32 m0, s3\n s_nop 2\n buffer_load_dwordx4 v6, s[4:7], s2 offen lds")[1]
    assert check("v_readfirstlane_b32 s5, v5\n s_mov_b32 m0, s3\n s_nop 3\n buffer_load_dwordx4 v6, s[4:7], s2 offen lds") == (1, [])
    assert check("s_add_i32 m0, s3, 4\n v_add_u32 v1, v2, v3\n global_load_lds_dwordx4 v[8:9], off") == (1, [])


def test_waits_before_loads_to_lds(tmp_path):
    src, out = str(tmp_path / "probe.hip"), str(tmp_path / "probe.s")
    with open(src, "w") as f:
        f.write(SOURCE)
    res = subprocess.run([build._hipcc(), *build.FLAGS, "-I", build.CSRC, "-S", "--cuda-device-only", src, "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    with open(out) as f:
        text = f.read()
    loads, faults = check(text)
    assert loads == 4 and not faults, faults
    # what is checked against the buffer's bytes is the lane's offset: all of it stands there, none in a scalar register
    assert re.findall(r"buffer_load_dwordx4 v\d+, s\[\d+:\d+\], (\S+) offen lds", text) == ["0", "0"]


def test_no_other_way_to_lds():
    """every load to LDS of the sources is one of those that the probe holds"""
    for name in os.listdir(build.CSRC):
        with open(os.path.join(build.CSRC, name)) as f:
            text = re.sub(r"//.*", "", f.read())
        assert len(re.findall(r"load_lds_dword|offen lds", text)) == (3 if name == "attend.h" else 0), name
        assert "load_lds(" not in text, name
