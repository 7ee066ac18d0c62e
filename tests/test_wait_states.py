"""Wait states that the hardware asks of the program and the compiler does not add
inside or around inline assembly, looked for in the built library's own gfx950
code (no GPU):

- a load into LDS reads M0, and must not be the instruction after the scalar
  write of M0;
- a memory instruction must not read a scalar register within five wait states
  of the vector instruction that wrote it (readfirstlane and the like).
"""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

import paper_1911_08076_amd as P

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
LIB = os.path.join(os.path.dirname(P.__file__), "libifq.so")
SCALAR = re.compile(r"s\[\d+:\d+\]|\bs\d+\b|\bvcc\b")


def _numbers(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.fullmatch(r"s(\d+)", operand)
    return {int(m[1])} if m else ({"vcc"} if operand == "vcc" else set())


def _written(name, ops):
    """Scalar registers that a vector instruction writes."""
    if name.startswith(("v_readfirstlane", "v_readlane", "v_cmp")):
        return _numbers(ops[0])
    if "_co_" in name or name.startswith("v_div_scale"):
        return _numbers(ops[1])
    return set()


def faults(listing):
    """(loads into LDS seen, the places where a wait state is missing) of a listing."""
    bad, loads, kernel, before = [], 0, "", []
    for line in listing:
        head = re.match(r"<(.*)>:$", line)
        if head:
            kernel = kernel if head[1].startswith("L") else head[1]
            continue
        text = line.split("//")[0].strip()
        if not text:
            continue
        name, _, rest = text.partition(" ")
        ops = [o.strip() for o in rest.split(",")]
        if name.startswith(("global_", "buffer_", "flat_", "scratch_")):
            if "_lds_" in name or rest.endswith(" lds"):
                loads += 1
                if before and before[-1][0].startswith("s_") and before[-1][1][0] == "m0":
                    bad.append("%s: M0 written right before %s" % (kernel, text))
            reads = set().union(*[_numbers(o) for o in SCALAR.findall(rest)])
            waited = 0
            for n, o in reversed(before if reads else []):
                if waited >= 5:
                    break
                if n.startswith("v_") and _written(n, o) & reads:
                    bad.append("%s: %s %s, %d wait states before %s" % (
                        kernel, n, o[0], waited, text))
                waited += int(o[0]) + 1 if n == "s_nop" else 1
        before = before[-7:] + [(name, ops)]
    return loads, bad


def test_the_search_finds_what_it_is_for():
    ok = ["<k>:", "s_mov_b32 m0, s2", "s_nop 0", "global_load_lds_dwordx4 v1, s[4:5]"]
    assert faults(ok) == (1, [])
    assert len(faults(ok[:2] + ok[3:])[1]) == 1
    near = ["<k>:", "v_readfirstlane_b32 s5, v0", "s_nop 3", "global_load_dword v1, v0, s[4:5]"]
    assert len(faults(near)[1]) == 1
    assert faults(near[:2] + ["s_nop 4"] + near[3:]) == (0, [])
    assert len(faults(["v_cmp_lt_u32_e64 s[2:3], v0, v1",
                       "buffer_load_dword v1, v0, s[0:3], 0 offen"])[1]) == 1


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not found")
def test_wait_states_of_the_built_kernels(tmp_path):
    shutil.copy(LIB, tmp_path / "libifq.so")
    subprocess.run([OBJDUMP, "--offloading", "libifq.so"], cwd=tmp_path, check=True,
                   capture_output=True)
    objects = sorted(p for p in os.listdir(tmp_path) if p.endswith("gfx950"))
    assert objects

    def listing(name):
        r = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", name],
                           cwd=tmp_path, check=True, capture_output=True, text=True)
        return r.stdout.splitlines()

    with ThreadPoolExecutor(4) as ex:
        found = [faults(lines) for lines in ex.map(listing, objects)]
    assert sum(loads for loads, _ in found) > 0
    bad = [b for _, more in found for b in more]
    assert not bad, "%d missing, first: %s" % (len(bad), bad[:5])
