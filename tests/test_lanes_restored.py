"""In the built kernels no vector register is written at a place that a branch reaches with no lane on, ahead of the instruction that turns
the lanes on again: such a write does nothing, and what it should have kept is lost.  The compiler has put moves of live values there
(a backward pass out of registers, behind a condition that was the same for all lanes but written in the lanes' registers)."""
import os
import re
import subprocess

import pytest

from paper_2603_09237_amd import binding
from test_kernel_resources import code_objects

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def places(listing):
    """[(kernel, address, instructions)] of writes ahead of the lanes' return in a disassembly."""
    found, kernel, code = [], None, []

    def look():
        at = {a: i for i, (a, _) in enumerate(code)}
        reached, starts = set(), set()   # by a branch without lanes; by any branch
        for a, s in code:
            m = re.match(r"s_c?branch\w* (\d+)", s)
            if m:
                d = int(m.group(1))
                to = a + 4 + 4 * (d - 65536 if d >= 32768 else d)
                starts.add(to)
                if s.startswith("s_cbranch_execz"):
                    reached.add(to)
        for a in reached:
            hits = []
            for b, s in code[at[a]:at[a] + 200] if a in at else []:
                if b != a and b in starts:   # the next block: the lanes that run it have come from elsewhere too
                    break
                if re.match(r"s_or_b64 exec, exec,|s_mov_b64 exec|s_andn2_saveexec|s_or_saveexec", s):
                    if hits:
                        found.append((kernel, a, hits))
                    break
                if s.startswith(("s_branch", "s_cbranch", "s_endpgm")):
                    break
                if re.match(r"(v_(?!writelane|readlane|readfirstlane|cmp)|scratch_|buffer_|global_|ds_)", s):
                    hits.append(s)

    for line in listing.splitlines():
        m = re.match(r"^[0-9a-f]+ <(.+)>:", line)
        if m:
            look()
            kernel, code = m.group(1), []
            continue
        m = re.match(r"^\s+(\S.*?)\s*// ([0-9A-F]+):", line)
        if m:
            code.append((int(m.group(2), 16), m.group(1)))
    look()
    return found


def test_the_reading_itself():
    ahead = "0 <k>:\n\ts_cbranch_execz 1  // 000000000000: BF\n\tv_mov_b32_e32 v1, v2 // 000000000004: 7E\n" \
            "\tv_accvgpr_write_b32 a1, v2 // 000000000008: D3\n\ts_or_b64 exec, exec, s[0:1] // 000000000010: 87\n"
    assert [p[1:] for p in places(ahead)] == [(8, ["v_accvgpr_write_b32 a1, v2"])]
    assert places(ahead.replace("v_accvgpr_write_b32 a1, v2", "v_writelane_b32 v1, s2, 3")) == []


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_no_write_ahead_of_the_lanes_return(tmp_path):
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_09237_amd import build
        build.build(verbose=False)
    kernels = 0
    for i, elf in enumerate(code_objects(open(binding.LIB_PATH, "rb").read())):
        path = tmp_path / f"{i}.co"
        path.write_bytes(elf)
        r = subprocess.run([OBJDUMP, "-d", str(path)], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr
        kernels += len(re.findall(r"^[0-9a-f]+ <.+>:", r.stdout, re.M))
        assert places(r.stdout) == []
    assert kernels > 100
