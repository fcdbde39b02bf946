"""The compiled kernels' hand-written loads into LDS and the wait states that they need. The compiler puts wait states in front of
its own instructions; of a hand-written one it sees neither that it reads a scalar base nor that it reads M0.

- A scalar register that a vector instruction has written (a base that was spilled into the lanes of a vector register) may be
  read as an address five wait states later.
- M0 that a scalar instruction has written may be read by a load into LDS one wait state later."""

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2504_09590_amd", "libbros_attn.so")
OBJDUMP = next((p for p in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump") or "") if os.path.exists(p)), None)


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    """The code objects of the built library."""
    if OBJDUMP is None or not os.path.exists(LIB):
        pytest.skip("no disassembler, or nothing is built")
    d = tmp_path_factory.mktemp("code")
    shutil.copy(LIB, d / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=d, check=True, capture_output=True)
    found = [d / f for f in sorted(os.listdir(d)) if "gfx950" in f]
    assert found
    return found


def test_loads_into_lds_stand_behind_their_wait_states(code):
    loads = 0
    for obj in code:
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(obj)], check=True, capture_output=True, text=True).stdout
        kernel = before = ""
        for line in text.splitlines():
            line = line.split("//")[0].strip()
            if not line:
                continue
            if line.endswith(">:"):
                kernel = line
            if re.match(r"(global|buffer|scratch)_load.*lds|buffer_load.* lds", line):
                loads += 1
                need = 1 if line.endswith(" off") else 5
                wait = re.fullmatch(r"s_nop (\d+)", before)
                assert wait and int(wait[1]) + 1 >= need, f"{kernel}: {line!r} behind {before!r}"
            before = line
    assert loads > 1000
