"""m0, the LDS address of a copy into LDS, through code that has copies of both
kinds (pask_latent_device.h): the compiler's, whose settings of m0 it merges,
and those in asm, which it cannot see set it.  The assembly of
tests/native/lds_copies.hip is followed instruction by instruction."""

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC) and shutil.which("hipcc") is None, reason="no hipcc")
def test_copies_in_asm_leave_m0_as_it_was(tmp_path):
    asm = tmp_path / "lds_copies.s"
    b = subprocess.run([HIPCC, "-O3", "-std=c++17", "--offload-arch=gfx950", "--cuda-device-only", "-S",
                        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", f"-I{ROOT}/include",
                        f"-I{ROOT}/paper_2608_28276_amd/csrc", f"{ROOT}/tests/native/lds_copies.hip", "-o", str(asm)],
                       capture_output=True, text=True, timeout=300)
    assert b.returncode == 0, b.stderr[-4000:]
    copies = {True: 0, False: 0}                      # in asm, the compiler's
    m0 = owner = None                                 # what m0 holds and who set it last: the compiler's must be its own
    in_asm, held = False, {}
    for line in asm.read_text().splitlines():
        line = line.strip()
        if line.startswith(";;#ASM"):
            in_asm = line.startswith(";;#ASMSTART")
        if re.match(r"_Z\w+:", line):                 # a kernel starts
            m0, owner, held = "unset", None, {}
        if m := re.match(r"s_mov_b32 (s\d+), m0", line):
            held[m.group(1)] = (m0, owner)
        elif m := re.match(r"s_mov_b32 m0, (\w+)", line):
            m0, owner = held.pop(m.group(1), (m.group(1), in_asm))
        elif re.search(r"\bm0\b", line) and not line.startswith(";"):
            pytest.fail(f"m0 in an instruction that this test does not follow: {line}")
        elif line.startswith("global_load_lds_dwordx4"):
            copies[in_asm] += 1
            assert owner == in_asm, f"m0 of '{line}' was set by {'asm' if owner else 'the compiler'}"
    assert copies == {True: 2, False: 4}
