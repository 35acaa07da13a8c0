"""Loads to LDS take their place there from m0, which inline assembly writes: the compiler is told so, and nothing of what it
makes of such kernels depends on m0 across one."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2411_03357_amd as pgcm
from test_kernel_scratch import _code_objects, _kernels

CSRC = os.path.join(os.path.dirname(os.path.abspath(pgcm.__file__)), "csrc")
OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"


def test_assembly_that_writes_m0_names_it():
    seen = 0
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".hip", ".h")):
            continue
        text = open(os.path.join(CSRC, name)).read()
        for statement in re.findall(r"\basm\b(?:\s+volatile)?\s*\((.*?)\);", text, flags=re.S):
            if re.search(r"\bm0\b", statement):
                assert '"m0"' in statement.rsplit(":", 1)[-1], (name, statement)
                seen += 1
    assert seen >= 1


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_m0_is_written_right_before_each_use(tmp_path):
    with open(pgcm.library_path(), "rb") as f:
        image = f.read()
    seen = 0
    for n, elf in enumerate(_code_objects(image)):
        names = [k[".name"] for k in _kernels(elf) if "many_kernel" in k[".name"]]
        if not names:
            continue
        path = tmp_path / ("object_%d" % n)
        path.write_bytes(elf)
        out = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--disassemble-symbols=" + ",".join(names), str(path)],
                             stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
        assert out.returncode == 0, out.stderr[-500:]
        for kernel in re.split(r"^[0-9a-f]+ <", out.stdout, flags=re.M)[1:]:
            name, code = kernel.split(">:", 1)
            code = [line.split("//")[0].strip() for line in code.splitlines()]
            code = [line for line in code if line]
            for i, line in enumerate(code):
                if re.search(r"\bm0\b", line):
                    assert re.match(r"s_mov_b32 m0, s\d+$", line), (name, line)
                    assert code[i + 1] == "s_nop 0" and code[i + 2].startswith("global_load_lds_dwordx4 "), (name, code[i:i + 3])
                    seen += 1
            assert sum(line.startswith("global_load_lds") for line in code) == sum(line.startswith("s_mov_b32 m0") for line in code), name
    assert seen >= 24, seen      # of two types, three widths, exact or not, cut or not
