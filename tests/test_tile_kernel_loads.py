"""Host-only: the grouped product's tile kernels count the loads to LDS that are in flight.  A load to a register between them would be waited
for together with all of these and with a tile's stores, so there is none once the first load to LDS has gone out."""
import os
import re
import shutil
import subprocess

import pytest

from test_kernel_resources import LIB, _code_objects

OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
@pytest.mark.parametrize("kernel", ["tile_matmul_kernel", "ring_matmul_kernel"])
def test_no_load_to_registers_behind_the_first_to_lds(kernel, tmp_path):
    if not os.path.exists(LIB):
        pytest.fail(f"{LIB} not built (run __graft_entry__.build())")
    with open(LIB, "rb") as f:
        data = f.read()
    seen = 0
    for i, elf in enumerate(_code_objects(data)):
        if kernel.encode() not in elf:
            continue
        path = tmp_path / f"{i}.co"
        path.write_bytes(elf)
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
        for name, body in re.findall(r"<(\S+)>:\n(.*?)(?=\n\n|\Z)", text, re.S):
            if kernel not in name or "global_load_lds" not in body:
                continue
            seen += 1
            behind = body[body.index("global_load_lds"):]
            found = [l.split("//")[0].strip() for l in behind.splitlines() if re.search(r"\b(global|flat|buffer|scratch)_load_(?!lds)", l)]
            assert not found, (name, found)
    assert seen, "no such kernel in the library"
