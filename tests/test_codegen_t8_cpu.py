"""What the compiled kernels of the 8-bit layers with a scale for each token must keep that no run shows reliably."""
import os
import re
import subprocess

import pytest

from test_codegen_cpu import LLVM, PKG, _code_objects, _resources

LIB = os.path.join(PKG, "libqc.so")


def test_nothing_but_the_loads_to_lds_writes_their_address_register(tmp_path):
    """The products' loads go straight to LDS at the address in m0, which their inline assembly sets and cannot name as overwritten."""
    if not os.path.exists(LLVM + "llvm-objdump"):
        pytest.skip("no llvm-objdump")
    seen = 0
    for obj in _code_objects(LIB, str(tmp_path)):
        text = subprocess.run([LLVM + "llvm-objdump", "-d", "--mcpu=gfx950", "--symbolize-operands", "--no-show-raw-insn", "--no-leading-addr", obj],
                              check=True, stdout=subprocess.PIPE, text=True).stdout
        for part in re.split(r"^(?=<_Z\w+>:)", text, flags=re.M)[1:]:
            name, _, body = part.partition("\n")
            if "t8_tile_kernel" not in name and "t8_few_kernel" not in name:
                continue
            lines = [l.strip() for l in body.splitlines()]
            loads = [i for i, l in enumerate(lines) if l.startswith("global_load_lds_dwordx4")]
            assert loads
            assert all(l.startswith("s_mov_b32 m0,") for l in lines if re.search(r"\bm0\b", l)), name
            assert all(lines[i - 1].startswith("s_nop 0") and lines[i - 2].startswith("s_mov_b32 m0,") for i in loads), name
            seen += 1
    assert seen >= 9


def test_no_register_goes_to_scratch_memory(tmp_path):
    if not os.path.exists(LLVM + "llvm-readobj"):
        pytest.skip("no llvm-readobj")
    seen = 0
    for obj in _code_objects(LIB, str(tmp_path)):
        for name, (_, _, scratch) in _resources(obj).items():
            if re.match(r"_ZN2qc\d+t8_", name):
                seen += 1
                assert scratch == 0, (name, scratch)
    assert seen >= 60
