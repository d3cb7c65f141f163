"""What the hand-written assembly of the cross entropy's products relies on and the compiler does not know, looked up in the built library.

Loads into LDS set m0 (the bytes' place), which assembly cannot name as overwritten: no other instruction of these kernels may use it.  Products of the
256 x 256 tiles write accumulation registers behind the compiler's back: it may neither move these registers in between nor read them at once.
"""
import os
import re
import shutil
import subprocess

import pytest

import paper_2407_00243_amd as tf
from paper_2407_00243_amd import build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
# instructions that read m0 without naming it
READS_M0 = ("s_sendmsg", "s_movrel", "v_movrel", "ds_gws", "ds_ordered", "s_ttracedata", "global_load_lds", "ds_read_addtid", "ds_write_addtid", "v_interp")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    tf.load_library()
    folder = tmp_path_factory.mktemp("code")
    library = shutil.copy(build.LIB, folder)
    subprocess.run([OBJDUMP, "--offloading", library], cwd=folder, check=True, capture_output=True)
    out = {}
    for name in sorted(os.listdir(folder)):
        path = os.path.join(folder, name)
        with open(path, "rb") as f:
            if "gfx950" not in name or b"k_product" not in f.read():
                continue
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]{16} <)", text):
            head = re.match(r"[0-9a-f]{16} <(\S*k_product\S*)>:", part)
            if head:
                out[head[1]] = [line.split("//")[0].strip() for line in part.split("\n")[1:] if line.startswith("\t")]
    # 3 element types; 16-bit ones with tiles of four sizes
    assert len(out) >= 40
    return out


def test_nothing_else_uses_m0(kernels):
    loads = 0
    for name, code in kernels.items():
        for i, line in enumerate(code):
            assert not line.startswith(READS_M0), f"{name}: {line}"
            if re.search(r"\bm0\b", line):
                assert re.match(r"s_add_u32 m0, s\d+, ", line) and code[i + 1] == "s_nop 0" and re.match(r"buffer_load_dwordx4 .* lds$", code[i + 2]), \
                    f"{name}: {code[i:i + 3]}"
                loads += 1
            if re.search(r"\blds$", line):
                assert code[i - 2].startswith("s_add_u32 m0,"), f"{name}: {line}"
    assert loads


def test_sums_in_accumulation_registers_are_left_alone(kernels):
    large = {name: code for name, code in kernels.items() if "Li8ELi8E" in name}
    assert large
    for name, code in large.items():
        behind = None       # what came last: a product, or the wait behind the last of them
        reads = 0
        for i, line in enumerate(code):
            if line.startswith("v_mfma"):
                assert "accvgpr_write" not in code[i - 1] + code[i - 2], f"{name}: {code[i - 2:i + 1]}"
                behind = "product"
            elif line == "s_nop 15" and code[i - 1] == "s_nop 15":
                behind = "wait"
            elif line.startswith("v_accvgpr_read"):
                assert behind == "wait", f"{name}: {code[i - 5:i + 1]}"
                reads += 1
            else:
                # zeros at first; nothing is moved, spilled or stored from there
                assert not line.startswith("v_accvgpr") or re.match(r"v_accvgpr_write_b32 a\d+, 0$", line), f"{name}: {line}"
                assert not (line.startswith(("scratch_", "global_store", "ds_write", "v_mov")) and re.search(r"\ba(\d+|\[)", line)), f"{name}: {line}"
        assert reads >= 256, name
