"""The checks of the built library's code reach the kernels of the biased gate and of the 4-bit calls: their copies to LDS keep the wait
states, and none of them uses private scratch."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2602_21140_amd import build
from test_copy_wait_states_cpu import OBJDUMP, WRITES_M0, late_base
from test_no_private_scratch_cpu import LLVM

KERNELS = ("route_biased_kernel", "route_biased_rows_kernel", "dispatch_place_kernel", "mx_quantize_kernel", "mx_dequantize_kernel", "mx_pack_kernel",
           "mx_stream_kernel", "mx_tile_kernel")


def code_objects(tmp_path):
    if not os.path.exists(build.LIB_PATH):
        build.build(verbose=False)
    lib = shutil.copy(build.LIB_PATH, tmp_path)  # the code objects are written beside the file
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True, cwd=tmp_path)
    return sorted(tmp_path.glob("*gfx950*"))


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_copies_of_the_4_bit_tiles(tmp_path):
    where, history, copies = "", [], {}
    for obj in code_objects(tmp_path):
        r = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(obj)], check=True, capture_output=True, text=True)
        for line in r.stdout.splitlines():
            text = line.split("//")[0].strip()
            if text.startswith("<") and text.endswith(">:"):
                where, history = text[1:-2], []
            elif text:
                if "mx_tile_kernel" in where and "global_load_lds" in text:
                    copies[where] = copies.get(where, 0) + 1
                    assert not (history and WRITES_M0.match(history[-1])) and not late_base(history, text), (where, history, text)
                history = history[-7:] + [text]
    # both products; at least the prologue's copies and those of a step each
    assert len(copies) == 2 and min(copies.values()) >= 20, copies


@pytest.mark.skipif(not os.path.exists(os.path.join(LLVM, "llvm-readelf")), reason="no llvm-readelf")
def test_no_private_scratch(tmp_path):
    found = {}
    for obj in code_objects(tmp_path):
        notes = subprocess.run([os.path.join(LLVM, "llvm-readelf"), "--notes", str(obj)], check=True, capture_output=True, text=True).stdout
        names = re.findall(r"^\s*\.name:\s+(_Z\S+)", notes, re.M)
        sizes = [int(n) for n in re.findall(r"\.private_segment_fixed_size:\s+(\d+)", notes)]
        assert len(names) == len(sizes)
        found.update(zip(names, sizes))
    for kernel in KERNELS:
        sizes = [s for n, s in found.items() if kernel in n]
        assert sizes and not any(sizes), kernel
