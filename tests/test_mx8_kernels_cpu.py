"""The checks of the built library's code reach the kernels of the norm and of the 8-bit calls: the tiles' copies to LDS keep the wait
states, none of the kernels uses private scratch, and the library's host code refuses what it cannot take without a GPU."""
import os
import re
import subprocess

import pytest

from paper_2602_21140_amd import binding
from test_copy_wait_states_cpu import OBJDUMP, WRITES_M0, late_base
from test_mx_kernels_cpu import code_objects
from test_no_private_scratch_cpu import LLVM

KERNELS = ("add_rms_norm_kernel", "add_rms_norm_long_kernel", "mx8_quantize_kernel", "mx8_dequantize_kernel", "mx8_pack_kernel", "mx8_stream_kernel",
           "mx8_tile_kernel")


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_copies_of_the_8_bit_tiles(tmp_path):
    where, history, copies = "", [], {}
    for obj in code_objects(tmp_path):
        r = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(obj)], check=True, capture_output=True, text=True)
        for line in r.stdout.splitlines():
            text = line.split("//")[0].strip()
            if text.startswith("<") and text.endswith(">:"):
                where, history = text[1:-2], []
            elif text:
                if "mx8_tile_kernel" in where and "global_load_lds" in text:
                    copies[where] = copies.get(where, 0) + 1
                    assert not (history and WRITES_M0.match(history[-1])) and not late_base(history, text), (where, history, text)
                history = history[-7:] + [text]
    # two widths of the linear product's, two epilogues of the FFN's, scales by words or not; at least the prologue's copies and those of a step each
    assert len(copies) == 8 and min(copies.values()) >= 18, copies


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


def test_host_checks_without_a_gpu():
    """Every refusal comes before the first thing that needs a device; the addresses are never followed."""
    L, p = binding.lib(), 1 << 20
    assert L.revive_mx_eight_linear(p, p, 1 << 30, 32, p, 1 << 26, None, 0, None, 0, p, 1 << 26, None) == -1 and b"one launch" in L.revive_last_error(None)
    assert L.revive_mx_eight_linear(p, p, (1 << 30) + 1, 32, p, 32, None, 0, None, 0, p, 32, None) == -1
    # rows longer than the kernels' 32-bit offsets reach across a tile
    assert L.revive_mx_eight_linear(p, p, 16, (1 << 24) + 32, p, 7, None, 0, None, 0, p, 7, None) == -1 and b"2^24" in L.revive_last_error(None)
    with pytest.raises(binding.ReviveError):
        binding.mx8_packed_bytes(7, (1 << 24) + 32)
    assert binding.mx8_packed_bytes(7, 1 << 24) == (1 << 24) * 132
    assert L.revive_mx_eight_linear(p, p, 0, 32, p, 32, None, 0, None, 0, p, 32, None) == 0
    assert L.revive_add_rms_norm(p, None, p, 1, 0, 64, 64, 0, 1e-6, None, p, None, None, None) == 0
    assert L.revive_add_rms_norm(p, None, p, 1, 4, 64, 64, 0, 1e-6, p, p + 4096, None, None, None) == -1  # a sum without a residual
    assert L.revive_mx_eight_quantize(p, 1, 0, 64, 64, p, p, None) == 0 and L.revive_mx_eight_dequantize(p, p, 0, 64, 1, p, 64, None) == 0
    assert binding.mx8_packed_bytes(1, 32) == 128 * 132 and binding.mx8_packed_bytes(129, 160) == 2 * 128 * 2 * 132
    with pytest.raises(binding.ReviveError):
        binding.mx8_packed_bytes(1 << 20, 1 << 12)


def test_public_names():
    import paper_2602_21140_amd as package
    from paper_2602_21140_amd import binding as calls
    names = [n for n in vars(package) if n.startswith("mx8_") or n == "add_rms_norm"]
    assert len(names) == 6 and all(n in package.__all__ and getattr(package, n) is getattr(calls, n) for n in names)
    assert all(hasattr(package, n) for n in package.__all__)
