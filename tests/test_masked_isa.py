"""Host-side check of what the compiler made of the walks under masks: no scratch memory, registers for two waves a SIMD (for three where heads are 64 wide and
come in groups of 128 columns), and one inner loop without masks that meets once."""
import re

import pytest

from test_kernel_isa import device_assembly, innermost_mfma_loops
from test_operator_isa import check


def vgprs(asm, name):
    return [int(x) for x in re.findall(r"\.name:\s+\S*" + name + r"\S*\s*\n(?:.*\n){0,40}?\s+\.vgpr_count:\s+(\d+)", asm)]


@pytest.fixture(scope="module")
def asm():
    return device_assembly("mask_kernels.hip")


def test_window_decode(asm):
    for d, dtype in ((128, 0), (64, 0), (128, 1), (64, 1)):
        check(asm, f"15k_window_decodeILi{d}ELi{dtype}E")


def test_units(asm):
    for d, dtype in ((128, 0), (64, 0), (128, 1), (64, 1)):
        for tiles in (1, 2):
            check(asm, f"8k_maskedILi{d}ELi{dtype}ELi{tiles}E")
        assert max(vgprs(asm, f"8k_maskedILi64ELi{dtype}ELi1E")) <= 128            # (four waves a SIMD)


def test_groups(asm):
    for d, dtype, meet in ((128, 0, 2), (64, 0, 2), (128, 1, 2), (64, 1, 2), (128, 1, 4), (64, 1, 4)):
        name = f"13k_masked_wideILi{d}ELi{dtype}ELi{meet}E"
        insn, labels = check(asm, name)
        if d == 64:
            assert max(vgprs(asm, name)) <= 168
        plain = [insn[a:b] for a, b in innermost_mfma_loops(insn, labels, min_mfma=3 * d // 16) if insn[a:b].count("s_barrier") == 1]
        assert any(sum(t.startswith("v_mfma") for t in x) == 3 * d // 16 for x in plain), (d, dtype)
