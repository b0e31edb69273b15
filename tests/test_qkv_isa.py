"""Host-side check of what the compiler made of the appends from the projections: no scratch memory, registers for four waves a SIMD."""
import re

from test_kernel_isa import device_assembly, kernel_body


def test_registers():
    asm = device_assembly("qkv_kernels.hip")
    names = [f"12k_qkv_appendILi{t}E" for t in (0, 1)] + [f"18k_qkv_append_chunkILi{d}ELi{t}ELi{n}E" for d in (64, 128) for t in (0, 1) for n in (127, 447)]
    for name in names:
        insn, _, _ = kernel_body(asm, name)
        assert not any(t.startswith("scratch_") for t in insn), name
        vg = [int(x) for x in re.findall(r"\.name:\s+\S*" + name + r"\S*\s*\n(?:.*\n){0,40}?\s+\.vgpr_count:\s+(\d+)", asm)]
        private = re.findall(r"\.name:\s+\S*" + name + r"\S*\s*\n(?:.*\n){0,3}?\s+\.private_segment_fixed_size:\s+(\d+)", asm)
        assert vg and max(vg) <= 128 and set(private) == {"0"}, (name, vg, private)
