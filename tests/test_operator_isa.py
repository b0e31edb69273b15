"""Host-side check of what the compiler made of the walks behind shared prefixes: they are the prefill kernel's and the small decode kernel's, and
keep what those live on: no scratch memory, no wait in a step that is not written there, registers for two waves a SIMD."""
import re

from test_kernel_isa import device_assembly, innermost_mfma_loops, kernel_body


def check(asm, name):
    insn, labels, _ = kernel_body(asm, name)
    assert not any(t.startswith("scratch_") for t in insn), name
    vg = [int(x) for x in re.findall(r"\.name:\s+\S*" + name + r"\S*\s*\n(?:.*\n){0,40}?\s+\.vgpr_count:\s+(\d+)", asm)]
    private = re.findall(r"\.name:\s+\S*" + name + r"\S*\s*\n(?:.*\n){0,3}?\s+\.private_segment_fixed_size:\s+(\d+)", asm)
    assert vg and max(vg) <= 256 and set(private) == {"0"}, (name, vg, private)
    return insn, labels


def test_prefix_sums():
    asm = device_assembly("prefix_kernels.hip")
    for d, dtype, meet in ((128, 0, 2), (64, 0, 2), (128, 1, 4), (64, 1, 4)):
        insn, labels = check(asm, f"13k_prefix_sumsILi{d}ELi{dtype}ELi{meet}E")
        loops = innermost_mfma_loops(insn, labels, min_mfma=3 * d // 16)
        steps = [(a, b) for a, b in loops if insn[a:b].count("s_barrier") == 1]
        assert len(steps) == 2, (d, dtype, loops)                   # of the prefixes: without masks, and the last pair
        for a, b in steps:
            seg = insn[a:b]
            assert sum(t.startswith("v_mfma") for t in seg) == 3 * d // 16      # scores, probabilities' high and low halves
            full = [t for t in seg if t.startswith("s_waitcnt") and "vmcnt(0)" in t]
            assert len(full) <= (3 if dtype == 0 else 5), (d, dtype, full)


def test_prefixed_prefill_and_small_calls():
    asm = device_assembly("prefill_kernels.hip")
    for d, dtype, meet in ((128, 0, 2), (64, 0, 2), (128, 1, 4), (64, 1, 4)):
        insn, labels = check(asm, f"18k_prefill_prefixedILi{d}ELi{dtype}ELi{meet}E")
        assert len(innermost_mfma_loops(insn, labels, min_mfma=3 * d // 16)) == 2
    asm = device_assembly("prefix_kernels.hip")
    for d, dtype in ((128, 0), (64, 0), (128, 1), (64, 1)):
        check(asm, f"20k_attention_prefixedILi{d}ELi{dtype}E")
