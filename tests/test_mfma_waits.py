"""Host-side check that no instruction reads or overwrites what a matrix product is still writing.

The chip does not wait by itself: between a product and the first other vector instruction that touches its result there have to be so many issue slots,
8 for the 16x16x32 products of the kernels and 12 for the 32x32x16 ones.  The compiler puts them in, but where two ways part behind
a product and meet again in front of the first reader it has been seen to count along one of them only, the longer one; the
shorter one then read a stale score.  So every way from every product is walked here."""
import re

import pytest

from test_kernel_isa import device_assembly

NEEDED = {"16x16": 8, "32x32": 12}
SOURCES = ["attn_kernels.hip", "prefill_kernels.hip", "prefix_kernels.hip", "mask_kernels.hip"]


def kernels(asm):
    """{name: (instructions as (mnemonic, operands), {label: index})} of an assembly listing."""
    found, name = {}, None
    for line in asm.split("\n"):
        line = line.split(";")[0].rstrip()
        m = re.match(r"^(_Z\w+):", line)
        if m:
            name, insn, labels = m.group(1), [], {}
            found[name] = insn, labels
        elif ".amdhsa_kernel" in line:
            name = None
        elif name:
            m = re.match(r"^(\.LBB\d+_\d+):", line)
            t = line.strip()
            if m:
                labels[m.group(1)] = len(insn)
            elif t and not t.startswith((".", "//")):
                mnemonic, _, rest = t.partition(" ")
                insn.append((mnemonic, [x.strip() for x in rest.split(",")]))
    return found


def registers(operand):
    m = re.match(r"^[-|]*([va])\[(\d+):(\d+)\]", operand)
    if m:
        return {(m.group(1), i) for i in range(int(m.group(2)), int(m.group(3)) + 1)}
    m = re.match(r"^[-|]*([va])(\d+)\b", operand)
    return {(m.group(1), int(m.group(2)))} if m else set()


def too_early(insn, labels):
    """(slots, product, instruction) of every instruction that touches a product's result before it may."""
    bad = []
    for i, (m, ops) in enumerate(insn):
        if not m.startswith("v_mfma"):
            continue
        needed = next(n for shape, n in NEEDED.items() if shape in m)
        seen, ways = {}, [(i + 1, 0, frozenset(registers(ops[0])))]
        while ways:
            j, slots, live = ways.pop()
            while j < len(insn) and slots < needed and live and seen.get(j, needed) > slots:
                seen[j] = slots
                name, args = insn[j]
                if name.startswith("v_mfma"):
                    live = live - registers(args[0])         # (products wait for products by rules of their own; this one's result is looked at from there)
                elif name.startswith(("v_", "buffer_", "global_", "ds_", "flat_", "scratch_")):
                    if any(registers(x) & live for x in args):
                        bad.append((slots, " ".join([m] + ops), " ".join([name] + args)))
                        break
                if name == "s_endpgm":
                    break
                slots += int(args[0]) + 1 if name == "s_nop" else 1
                if name == "s_branch":
                    j = labels[args[0]]
                    continue
                if name.startswith("s_cbranch"):
                    ways.append((labels[args[0]], slots, live))
                j += 1
    return bad


@pytest.mark.parametrize("source", SOURCES)
def test_results_are_waited_for(source):
    found = kernels(device_assembly(source))
    assert sum(m.startswith("v_mfma") for insn, _ in found.values() for m, _ in insn) > 100
    for name, (insn, labels) in found.items():
        assert not too_early(insn, labels), (name, too_early(insn, labels)[:3])


def test_the_check_sees_both_ways():
    """Two ways that meet: eight slots along one, two along the other."""
    asm = "\n".join(["_Zk:", "v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0", "s_cbranch_vccnz .LBB0_1", "s_nop 7", ".LBB0_1:", "s_nop 0", "v_mul_f32_e32 v9, s0, v2"])
    bad = too_early(*kernels(asm)["_Zk"])
    assert [x[0] for x in bad] == [2]
    assert not too_early(*kernels(asm.replace("s_nop 0", "s_nop 6"))["_Zk"])
