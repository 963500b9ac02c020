"""No instruction of the built window attention kernels reads a matrix instruction's result before it is there.

A 32x32x16 bf16 product's registers may be read by an ordinary instruction twelve issue slots behind it: so many the compiler leaves within straight code.
Where a conditional branch lies between the two, it has been seen not to (a wrong gradient, different from run to run), so the kernels keep
branches away from there, and this reads the code that was built from them: every path from every such product, over its branches."""
import re

import pytest

from tests.test_abi_host import code_objects

WAIT = 12


def registers(text):
    found = set()
    for kind, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        found |= {kind + str(i) for i in range(int(a), int(b) + 1)}
    return found | {kind + n for kind, n in re.findall(r"\b([va])(\d+)\b", text)}


def functions(listing):
    """(name, [(mnemonic, operands)], {index: target's index}) of each function of a disassembly."""
    for m in re.finditer(r"^([0-9a-f]+) <(\S+)>:\n(.*?)(?=^\S|\Z)", listing, re.S | re.M):
        start, name, code, index, jumps = int(m.group(1), 16), m.group(2), [], {}, {}
        for line in m.group(3).splitlines():
            text, _, note = line.partition("//")
            if not text.strip() or not note:  # (the space behind the last instruction is left out)
                continue
            index[int(note.split(":")[0], 16)] = len(code)
            op, _, args = text.strip().partition(" ")
            if op.startswith("s_cbranch") or op == "s_branch":
                jumps[len(code)] = start + int((re.search(r"\+0x([0-9a-f]+)>", note) or [0, "0"])[1], 16)
            code.append((op, args.strip()))
        yield name, code, {i: index[a] for i, a in jumps.items()}


def reads(op, args):
    parts = re.split(r",\s*(?![^\[]*\])", args)
    if op.startswith(("ds_write", "ds_add", "global_store", "buffer_store", "scratch_store")) or "swap" in op:
        return registers(args)
    return registers(",".join(parts[1:]))


def too_early(code, jumps):
    """(product, reader, wait states between) wherever there are too few."""
    found = []
    for i, (op, args) in enumerate(code):
        if not op.startswith("v_mfma"):
            continue
        result = registers(args.split("]")[0] + "]")
        paths, seen = [(i + 1, 0)], {}
        while paths:
            j, waited = paths.pop()
            while j < len(code) and waited < WAIT and seen.get(j, WAIT) > waited:
                seen[j] = waited
                op2, args2 = code[j]
                if op2 == "s_endpgm":
                    break
                if op2 == "s_nop":
                    waited += int(args2, 0)
                elif op2 == "s_branch":
                    j, waited = jumps[j], waited + 1
                    continue
                elif j in jumps:
                    paths.append((jumps[j], waited + 1))
                elif op2.startswith("v_mfma"):
                    to, a, b, c = re.split(r",\s*(?![^\[]*\])", args2)[:4]
                    if registers(a + "," + b) & result:
                        found.append((args, op2 + " " + args2, waited))
                        break
                    if registers(c) & result:
                        break  # the same sums go on: handed over inside the unit
                    waited += 7  # (the unit takes one product in eight)
                elif op2.startswith(("v_", "ds_", "global_", "buffer_", "scratch_")) and reads(op2, args2) & result:
                    found.append((args, op2 + " " + args2, waited))
                    break
                j, waited = j + 1, waited + 1
    return found


def test_a_listing_with_and_without_the_fault():
    def listing(*lines):
        return "0000000000000100 <kernel>:\n" + "".join(f"\t{t:60s}// {0x100 + 4 * i:012X}: 00000000{n}\n" for i, (t, n) in enumerate(lines))

    product, end = ("v_mfma_f32_32x32x16_bf16 v[0:15], v[16:19], v[20:23], 0", ""), ("s_endpgm", "")
    read = ("v_add_f32_e32 v30, v31, v5", "")
    cases = [([product, ("s_nop 11", ""), read, end], 0),
             ([product, ("s_nop 10", ""), read, end], 1),
             ([product, ("v_add_f32_e32 v30, v31, v16", ""), end], 0),
             # over a taken branch, and the product behind it in a loop
             ([product, ("s_cbranch_scc1 1", " <kernel+0xc>"), ("s_nop 11", ""), read, end], 1),
             ([read, ("s_nop 11", ""), product, ("s_branch 65500", " <kernel+0x0>"), end], 1)]
    for lines, count in cases:
        (name, code, jumps), = functions(listing(*lines))
        assert name == "kernel" and len(too_early(code, jumps)) == count, lines


@pytest.mark.parametrize("kernel", [b"window_forward_kernel", b"window_dkv_kernel"])
def test_products_are_there_before_they_are_read(kernel):
    products = 0
    for text in code_objects(("llvm-objdump", "-d", "--no-show-raw-insn"), kernel):
        for name, code, jumps in functions(text):
            if "window_" in name:
                products += sum(op.startswith("v_mfma") for op, _ in code)
                assert not too_early(code, jumps), (name, too_early(code, jumps)[:3])
    assert products > 300
