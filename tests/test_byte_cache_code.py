"""The 8-bit cache's kernels as the compiler left them in the built library.

A matrix instruction writes its result some cycles after it was issued, and nothing in the hardware makes an ordinary instruction
wait for it: the compiler counts wait states and puts s_nop in between.  Where the first use of a result stood behind a branch,
it left one or two of the eight that it keeps elsewhere, and sums came out wrong on the path where the branch is taken.  So every
path from every matrix instruction is walked here."""

import os
import re
import subprocess

import pytest

from test_kernel_registers import LIB, READELF, device_objects

OBJDUMP = os.path.join(os.path.dirname(READELF), "llvm-objdump")
WAIT = 8                                      # wait states between a product of four passes and the first use of its result
# kernels that keep some registers in scratch memory: bytes per lane
SPILLS = {"_Z12k_byte_pieceIDF16_Li128ELb1E": 40, "_Z12k_byte_storeItLi128E": 16}


def registers(text):
    """Numbers of the vector registers that an operand, or several, names."""
    out = set()
    for low, high, one in re.findall(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b", text):
        out |= {int(one)} if one else set(range(int(low), int(high) + 1))
    return out


def kernels(listing):
    """name -> ([(operation, operands, target index or None)]) of llvm-objdump's listing."""
    out, code, place, name = {}, None, None, None
    for line in listing.splitlines():
        head = re.match(r"[0-9a-f]+ <(\S+)>:", line)
        if head:
            name, code, place = head.group(1), [], {}
            out[name] = (code, place)
            start = None
            continue
        m = re.match(r"\s+(\S+)\s*(.*?)\s*// ([0-9A-F]+): [0-9A-F ]+(?:<\S+?\+0x([0-9a-f]+)>)?$", line)
        if code is None or not m:
            continue
        at = int(m.group(3), 16)
        start = at if start is None else start
        place[at - start] = len(code)
        code.append((m.group(1), m.group(2), int(m.group(4), 16) if m.group(4) else None))
    return {k: [(op, args, place.get(to) if to is not None else None) for op, args, to in c] for k, (c, place) in out.items()}


def early_uses(code):
    """(operation, wait states) of every instruction that reads or writes a matrix instruction's result before it has arrived.
    A later matrix instruction may add to it or overwrite it at once: those follow each other in their own unit."""
    found = []
    for i, (op, args, _) in enumerate(code):
        if not op.startswith("v_mfma"):
            continue
        result, seen, open_ = registers(args.split(",")[0] if "[" not in args else args[:args.index("]") + 1]), set(), [(i + 1, 0)]
        while open_:
            at, waited = open_.pop()
            if at >= len(code) or waited >= WAIT or (at, waited) in seen:
                continue
            seen.add((at, waited))
            op, args, to = code[at]
            if op == "s_endpgm":
                continue
            if op.startswith("v_mfma"):
                parts = re.findall(r"[va]\[\d+:\d+\]|[^,\s]+", args)
                if registers(parts[1] + " " + parts[2]) & result:
                    found.append((op, waited))
                    continue
                if registers(parts[0]) & result:
                    continue
            elif op.startswith(("v_", "ds_", "global_", "flat_", "scratch_", "buffer_")) and registers(args) & result:
                found.append((op, waited))
                continue
            waited += int(args.split()[0]) + 1 if op == "s_nop" else 1
            if to is not None:
                open_.append((to, waited))
            if op != "s_branch":
                open_.append((at + 1, waited))
    return found


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    """The code object that holds the kernels: its path."""
    if not os.path.exists(LIB) or not os.path.exists(OBJDUMP):
        pytest.skip("no built library, or no llvm-objdump beside the compiler")
    path = tmp_path_factory.mktemp("code") / "object"
    for obj in device_objects(open(LIB, "rb").read()):
        if b"k_byte_attn" in obj:
            path.write_bytes(obj)
    return str(path)


def test_results_of_matrix_instructions_have_arrived_where_they_are_used(built):
    code = kernels(subprocess.check_output([OBJDUMP, "-d", built]).decode())
    attention = {k: c for k, c in code.items() if "k_byte_attn" in k or "k_byte_piece" in k}
    assert len(attention) >= 40 and all(sum(op.startswith("v_mfma") for op, _, _ in c) > 10 for c in attention.values())
    assert all(to is not None for c in attention.values() for op, _, to in c if op.startswith(("s_cbranch", "s_branch")))
    assert {k: early_uses(c) for k, c in attention.items() if early_uses(c)} == {}


LISTING = """
0000000000001000 <k>:
	v_mfma_f32_16x16x32_f16 v[8:11], v[0:3], v[4:7], 0// 000000001000: D3D40008 02020900
	s_cbranch_scc1 {skip}                                          // 000000001008: BF850001 <k+0x14>
	s_nop 7                                                    // 00000000100C: BF800007
	v_add_f32_e32 v1, v{used}, v2                                 // 000000001010: 02020508
	v_add_f32_e32 v2, v{used}, v2                                 // 000000001014: 02020508
	s_endpgm                                                   // 000000001018: BF810000
"""


@pytest.mark.parametrize("used,found", [(9, [("v_add_f32_e32", 1)]), (12, [])])
def test_a_use_behind_a_branch_is_found(used, found):
    assert early_uses(kernels(LISTING.format(skip=1, used=used))["k"]) == found


def test_who_keeps_registers_in_scratch_memory(built):
    """Two kernels, a few each; what a loop keeps there costs (fp32 pieces of heads of 128 217 us against 183 without)."""
    notes = subprocess.check_output([READELF, "--notes", built]).decode()
    scratch = {}
    for kernel in re.split(r"\n  - \.a", notes)[1:]:
        size = int(re.search(r"\.private_segment_fixed_size:\s*(\d+)", kernel).group(1))
        if size:
            scratch[re.findall(r"\n    \.name:\s*(\S+)", kernel)[-1]] = size
    assert all(any(k.startswith(p) and size <= most for p, most in SPILLS.items()) for k, size in scratch.items()), scratch
