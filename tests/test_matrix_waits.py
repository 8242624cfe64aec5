"""Waits behind matrix products in double.  A result of v_mfma_f64_16x16x4 may be read 18 wait states after the product at the earliest
(what the compiler leaves between them); the hardware does not wait by itself.  At one place the compiler has left four, and the
source has a wait of its own there; a later compiler may have others.  So every way from every such product to the first
reading of its result is looked up in the built library."""
import os
import re
import shutil
import subprocess

import pytest

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
STATES = 18
LINE = re.compile(r"\s+(\S+)\s*(.*?)\s*// ([0-9A-F]+): [0-9A-F ]+(?:<.*\+0x([0-9a-f]+)>)?\s*$")
WRITES_FIRST = ("v_", "ds_read", "ds_bpermute", "global_load", "buffer_load", "flat_load", "scratch_load")
READS_ALL = ("v_cmp", "v_swap", "v_readlane", "v_readfirstlane")


def registers(text):
    found = set()
    for kind, low, high in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        found |= {(kind, i) for i in range(int(low), int(high) + 1)}
    return found | {(kind, int(i)) for kind, i in re.findall(r"\b([va])(\d+)\b", text)}


def functions(listing):
    """name -> (address, [(address, instruction, operands, branch target)])"""
    found, name = {}, None
    for line in listing.splitlines():
        start = re.match(r"([0-9a-f]+) <(.*)>:$", line)
        if start:
            name = start.group(2)
            found[name] = (int(start.group(1), 16), [])
        elif name:
            m = LINE.match(line)
            if m:
                found[name][1].append((int(m.group(3), 16), m.group(1), m.group(2), int(m.group(4), 16) if m.group(4) else None))
    return found


def nearest_reading(base, code):
    """(wait states, where) of the earliest reading of a product's result on any way through the function, up to STATES."""
    place = {address: i for i, (address, *_) in enumerate(code)}
    nearest = (STATES, None)
    for i, (address, op, operands, _) in enumerate(code):
        if not op.startswith("v_mfma_f64_16x16"):
            continue
        result = registers(operands.split(",")[0])
        ways, seen = [(i + 1, 0)], {}
        while ways:
            j, states = ways.pop()
            while j < len(code) and states < nearest[0] and seen.get(j, STATES) > states:
                seen[j] = states
                _, what, text, target = code[j]
                parts = text.split(",")
                if what.startswith("v_mfma"):
                    to, sums = registers(parts[0]), registers(parts[3])
                    read = (registers(parts[1]) | registers(parts[2])) & result or (sums & result and sums != result)
                    if not read and to == result:
                        break  # added up further (or made anew): its own way
                elif what.startswith(WRITES_FIRST) and not what.startswith(READS_ALL):
                    read = registers(",".join(parts[1:])) & result
                else:
                    read = registers(text) & result
                if read:
                    nearest = (states, "%x: %s %s after %x" % (code[j][0], what, text, address))
                    break
                states += int(text.split()[0], 0) + 1 if what == "s_nop" else 1
                if what == "s_endpgm":
                    break
                if what == "s_branch":
                    j = place[base + target]
                    continue
                if what.startswith("s_cbranch"):
                    ways.append((place[base + target], states))
                j += 1
    return nearest


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler for the GPU's code")
def test_results_of_products_in_double_are_waited_for(tmp_path):
    import paper_2302_00845_amd as pkg
    if not os.path.exists(pkg.library_path()):
        from paper_2302_00845_amd import build
        build.build_library(verbose=False)
    shutil.copy(pkg.library_path(), tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    code, = [f for f in os.listdir(tmp_path) if "gfx950" in f]
    listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", code], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
    looked_at = 0
    for name, (base, lines) in functions(listing).items():
        if any(op.startswith("v_mfma_f64") for _, op, _, _ in lines):
            looked_at += 1
            states, where = nearest_reading(base, lines)
            assert states >= STATES, "%s: %d wait states, %s" % (name, states, where)
    assert looked_at >= 100 and any("ortho_narrow" in name for name in functions(listing))


def listing_of(*lines):
    """A function at 0x100 of the given lines, eight bytes each; '-> n' is a branch to line n."""
    out = ["0000000000000100 <f>:"]
    for i, line in enumerate(lines):
        text, _, to = line.partition(" -> ")
        out.append("\t%-58s // %012X: BF800000 %s" % (text, 0x100 + 8 * i, "<f+0x%x>" % (8 * int(to)) if to else ""))
    return "\n".join(out)


PRODUCT = "v_mfma_f64_16x16x4_f64 v[0:7], v[10:11], v[12:13], 0"


@pytest.mark.parametrize("lines,states", [
    ([PRODUCT, "s_nop 15", "s_nop 1", "v_mov_b32_e32 v20, v7", "s_endpgm"], 18),
    ([PRODUCT, "s_nop 3", "v_mov_b32_e32 v20, v7", "s_endpgm"], 4),
    ([PRODUCT, "v_mov_b32_e32 v30, v29", "global_store_dwordx4 v[30:31], v[4:7], off", "s_endpgm"], 1),
    ([PRODUCT, "v_mov_b32_e32 v3, v29", "s_endpgm"], 18),  # (written, not read)
    ([PRODUCT, "v_mfma_f64_16x16x4_f64 v[0:7], v[10:11], v[12:13], v[0:7]", "s_nop 9", "v_add_f64 v[20:21], v[2:3], 0", "s_endpgm"], 10),
    ([PRODUCT, "v_mfma_f64_16x16x4_f64 v[20:27], v[0:1], v[12:13], 0", "s_endpgm"], 0),
    # at a loop's head, reached from its end
    (["v_accvgpr_write_b32 a5, v6", "s_nop 15", "s_nop 15", PRODUCT, "s_nop 2", "s_cbranch_scc1 5 -> 0", "s_endpgm"], 4),
    ([PRODUCT, "s_branch 7 -> 4", "s_nop 15", "s_nop 15", "v_mov_b32_e32 v20, v0", "s_endpgm"], 1),
])
def test_the_look_up(lines, states):
    (base, code), = functions(listing_of(*lines)).values()
    assert len(code) == len(lines) and nearest_reading(base, code)[0] == states
