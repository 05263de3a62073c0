"""The waits between matrix instructions and the readers of their results, in the library
as it is built.

A matrix instruction's result is in its registers some issue slots after it has begun,
and the hardware does not wait by itself: the compiler puts other instructions or s_nop
between.  It counts along straight code; where several ways lead to a reader it has left
some short, and the reader then took what the registers held before.  Here every way
through every kernel is walked."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_13500_amd import _lib, build

# Slots between a matrix instruction of so many passes (of 4 cycles) and an instruction
# other than a matrix one that reads or overwrites its result, or a matrix one that takes
# it as a factor.
SLOTS = {4: 8, 8: 12}
PASSES = {"v_mfma_f32_16x16x32_bf16": 4, "v_mfma_f32_32x32x16_bf16": 8}

_REGISTERS = re.compile(r"\b([av])(?:\[(\d+):(\d+)\]|(\d+))")
_LOADS = ("global_load", "buffer_load", "flat_load", "scratch_load", "ds_read")


def registers(text):
    out = set()
    for kind, first, last, one in _REGISTERS.findall(text):
        out.update((kind, n) for n in range(int(first or one), int(last or one) + 1))
    return out


def operands(text):
    return [x.strip() for x in text.split(",")]


class Instruction:
    def __init__(self, address, text):
        self.address, self.after = address, []
        self.op, _, rest = text.partition(" ")
        self.matrix = self.op.startswith("v_mfma")
        parts = operands(rest)
        self.result, self.factors, self.added = set(), set(), set()
        if self.matrix:
            self.result, self.factors, self.added = registers(parts[0]), registers(parts[1]) | registers(parts[2]), registers(parts[3])
        elif self.op.startswith(("v_", "global_", "buffer_", "flat_", "scratch_", "ds_")):
            # what a load overwrites arrives long after
            self.factors = registers(",".join(parts[1:] if self.op.startswith(_LOADS) else parts))
        self.slots = int(rest, 0) + 1 if self.op == "s_nop" else 1


def kernels(listing):
    """(name, instructions) of a disassembly, each instruction with the ones it can be followed by."""
    for chunk in re.split(r"\n(?=[0-9a-f]{16} <)", listing):
        head = re.match(r"([0-9a-f]{16}) <(\S+)>:", chunk)
        if not head:
            continue
        base, code = int(head.group(1), 16), []
        targets = {}
        for line in chunk.splitlines()[1:]:
            m = re.match(r"\t(\S.*?)\s*// ([0-9A-F]{12}):(?: [0-9A-F]{8})+(?: <[^>+]*(?:\+0x([0-9a-f]+))?>)?", line)
            if not m:
                continue
            code.append(Instruction(int(m.group(2), 16), m.group(1)))
            if code[-1].op.startswith(("s_branch", "s_cbranch")):
                targets[len(code) - 1] = base + int(m.group(3) or "0", 16)
        at = {i.address: n for n, i in enumerate(code)}
        for n, i in enumerate(code):
            if i.op in ("s_endpgm", "s_setpc_b64"):
                continue
            if i.op != "s_branch" and n + 1 < len(code):
                i.after.append(n + 1)
            if n in targets:
                i.after.append(at[targets[n]])
        yield head.group(2), code


def least_slots(code, start):
    """Fewest slots between the matrix instruction and a use of its result, and the use; up
    to what it needs."""
    need = SLOTS[PASSES[code[start].op]]
    seen, ways, least = {}, [(n, 0, frozenset(code[start].result)) for n in code[start].after], (need, None)
    while ways:
        n, slots, live = ways.pop()
        if slots >= least[0] or seen.get((n, live), need) <= slots:
            continue
        seen[n, live] = slots
        i = code[n]
        if i.factors & live:
            least = (slots, n)
            continue
        if i.matrix and (i.added & live or i.result & live):
            live = live - i.result        # sums go on in order; what is read then is the later one's
        if live:
            ways += [(m, slots + i.slots, live) for m in i.after]
    return least


def short_of(listing):
    """Uses that come too early (kernel, product, its address, use, its address, slots), and
    how many products there are."""
    found, products = [], 0
    for name, code in kernels(listing):
        for n, i in enumerate(code):
            if i.matrix:
                products += 1
                slots, use = least_slots(code, n)
                if use is not None:
                    found.append((name, i.op, hex(i.address), code[use].op, hex(code[use].address), slots))
    return found, products


def listing_of(lines):
    """A disassembly of one kernel of 4-byte instructions; "-> n" branches to line n."""
    out = ["", "%016x <kernel>:" % 0x100]
    for n, line in enumerate(lines):
        text, _, target = line.partition(" -> ")
        out.append("\t%-50s // %012X: BF800000%s" % (text, 0x100 + 4 * n, " <kernel+0x%x>" % (4 * int(target)) if target else ""))
    return "\n".join(out) + "\n"


PRODUCT = "v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]"


@pytest.mark.parametrize("lines,slots", [
    ([PRODUCT, "s_nop 7", "v_accvgpr_read_b32 v9, a2", "s_endpgm"], None),
    ([PRODUCT, "s_nop 6", "v_accvgpr_read_b32 v9, a2", "s_endpgm"], 7),
    ([PRODUCT, "s_nop 6", "v_accvgpr_read_b32 v9, a4", "s_endpgm"], None),
    ([PRODUCT, "global_store_dwordx4 v8, a[0:3], s[0:1]", "s_endpgm"], 0),
    ([PRODUCT, "v_mov_b32_e32 a3, v1", "s_endpgm"], 0),                                        # overwritten
    ([PRODUCT, PRODUCT.replace("16x16x32", "32x32x16").replace("v[4:7]", "a[0:3]"), "s_endpgm"], 0),   # a factor
    ([PRODUCT, PRODUCT, "s_nop 7", "v_accvgpr_read_b32 v9, a2", "s_endpgm"], None),            # sums in order
    # the way along is long enough, the branch is not
    ([PRODUCT, "s_cbranch_scc1 1 -> 3", "s_nop 7", "s_nop 3", "v_accvgpr_read_b32 v9, a2", "s_endpgm"], 5),
    # around a loop
    (["v_accvgpr_read_b32 v9, a2", "s_nop 7", PRODUCT, "s_cbranch_scc1 1 -> 0", "s_endpgm"], 1)])
def test_the_walk(lines, slots):
    found, products = short_of(listing_of(lines))
    assert products == sum("mfma" in x for x in lines) and [f[-1] for f in found] == ([] if slots is None else [slots])


def test_no_result_is_read_too_early(tmp_path):
    tool = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.hipcc()))), "llvm", "bin", "llvm-objdump")
    if not os.path.exists(tool):
        tool = shutil.which("llvm-objdump")
    _lib.load()                                  # builds it where there is none
    library = str(tmp_path / "library.so")
    shutil.copy(_lib.LIB_PATH, library)
    subprocess.run([tool, "--offloading", library], check=True, capture_output=True)
    objects = [f for f in sorted(os.listdir(tmp_path)) if f.endswith("gfx950")]
    found, products, ops = [], 0, set()
    for f in objects:
        listing = subprocess.run([tool, "-d", str(tmp_path / f)], check=True, capture_output=True, text=True).stdout
        ops |= set(re.findall(r"\bv_mfma\w+", listing))
        short, n = short_of(listing)
        found += short
        products += n
    assert products > 1000 and ops <= set(PASSES) and not found, found
