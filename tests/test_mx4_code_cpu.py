"""What the compiler does not look after around the matrix instructions that the 4-bit tiles issue in statements of their own: wait states
before and behind them, and that their sums stay where they are."""
import re
import subprocess

import pytest

from test_code_objects_cpu import LLVM, _kernels, objects  # noqa: F401 (objects is a fixture)


def _registers(operand):
    m = re.fullmatch(r"([va])(\d+)|([va])\[(\d+):(\d+)\]", operand)
    if not m:
        return set()
    return {(m[1], int(m[2]))} if m[1] else {(m[3], i) for i in range(int(m[4]), int(m[5]) + 1)}


@pytest.fixture(scope="module")
def tiles(objects):  # noqa: F811
    """name -> instructions, as lists of words"""
    found = {}
    for obj in objects:
        if not any("k_mx4_tile" in n for n in _kernels(obj)):
            continue
        name = None
        for line in subprocess.run([LLVM + "/llvm-objdump", "-d", "--no-show-raw-insn", obj], check=True, stdout=subprocess.PIPE, text=True).stdout.split("\n"):
            if m := re.match(r"[0-9a-f]+ <(\S+)>:", line):
                name = m[1] if "k_mx4_tile" in m[1] and ".L" not in m[1] else None if ".L" not in m[1] else name
            elif name and line.strip():
                words = re.split(r"[ ,]+", line.split("//")[0].strip())
                if words[0]:
                    found.setdefault(name, []).append(words)
    assert len(found) == 6
    return found


def _waits(words):
    return int(words[1], 0) + 1 if words[0] == "s_nop" else 1


def test_operands_are_there_two_wait_states_before(tiles):
    """gfx9: two wait states between a vector instruction's write of a register and a matrix instruction that reads it."""
    for name, code in tiles.items():
        count = 0
        for i, w in enumerate(code):
            if not w[0].startswith("v_mfma_scale"):
                continue
            count += 1
            reads, waits = set().union(*[_registers(o) for o in w[2:7]]), 0
            for prev in reversed(code[max(0, i - 4):i]):
                if waits >= 2:
                    break
                if prev[0].startswith("v_") and not prev[0].startswith(("v_mfma", "v_cmp")):
                    assert not _registers(prev[1]) & reads, (name, prev, w)
                waits += _waits(prev)
        assert count >= 16


def test_sums_stay_in_place_and_are_read_late_enough(tiles):
    """Every product adds into the registers it reads its sums from; nothing else touches them in the loops, and 20 wait states pass
    between the last product and the first instruction that reads them."""
    for name, code in tiles.items():
        last = None
        for i, w in enumerate(code):
            if w[0].startswith("v_mfma_scale"):
                assert w[1] == w[4] and w[1].startswith("a["), (name, w)
                last, waits = i, 0
            elif last is not None:
                if w[0].startswith("v_accvgpr_read"):
                    assert waits >= 20, (name, waits, w)
                waits += _waits(w)


def test_no_scratch(objects):  # noqa: F811
    found = {n: v for obj in objects for n, v in _kernels(obj).items() if "k_mx4_" in n}
    assert len(found) > 20 and all(scratch == 0 for _, scratch in found.values()), found
