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


# ------------------------------------------------------------------ the same over every path, branches back included

class Paths:
    """A kernel's instructions (lists of words) and where each may go on."""

    def __init__(self, lines):
        self.code, at, targets = [], {}, {}
        for line in lines:
            text, _, note = line.partition("//")
            words = re.split(r"[ ,]+", text.strip())
            at[int(note.split(":")[0], 16)] = len(self.code)
            if words[0].startswith(("s_branch", "s_cbranch")):
                targets[len(self.code)] = int(note.split(":")[0], 16) + 4 + 4 * ((int(words[1], 0) + 0x8000) % 0x10000 - 0x8000)
            self.code.append(words)
        assert not any(w[0].startswith(("s_setpc", "s_swappc", "s_call")) for w in self.code)
        self.next = []
        for i, w in enumerate(self.code):
            n = [] if w[0] in ("s_endpgm", "s_branch") or i + 1 == len(self.code) else [i + 1]
            self.next.append(n + ([at[targets[i]]] if i in targets else []))

    def loops(self):
        """Instructions that can be reached from themselves, by their strongly connected components."""
        order, seen, back = [], set(), [[] for _ in self.code]
        for i, n in enumerate(self.next):
            for k in n:
                back[k].append(i)
        for root in range(len(self.code)):
            stack = [(root, iter(self.next[root]))] if root not in seen else []
            seen.add(root)
            while stack:
                node, it = stack[-1]
                k = next((k for k in it if k not in seen), None)
                if k is None:
                    order.append(stack.pop()[0])
                else:
                    seen.add(k)
                    stack.append((k, iter(self.next[k])))
        found, done = [], set()
        for root in reversed(order):
            part, todo = [], [] if root in done else [root]
            done.add(root)
            while todo:
                part.append(todo.pop())
                fresh = [k for k in back[part[-1]] if k not in done]
                done.update(fresh)
                todo += fresh
            if len(part) > 1:
                found.append(sorted(part))
        return found

    def least(self, start, step):
        """The state before every instruction that holds on all paths: numbers by name, the least of those of the paths.  step(words, state) is the
        state behind an instruction; a name that is not there is far enough away."""
        state, todo = {0: start}, [0]
        while todo:
            i = todo.pop()
            out = step(self.code[i], state[i])
            for k in self.next[i]:
                old = state.get(k)
                new = out if old is None else {**out, **{n: min(v, out.get(n, v)) for n, v in old.items()}}
                if new != old:
                    state[k] = new
                    todo.append(k)
        return state


@pytest.fixture(scope="module")
def paths(objects):  # noqa: F811
    found = {}
    for obj in objects:
        if not any("k_mx4_tile" in n for n in _kernels(obj)):
            continue
        name = None
        for line in subprocess.run([LLVM + "/llvm-objdump", "-d", "--no-show-raw-insn", obj], check=True, stdout=subprocess.PIPE, text=True).stdout.split("\n"):
            if m := re.match(r"[0-9a-f]+ <(\S+)>:", line):
                if ".L" not in m[1]:
                    name = m[1] if "k_mx4_tile" in m[1] else None
            elif name and "//" in line:
                found.setdefault(name, []).append(line)
    assert len(found) == 6
    return {n: Paths(lines) for n, lines in found.items()}


def test_the_walk_over_paths():
    """A read behind a loop's branch back is found, one beside it is not."""
    text = ["s_mov_b32 s0, 0", "v_mfma_scale_x a[0:3], v[0:3], v[4:7], a[0:3], v8, v9", "s_nop 1", "s_cbranch_scc1 65533", "v_accvgpr_read_b32 v1, a0", "s_endpgm"]
    p = Paths(["\t%s // %012X: 00000000" % (t, 4 * i) for i, t in enumerate(text)])
    assert p.next == [[1], [2], [3], [4, 1], [5], []] and p.loops() == [[1, 2, 3]]
    state = p.least({}, _since_product)
    assert state[1] == {"product": 3} and state[4] == {"product": 3}


def _since_product(words, state):
    """Wait states since the last matrix instruction, up to 20."""
    if words[0].startswith("v_mfma"):
        return {"product": 0}
    return {n: v + _waits(words) for n, v in state.items() if v + _waits(words) < 20}


def _since_writes(words, state):
    """Wait states since a vector instruction wrote a register, up to 2."""
    state = {r: v + _waits(words) for r, v in state.items() if v + _waits(words) < 2}
    if words[0].startswith("v_") and not words[0].startswith(("v_mfma", "v_cmp")):
        state.update({r: 0 for r in _registers(words[1])})
    return state


def test_waits_hold_on_every_path(paths):
    for name, p in paths.items():
        written, product = p.least({}, _since_writes), p.least({}, _since_product)
        reads = 0
        for i, w in enumerate(p.code):
            if i not in product:
                continue  # (padding)
            if w[0].startswith("v_mfma_scale"):
                assert not set().union(*[_registers(o) for o in w[2:7]]) & set(written[i]), (name, i, w)
            elif any(k == "a" for o in w[1:] for k, _ in _registers(o)):
                reads += "product" not in product[i] and w[0].startswith(("v_accvgpr_read", "ds_write"))
                assert not product[i], (name, i, w, product[i])
        assert reads >= 16


def test_only_products_touch_the_sums_in_the_loops(paths):
    for name, p in paths.items():
        products = 0
        for loop in p.loops():
            found = [p.code[i] for i in loop if p.code[i][0].startswith("v_mfma_scale")]
            products += len(found)
            others = [p.code[i] for i in loop if not p.code[i][0].startswith("v_mfma_scale") and any(k == "a" for o in p.code[i][1:] for k, _ in _registers(o))]
            assert not found or not others, (name, others[:3])
        assert products >= 16


def test_scratch_of_the_norms(objects):  # noqa: F811
    """Registers hold what the norms keep, but for rows of more than 8192 columns, two pieces a lane, and the gradients of both lines with a float16
    layer norm's biases in 16 waves."""
    found = {n: v[1] for obj in objects for n, v in _kernels(obj).items() if re.search(r"k_norm(_back|_sums)?I", n)}
    assert len(found) > 100
    for name, scratch in found.items():
        two = re.search(r"Li16ELi2EEEv", name) and not re.search(r"6k_normI\S*Lb1ELb0ELi16|6k_normI\S*Lb0ELb1ELi16", name)
        assert scratch == 0 or two or "k_norm_backINS0_3F16ELb1ELb1ELb1ELb1ELi16ELi1E" in name, (name, scratch)
    assert sum(s > 0 for s in found.values()) <= 20
