"""Static checks of w8a8_tile_kernel's machine code (CPU only), with the checkers of
test_asm_schedule.py: the matrix instructions' wait states and the LDS reads' waits,
of neither of which the compiler knows, and, since the kernel's counted waits rely on
it, the vector-memory operations of a pass of its loop."""
import os
import re
import tempfile

import pytest

import test_asm_schedule as T

FORMS = {(16, 4): 4, (8, 4): 8, (8, 2): 8, (4, 2): 8, (4, 1): 8}       # (RB, CB): steps a pass of the loop


def cut(body):
    """The instructions from the last barrier before the step loop (one block, which has
    all matrix instructions) up to it, the loop's, and those that follow it up to the
    next barrier."""
    blocks, names = [[]], [""]
    for line in body.splitlines():
        m = re.match(r"^(\.LBB\d+_\d+):", line)
        if m:
            blocks.append([])
            names.append(m.group(1))
        blocks[-1].append(line)
    code = [T.code(T.parse("\n".join(b))) for b in blocks]
    loops = [k for k, b in enumerate(code) if any(op.startswith("v_mfma") for op, _ in b)]
    assert len(loops) == 1, "one block with matrix instructions"
    k = loops[0]
    # a loop, left by falling through or by a branch
    then = k + 1
    if code[k][-1][0] == "s_branch":
        then = names.index(code[k].pop()[1])
    assert code[k][-1][0].startswith("s_cbranch") and code[k][-1][1] == names[k]
    before = sum(code[:k], [])
    last = max(i for i, (op, _) in enumerate(before) if op == "s_barrier")
    after = sum(code[then:], [])
    return before[last:], code[k], after[:next(i for i, (op, _) in enumerate(after) if op == "s_barrier")]


@pytest.fixture(scope="module")
def fns():
    if not os.path.exists(T.B.HIPCC):
        pytest.skip("hipcc not available")
    with tempfile.TemporaryDirectory(prefix="tf_asm_") as tmp:
        out = T._compile_asm(os.path.join(T.B.CSRC, "tf_w8a8_tile.hip"), os.path.join(tmp, "tile.s"))
        text = open(out).read()
    got = [(m.group(1), cut(m.group(2))) for m in re.finditer(r"^(_Z\S+):[^\n]*\n(.*?)^\.Lfunc_end", text, re.S | re.M)
           if "w8a8_tile_" in m.group(1)]
    assert len(got) == 3 * len(FORMS) + 1             # dense, experts with rows and without; K split
    return got


def form(name):
    m = re.search(r"FormILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)E", name)
    return [int(v) for v in m.groups()]               # RB, CB, P, R


def test_mfma_wait_states(fns):
    """In the loop, from the accumulators' zeros to it, and from it to their first reads."""
    for name, (before, loop, after) in fns:
        assert T.check_mfma_hazards(before + 2 * loop + after) == [], name


def test_fragments_are_waited_for(fns):
    """No register that an LDS read of fragments targets is touched before it has
    returned: before the loop, over three passes of it and behind it."""
    for name, (before, loop, after) in fns:
        first = next(i for i, (op, _) in enumerate(before) if op.startswith("ds_read_b128"))
        assert not any(op.startswith("scratch_") for op, _ in loop), name
        wait = next(i for i, (op, a) in enumerate(after) if op == "s_waitcnt" and "lgkmcnt(0)" in a)
        assert T.check_vm_waits(before[first:] + 3 * loop + after[:wait + 1]) == [], name
        assert not any(op.startswith("s_cbranch") for op, _ in after[:wait]), name


def test_operations_of_a_pass(fns):
    """Every step has the same vector-memory operations, direct loads before weights,
    and the barriers' waits leave as many on their way as the kernel's comment says."""
    for name, (_, loop, _) in fns:
        RB, CB, P, R = form(name)
        assert FORMS[RB, CB] == R
        dma, often = RB // 4, RB * CB >= 64
        steps, barriers, mfma = [[] for _ in range(R)], [], 0
        for i, (op, a) in enumerate(loop):
            mfma += op.startswith("v_mfma")
            if op.startswith("buffer_load"):
                steps[mfma // (RB * CB)].append("a" if a.endswith(" lds") else "b")
            assert not op.startswith(("global_", "buffer_store", "scratch_")), name
            if op == "s_barrier":
                m = re.search(r"vmcnt\((\d+)\)", loop[i - 1][1]) if loop[i - 1][0] == "s_waitcnt" else None
                barriers.append((mfma // (RB * CB), m and int(m.group(1))))
        assert mfma == R * RB * CB and steps == [["a"] * dma + ["b"] * CB] * R, name
        later = min(63, CB + (2 * P - (5 if often else 6)) * (dma + CB))
        want = [(s, later if s % 2 else None) for s in range(1, R + 1) if often or s % 2]
        assert barriers == want, name
