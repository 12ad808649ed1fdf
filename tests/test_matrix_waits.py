"""Waits behind the scaled matrix instructions of the 8-bit product, read from the assembly
that the compiler writes for its source (no GPU).

The result of such an instruction is touched by another kind of instruction, or is an
operand other than the accumulator of a further one, 20 wait states later at the earliest
(the instruction takes 8 passes, and 12 states would do); an instruction is one wait state,
s_nop N is N + 1.  Followed along every path through a kernel, around its loops as well."""
import os
import re
import subprocess

import pytest

from paper_2607_11185_amd import build as B

WAIT = 20
PRODUCT = "v_mfma_scale"


def _registers(text):
    out = set()
    for a, b, c in re.findall(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b", text):
        out |= {int(c)} if c else set(range(int(a), int(b) + 1))
    return out


def _blocks(lines):
    """{label: ([instructions], [labels that follow])} of a kernel's lines, in order."""
    blocks, name, order = {}, "", [""]
    blocks[name] = []
    ended = False                                # behind a branch: a block without a label
    for line in lines:
        line = line.split(";")[0].strip()
        m = re.match(r"(\.LBB\w+):", line)
        if m or ended:
            name = m[1] if m else f"{name}+"
            blocks.setdefault(name, [])
            order.append(name)
            ended = False
            if m:
                continue
        if not line or line.startswith("."):
            continue
        blocks[name].append(line)
        ended = line.startswith(("s_branch", "s_cbranch", "s_endpgm"))
    out = {}
    for i, name in enumerate(order):
        code = blocks[name]
        last = code[-1].split() if code else [""]
        to = [last[1]] if last[0].startswith(("s_branch", "s_cbranch")) else []
        if not last[0].startswith(("s_branch", "s_endpgm")) and i + 1 < len(order):
            to.append(order[i + 1])
        out[name] = (code, to)
    return out


def _states(line):
    m = re.match(r"s_nop (\d+)", line)
    return int(m[1]) + 1 if m else 1


def early(lines):
    """[(wait states, instruction)] that touch a result too early."""
    blocks = _blocks(lines)
    entry = {b: {} for b in blocks}              # register -> least wait states since it was written
    todo, bad, seen = [next(iter(blocks))], set(), set()
    while todo:
        name = todo.pop()
        seen.add(name)
        age = dict(entry[name])
        code, to = blocks[name]
        for line in code:
            op, _, rest = line.partition(" ")
            args = re.split(r",\s*(?![^\[]*\])", rest)
            product = op.startswith(PRODUCT)
            used = _registers(",".join(args[1:3] + args[4:])) if product else _registers(rest)
            for r in used & age.keys():
                bad.add((age[r], line))
            n = _states(line)
            age = {r: a + n for r, a in age.items() if a + n < WAIT}
            if product:
                age.update({r: 0 for r in _registers(args[0])})
        for b in to:
            new = {r: min(a, entry[b].get(r, WAIT)) for r, a in age.items()}
            if b not in seen or any(a < entry[b].get(r, WAIT) for r, a in new.items()):
                entry[b].update(new)
                todo.append(b)
    return sorted(bad)


def open_loops(lines):
    """Backward branches of loops with products that are reached with less than WAIT states
    of s_nop behind the last product, as (s_nop states, label)."""
    text = [l.split(";")[0].strip() for l in lines]
    at = {m[1]: i for i, l in enumerate(text) if (m := re.match(r"(\.LBB\w+):", l))}
    out = []
    for i, line in enumerate(text):
        m = re.match(r"s_c?branch\w* (\.LBB\w+)", line)
        if not m or at[m[1]] > i:
            continue
        body = text[at[m[1]]:i]
        last = max((j for j, l in enumerate(body) if l.startswith(PRODUCT)), default=None)
        if last is None:
            continue
        n = sum(_states(l) for l in body[last:] if l.startswith("s_nop"))
        if n < WAIT:
            out.append((n, m[1]))
    return out


P = "v_mfma_scale_f32_16x16x128_f8f6f4 v[0:3], v[8:15], v[16:23], v[0:3], v24, v25 op_sel_hi:[0,0,0]"


@pytest.mark.parametrize("code,want", [
    ([P, "v_mov_b32_e32 v30, v3"], 1), ([P, "s_nop 15", "s_nop 2", "v_mov_b32_e32 v30, v3"], 1),
    ([P, "s_nop 15", "s_nop 3", "v_mov_b32_e32 v30, v3"], 0), ([P, P, P], 0), ([P, "v_mov_b32_e32 v30, v4"], 0),
    ([P, P.replace("v[8:15]", "v[2:9]")], 1), ([P, "global_store_dwordx4 v40, v[0:3], s[0:1]"], 1), ([P, "v_mov_b32_e32 v2, 0"], 1),
    # around a loop, and past a branch
    ([".LBB0_1:", "v_mov_b32_e32 v30, v3", "s_nop 7", P, "s_cbranch_scc1 .LBB0_1", "s_endpgm"], 1),
    ([".LBB0_1:", "s_nop 15", "s_nop 3", "v_mov_b32_e32 v30, v3", P, "s_cbranch_scc1 .LBB0_1", "s_endpgm"], 0),
    ([P, "s_cbranch_scc1 .LBB0_2", "s_nop 15", "s_nop 15", ".LBB0_2:", "v_mov_b32_e32 v30, v3"], 1)])
def test_the_reading_itself(code, want):
    assert len(early(code)) == want


def test_the_reading_of_loops():
    assert open_loops([".LBB0_1:", P, "s_nop 15", "s_barrier", "s_cbranch_scc1 .LBB0_1"]) == [(16, ".LBB0_1")]
    assert open_loops([".LBB0_1:", P, "s_nop 15", "s_nop 3", "s_cbranch_scc1 .LBB0_1", "s_branch .LBB0_2", ".LBB0_2:"]) == []


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: lines} of the kernels that hold scaled products."""
    if not os.path.exists(B.HIPCC):
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("asm") / "product.s"
    subprocess.run([B.HIPCC, *B.FLAGS, "-I", B.INCLUDE, "-I", B.CSRC, "--cuda-device-only", "-S",
                    os.path.join(B.CSRC, "seg_fp8_gemm.hip"), "-o", str(out)], check=True, capture_output=True)
    found, name = {}, None
    for line in out.read_text().splitlines():
        m = re.match(r"(_Z\w+):", line)
        name = m[1] if m else None if line.startswith(".Lfunc_end") else name
        if name:
            found.setdefault(name, []).append(line)
    found = {n: l for n, l in found.items() if any(x.strip().startswith(PRODUCT) for x in l)}
    assert sum("k_gemm8" in n for n in found) == 8 and sum("k_few8" in n for n in found) == 14
    return found


def test_no_result_is_touched_early(kernels):
    assert {n: e for n, l in kernels.items() if (e := early(l))} == {}


def test_loops_close_behind_a_wait(kernels):
    assert {n: e for n, l in kernels.items() if (e := open_loops(l))} == {}
