"""Static check of the loads through inline asm in the compiled kernels of the products grouped by expert (no GPU needed).

The kernels load from memory into LDS with buffer instructions in asm blocks, which the compiler's hazard recogniser cannot see
into.  Checked on the compiled code, following branches:
* a vector-memory instruction reads a scalar register 5 wait states at the earliest after a vector instruction has written it
  (the descriptors end in v_readfirstlane, and spilled scalars come back through v_readlane);
* the register m0, which says where in LDS, is set one wait state at the least before the load, and nothing outside the asm blocks
  reads or writes it (the compiler is not told that they do);
* the loads have no output registers, so nothing in flight can be overwritten or copied too early."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_isa_hazards import _split

NEED = 5
UNITS = ("moe_grouped_row_major", "moe_grouped_transposed", "moe_grouped_mx", "moe_grouped_weights")


def scalars(tok):
    """Scalar registers named by an operand."""
    tok = tok.split()[0] if tok else ""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", tok)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.fullmatch(r"s(\d+)", tok)
    return {int(m.group(1))} if m else set()


def instructions(lines):
    """[(op, operands, in an asm block, line number)], {label: index of the instruction behind it}"""
    out, labels, in_asm = [], {}, False
    for i, l in enumerate(lines):
        s = l.strip()
        m = re.match(r"(\.LBB\d+_\d+):", l)
        if m:
            labels[m.group(1)] = len(out)
        if s.startswith(";;#ASM"):
            in_asm = s.startswith(";;#ASMSTART")
        if not s or s.startswith((";", ".")) or re.match(r"[\w.$]+:", s):
            continue
        op, ops = _split(s)
        out.append((op, ops, in_asm, i + 1))
    return out, labels


def written(op, ops):
    """Scalar registers that an instruction writes."""
    if op.startswith("v_"):
        both = "_co_" in op or op.startswith(("v_div_scale", "v_mad_u64", "v_mad_i64"))
        return set().union(*[scalars(t) for t in ops[:2 if both else 1]]) if ops else set()
    if op.startswith("s_") and ops and not op.startswith(("s_cmp", "s_bitcmp", "s_cbranch", "s_branch", "s_waitcnt", "s_nop", "s_barrier", "s_setprio")):
        return scalars(ops[0])
    return set()


def is_load(op, asm):
    return asm and op.startswith(("buffer_load", "global_load", "buffer_store", "global_store"))


def find_young_scalars(lines):
    """(asm memory instructions, hazards): scalars that they read too soon after a vector instruction wrote them."""
    ins, labels = instructions(lines)
    bad = []
    for i, (op, ops, _, line) in enumerate(ins):
        regs = written(op, ops) if op.startswith("v_") else set()
        if not regs:
            continue
        work, seen = [(i + 1, 0, frozenset(regs))], set()
        while work:
            j, t, live = work.pop()
            while j < len(ins) and t < NEED and live:
                o, oo, asm, at = ins[j]
                j += 1
                if is_load(o, asm) and set().union(*[scalars(x) for x in oo]) & live:
                    bad.append(f"line {at}: {o} reads a scalar that line {line} ({op}) wrote {t} states before")
                    break
                if o == "s_endpgm":
                    break
                live = live - written(o, oo)  # (what writes it next stands for itself)
                t += int(oo[0]) + 1 if o == "s_nop" else 1
                if o == "s_branch":
                    j = labels[oo[0]]
                elif o.startswith("s_cbranch") and (labels[oo[0]], t) not in seen:
                    seen.add((labels[oo[0]], t))
                    work.append((labels[oo[0]], t, live))
    return sum(is_load(o, a) for o, _, a, _ in ins), bad


def find_odd_loads(lines):
    """Asm memory instructions that are no loads into LDS, or whose m0 is not set in the same block a state before."""
    ins, _ = instructions(lines)
    bad = []
    for i, (op, ops, asm, line) in enumerate(ins):
        if not is_load(op, asm):
            continue
        if op != "buffer_load_dwordx4" or not ops[-1].endswith(" lds") or len(ops) != 3:
            bad.append(f"line {line}: not a load into LDS: {op} {ops}")
        elif not (ins[i - 1][0] == "s_nop" and ins[i - 1][2] and ins[i - 2][0] == "s_mov_b32" and ins[i - 2][1][0] == "m0" and ins[i - 2][2]):
            bad.append(f"line {line}: m0 is not set right before")
    return bad


def find_other_uses_of_m0(lines):
    ins, _ = instructions(lines)
    return [f"line {line}: {op} {ops}" for op, ops, asm, line in ins
            if not asm and (any(re.search(r"\bm0\b", o) for o in ops) or op.startswith(("v_movrel", "s_movrel", "s_set_gpr_idx", "ds_gws", "v_interp"))
                            or "load_lds" in op or (op.startswith(("buffer_load", "global_load")) and any(o.endswith(" lds") for o in ops)))]


LOAD = ["\t;;#ASMSTART", "\ts_mov_b32 m0, s9", "\ts_nop 0", "\tbuffer_load_dwordx4 v1, s[4:7], 0 offen lds", "\t;;#ASMEND"]


def test_lint_flags_a_young_scalar():
    for writer in ("v_readfirstlane_b32 s5, v3", "v_readlane_b32 s7, v3, 2", "v_cmp_gt_u32_e64 s[6:7], v3, v4", "v_add_co_u32_e64 v9, s[4:5], v3, v4"):
        for between, hazards in (([], 1), (["s_nop 1"], 1), (["s_nop 2"], 0), (["v_mov_b32_e32 v8, v9"] * 2, 1), (["v_mov_b32_e32 v8, v9"] * 3, 0)):
            assert len(find_young_scalars([writer] + between + LOAD + ["s_endpgm"])[1]) == hazards, (writer, between)
    # behind a loop's back edge, and on the taken side of a branch
    loop = [".LBB0_1:"] + LOAD + ["s_nop 4", "v_readfirstlane_b32 s4, v3", "s_cbranch_scc1 .LBB0_1", "s_endpgm"]
    side = ["v_readfirstlane_b32 s4, v3", "s_cbranch_scc1 .LBB0_1", "s_endpgm", ".LBB0_1:"] + LOAD + ["s_endpgm"]
    assert [len(find_young_scalars(x)[1]) for x in (loop, side)] == [1, 1]
    # another register, one written anew by the scalar unit, and loads the compiler knows
    assert find_young_scalars(["v_readfirstlane_b32 s8, v3"] + LOAD) == (1, [])
    assert find_young_scalars(["v_readfirstlane_b32 s4, v3", "s_mov_b32 s4, s20"] + LOAD) == (1, [])
    assert find_young_scalars(["v_readfirstlane_b32 s4, v3", LOAD[3]]) == (0, [])


def test_lint_flags_an_odd_load():
    assert find_odd_loads(LOAD) == []
    assert len(find_odd_loads([LOAD[0], LOAD[1], LOAD[3], LOAD[4]])) == 1
    assert len(find_odd_loads([LOAD[0], "\tglobal_load_dwordx4 v[10:13], v1, s[2:3]", LOAD[4]])) == 1
    assert len(find_odd_loads(LOAD[:3] + ["\tbuffer_load_dwordx4 v[10:13], v1, s[4:7], 0 offen", LOAD[4]])) == 1


def test_lint_flags_other_uses_of_m0():
    assert find_other_uses_of_m0(LOAD) == []
    for other in ("s_mov_b32 m0, s3", "s_add_i32 s4, m0, s5", "v_movrels_b32_e32 v3, v4", "s_set_gpr_idx_on s4, gpr_idx(SRC0)", "s_sendmsg_m0 m0",
                  "buffer_load_dword v1, s[4:7], 0 offen lds", "global_load_lds_dwordx4 v[2:3], off"):
        assert len(find_other_uses_of_m0(LOAD + [other])) == 1, other


@pytest.fixture(scope="module")
def grouped_unit_asm(tmp_path_factory):
    from paper_2605_19945_amd import build as moe_build
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("grouped_units")

    def compile_one(unit):
        path = out / (unit + ".s")
        r = subprocess.run([hipcc, *moe_build.FLAGS, "-S", "--cuda-device-only", "-o", str(path), os.path.join(moe_build.CSRC, unit + ".hip")],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        return path.read_text().splitlines()

    with ThreadPoolExecutor(len(UNITS)) as ex:
        return dict(zip(UNITS, ex.map(compile_one, UNITS)))


def test_no_hazard_around_the_loads_of_the_compiled_kernels(grouped_unit_asm):
    for unit, lines in grouped_unit_asm.items():
        n, young = find_young_scalars(lines)
        assert n > 50 and not young, f"{unit}:\n" + "\n".join(young[:10])
        odd = find_odd_loads(lines)
        assert not odd, f"{unit}:\n" + "\n".join(odd[:10])
        others = find_other_uses_of_m0(lines)
        assert not others, f"{unit}:\n" + "\n".join(others[:10])


def test_every_unit_with_loads_of_this_kind_is_looked_at():
    from paper_2605_19945_amd import build as moe_build
    with_engine = {u[:-len(".hip")] for u in moe_build.SOURCES if re.search(r'#include "moe_grouped(_stream)?\.h"', open(os.path.join(moe_build.CSRC, u)).read())}
    assert with_engine == set(UNITS) | {"moe_grouped"}  # (that one launches no kernel with loads)
