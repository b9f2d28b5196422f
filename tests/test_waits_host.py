"""Host analysis (no GPU) of the compiled kernels that load to LDS from inline statements: the wait states that such a
load needs behind the writes of what it reads, which the compiler puts in for its own instructions and cannot put into
an inline statement.

  a scalar write of M0, which says where in LDS the data go                   one wait state
  a vector instruction's write of the scalar registers that hold an address    five

Every instruction is a wait state, s_nop n is n + 1 of them.  The statements do not save M0: nothing outside of inline
statements may use it in these kernels."""
import concurrent.futures
import glob
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_00891_amd", "csrc")
READS_M0 = re.compile(r"^(global_load_lds_|buffer_load_.*\blds\b|s_movrel|v_movrel|s_sendmsg|ds_\w*(gws|addtid))")


VECTOR_MEMORY = re.compile(r"^(global_|buffer_|flat_|scratch_)")
SCALAR_SECOND = re.compile(r"^v_((add|sub|subrev|addc|subb|subbrev)_co_|div_scale|mad_[ui]64)")


def scalar_regs(text):
    out = set()
    for a, b, c in re.findall(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b", text):
        out |= {int(c)} if c else set(range(int(a), int(b) + 1))
    return out


def missing_waits(body):
    """(instructions that read M0, those and vector memory instructions too close behind a write of what they read, on any
    path) of one kernel's assembly."""
    ins, labels = [], {}
    for line in body.split("\n"):
        s = line.split(";")[0].strip()
        label = re.match(r"^(\.LBB\S+):", s)
        if label:
            labels[label.group(1)] = len(ins)
        elif s and s[0] not in ".#" and not s.endswith(":"):
            ins.append(s)
    # before each instruction: states since M0 was written, and since a vector instruction wrote a scalar register
    state, work, bad = {0: (99, {})}, [0], set()
    while work:
        i = work.pop()
        if i >= len(ins):
            continue
        s, (since_m0, written) = ins[i], state[i]
        op, _, operands = s.partition(" ")
        if READS_M0.match(s) and since_m0 < 1:
            bad.add(i)
        if VECTOR_MEMORY.match(s) and any(written.get(r, 99) < 5 for r in scalar_regs(operands)):
            bad.add(i)
        states = 1 + int(operands) if op == "s_nop" else 1
        since_m0 = min(99, since_m0 + states)
        written = {r: n + states for r, n in written.items() if n + states < 5}
        dst = operands.split(",")[:2 if SCALAR_SECOND.match(op) else 1]
        if op.startswith("s_") and not re.match(r"s_(bit)?cmp", op):
            if re.match(r"m0\b", operands.strip()):
                since_m0 = 0
            written = {r: n for r, n in written.items() if r not in scalar_regs(dst[0])}
        elif op.startswith("v_"):
            written.update({r: 0 for d in dst for r in scalar_regs(d)})
        branch = re.match(r"^s_(c?branch\S*)\s+(\.LBB\S+)", s)
        if branch:
            nxt = [labels[branch.group(2)]] + ([i + 1] if branch.group(1).startswith("cbranch") else [])
        else:
            nxt = [] if op == "s_endpgm" else [i + 1]
        for t in nxt:
            old = state.get(t, (99, {}))
            new = (min(old[0], since_m0), {r: min(old[1].get(r, 99), written.get(r, 99)) for r in {*old[1], *written}})
            if t not in state or new != old:
                state[t] = new
                work.append(t)
    return sum(READS_M0.match(s) is not None for s in ins), [ins[i] for i in sorted(bad)]


def test_analysis_counts_wait_states():
    load = "\tglobal_load_lds_dwordx4 v2, s[4:5] nt"
    for lines, wrong in ((["\ts_mov_b32 m0, s3", load], 1), (["\ts_mov_b32 m0, s3", "\ts_nop 0", load], 0),
                         (["\ts_mov_b32 m0, s3", ".LBB0_1:", "\t; a comment", load], 1),
                         (["\ts_add_u32 m0, m0, 0x400", load], 1), (["\ts_mov_b32 s3, m0", load], 0),
                         (["\ts_mov_b32 m0, s3", "\ts_mov_b64 exec, 15", load, "\ts_mov_b32 m0, s6"], 0),
                         (["\tv_readfirstlane_b32 s5, v9", "\ts_mov_b32 m0, s3", "\ts_nop 2", load], 1),
                         (["\tv_readfirstlane_b32 s5, v9", "\ts_mov_b32 m0, s3", "\ts_nop 3", load], 0),
                         (["\tv_readfirstlane_b32 s3, v9", "\ts_mov_b32 m0, s3", "\ts_nop 0", load], 0),
                         (["\tv_cmp_lt_u32_e64 s[4:5], v1, v2", "\ts_mov_b64 s[4:5], s[8:9]", load], 0),
                         (["\tv_cmp_lt_u32_e64 s[4:5], v1, v2", load], 1),
                         (["\tv_readlane_b32 s4, v1, 3", "\ts_cmp_lg_u32 s4, 0", load], 1),
                         (["\tv_readlane_b32 s4, v1, 3", "\ts_cbranch_scc1 .LBB0_2", "\ts_nop 7", ".LBB0_2:", load], 1),
                         (["\ts_nop 0", ".LBB0_2:", load, "\ts_mov_b32 m0, s3", "\ts_cbranch_scc1 .LBB0_2"], 0),
                         ([".LBB0_2:", load, "\ts_cbranch_scc0 .LBB0_3", "\tv_readlane_b32 s5, v1, 3", "\ts_branch .LBB0_2",
                           ".LBB0_3:", "\ts_endpgm"], 1)):
        readers, bad = missing_waits("\n".join(lines))
        assert readers == 1 and len(bad) == wrong, lines


def outside_inline(asm):
    """The instructions of an assembly that the compiler made itself."""
    inline, out = False, []
    for line in asm.split("\n"):
        if "#ASMSTART" in line or "#ASMEND" in line:
            inline = "#ASMSTART" in line
        elif not inline:
            out.append(line.split(";")[0].strip())
    return out


def loads_to_lds(path):
    text = open(path).read()
    return "global_load_lds" in text or any(loads_to_lds(os.path.join(CSRC, h)) for h in re.findall(r'#include "(cb_\w+\.h)"', text))


SOURCES = sorted(os.path.basename(s) for s in glob.glob(os.path.join(CSRC, "*.hip")) if loads_to_lds(s))


@pytest.fixture(scope="module")
def assemblies(tmp_path_factory):
    sys.path.insert(0, os.path.dirname(CSRC))
    try:
        import build as lib_build
    finally:
        sys.path.pop(0)
    out = tmp_path_factory.mktemp("asm")

    def compile_one(name):
        s = str(out / (name + ".s"))
        subprocess.run([lib_build._hipcc()] + lib_build.COMMON + ["-x", "hip", "-S", "--cuda-device-only",
                       os.path.join(CSRC, name), "-o", s], check=True, capture_output=True)
        return open(s).read()

    with concurrent.futures.ThreadPoolExecutor(max_workers=8) as ex:
        return dict(zip(SOURCES, ex.map(compile_one, SOURCES)))


def test_every_source_with_such_loads_is_looked_at():
    assert {"cb_apply.hip", "cb_apply_multi.hip", "cb_attn.hip", "cb_attn_paged.hip", "cb_stats.hip", "cb_stats_centered.hip",
            "cb_stats_multi.hip", "cb_stats_rope.hip"} <= set(SOURCES)


@pytest.mark.parametrize("name", SOURCES)
def test_loads_to_lds_wait_for_what_they_read(assemblies, name):
    readers = 0
    for kernel, body in re.findall(r"(?ms)^(_Z\S+):.*?\n(.*?)^\.Lfunc_end", assemblies[name]):
        n, bad = missing_waits(body)
        readers += n
        assert not bad, (kernel, len(bad), bad[:3])
    assert readers > 0


@pytest.mark.parametrize("name", SOURCES)
def test_the_compiler_keeps_nothing_in_m0(assemblies, name):
    used = [s for s in outside_inline(assemblies[name]) if re.search(r"\bm0\b", s) or READS_M0.match(s) or "set_gpr_idx" in s]
    assert not used, used[:3]
    assert "m0" not in "".join(outside_inline("\t;;#ASMSTART\n\ts_mov_b32 m0, s1\n\t;;#ASMEND\n\ts_nop 0"))
