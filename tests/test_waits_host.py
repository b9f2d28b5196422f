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


def missing_waits(asm):
    """(instructions that read M0, vector memory instructions and those too close behind a write of what they read) of an
    assembly."""
    readers, bad, since_m0, written = 0, [], 99, {}            # written: states since a vector write of a scalar register
    for line in asm.split("\n"):
        s = line.split(";")[0].strip()
        if not s or s[0] in ".#" or s.endswith(":"):
            continue
        op, _, operands = s.partition(" ")
        if READS_M0.match(s):
            readers += 1
            if since_m0 < 1:
                bad.append(s)
        if VECTOR_MEMORY.match(s) and any(written.get(r, 99) < 5 for r in scalar_regs(operands)):
            bad.append(s)
        states = 1 + int(operands) if op == "s_nop" else 1
        since_m0 += states
        written = {r: n + states for r, n in written.items() if n + states < 5}
        dst = operands.split(",")[:2 if SCALAR_SECOND.match(op) else 1]
        if op.startswith("s_"):
            if re.match(r"m0\b", operands.strip()) and not op.startswith("s_cmp"):
                since_m0 = 0
            written = {r: n for r, n in written.items() if r not in scalar_regs(dst[0])}
        elif op.startswith("v_"):
            written.update({r: 0 for d in dst for r in scalar_regs(d)})
    return readers, bad


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
                         (["\tv_cmp_lt_u32_e64 s[4:5], v1, v2", load], 1)):
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
    readers, bad = missing_waits(assemblies[name])
    assert readers > 0 and not bad, (len(bad), bad[:3])


@pytest.mark.parametrize("name", SOURCES)
def test_the_compiler_keeps_nothing_in_m0(assemblies, name):
    used = [s for s in outside_inline(assemblies[name]) if re.search(r"\bm0\b", s) or READS_M0.match(s) or "set_gpr_idx" in s]
    assert not used, used[:3]
    assert "m0" not in "".join(outside_inline("\t;;#ASMSTART\n\ts_mov_b32 m0, s1\n\t;;#ASMEND\n\ts_nop 0"))
