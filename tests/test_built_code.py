"""Wait states in the code that was built for gfx950, read from its disassembly.  The compiler keeps them in
the code that it makes; what is written out in assembly has to bring its own."""
import os
import re
import subprocess

import pytest

from paper_2604_21335_amd import build

LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
TARGET = "hipv4-amdgcn-amd-amdhsa--gfx950"
BRANCHES = re.compile(r"s_(c?branch|cbranch_\w+|setpc_b64|endpgm|trap)")
LINE = re.compile(r"^\s+(\S+)\s*(.*?)\s*// ([0-9A-F]{8,}):")


def _sgprs(operand):
    m = re.fullmatch(r"s(\d+)|s\[(\d+):(\d+)\]", operand)
    if not m:
        return {"vcc"} if operand in ("vcc", "vcc_lo", "vcc_hi") else set()
    return {int(m[1])} if m[1] else set(range(int(m[2]), int(m[3]) + 1))


def _operands(text):
    return [x.strip().split(" ")[0] for x in text.split(",")]


def _vector_writes(op, text):
    """Scalar registers that a vector instruction writes: a lane's value, a comparison's result, a carry."""
    if not op.startswith("v_"):
        return set()
    at = _operands(text)
    carries = re.match(r"v_(add_co|sub_co|subrev_co|addc_co|subb_co|subbrev_co|div_scale|mad_[ui]64)", op)
    return _sgprs(at[0]) | (_sgprs(at[1]) if carries and len(at) > 1 else set())


def _memory_reads(op, text):
    if not re.match(r"(buffer|global|flat|scratch|tbuffer)_", op):
        return set()
    return set().union(*(_sgprs(x) for x in _operands(text)))


def too_early(lines):
    """Vector memory instructions that read a scalar register less than five wait states behind a vector instruction that
    writes it (an instruction is one, s_nop n is n + 1), on any path: [(address, instruction, wait states)]."""
    code = []
    for line in lines:
        m = LINE.match(line)
        if m:
            code.append((int(m[3], 16), m[1], m[2]))
    at = {a: i for i, (a, _, _) in enumerate(code)}
    before = [[] for _ in code]
    for i, (a, op, text) in enumerate(code):
        if not re.fullmatch(r"s_(branch|endpgm|setpc_b64)", op) and i + 1 < len(code):
            before[i + 1].append(i)
        if re.match(r"s_c?branch", op):
            step = int(text.split()[0])
            target = at.get(a + 4 + 4 * (step - 65536 if step >= 32768 else step))
            if target is not None:
                before[target].append(i)
    found = []
    for i, (a, op, text) in enumerate(code):
        reads = _memory_reads(op, text)
        todo, seen = [(j, 0) for j in before[i]] if reads else [], {}
        while todo:
            j, states = todo.pop()
            if states >= 5 or seen.get(j, 5) <= states:
                continue
            seen[j] = states
            _, other, more = code[j]
            if _vector_writes(other, more) & reads:
                found.append((hex(a), op + " " + text, states))
                break
            states += int(more, 0) + 1 if other == "s_nop" else 1
            todo += [(k, states) for k in before[j]]
    return found


def test_the_search_finds_what_is_too_early():
    def code(*lines):
        return ["\t%s // %012X: 00000000" % (x, 0x1000 + 4 * i) for i, x in enumerate(lines)]
    first, load = "v_readfirstlane_b32 s20, v6", "buffer_load_dwordx4 v9, s[20:23], 0 offen lds"
    assert len(too_early(code(first, load))) == 1
    assert len(too_early(code(first, "s_mov_b32 m0, s2", "s_nop 0", load))) == 1
    assert len(too_early(code(first, "s_mov_b32 m0, s2", "s_nop 2", load))) == 1
    assert too_early(code(first, "s_mov_b32 m0, s2", "s_nop 3", load)) == []
    assert too_early(code("v_readfirstlane_b32 s24, v6", load)) == []
    assert too_early(code("s_mov_b32 s20, s3", load)) == []
    # around a branch: not in the text's order, and only there
    assert len(too_early(code("s_branch 2", load, "s_endpgm", first, "s_branch 65532"))) == 1
    assert too_early(code(first, "s_branch 1", load, "s_endpgm")) == []
    assert len(too_early(code("v_cmp_lt_i32_e64 s[4:5], v1, v2", "global_load_dword v1, v2, s[4:5]"))) == 1


@pytest.mark.parametrize("source", build.SOURCES)
def test_scalar_registers_are_there_for_memory_instructions(source, tmp_path):
    obj = os.path.join(build.BUILD_DIR, source.replace(".hip", ".o"))
    tools = [os.path.join(LLVM, x) for x in ("llvm-objcopy", "clang-offload-bundler", "llvm-objdump")]
    if not all(os.path.exists(x) for x in [obj, *tools]):
        pytest.skip("not built here, or no tools to look at it")
    fat, dev = str(tmp_path / "fat"), str(tmp_path / "dev.o")
    subprocess.run([tools[0], "--dump-section", ".hip_fatbin=" + fat, obj, os.devnull], check=True)
    subprocess.run([tools[1], "--unbundle", "--type=o", "--targets=" + TARGET, "--input=" + fat, "--output=" + dev],
                   check=True)
    text = subprocess.run([tools[2], "-d", "--mcpu=gfx950", dev], check=True, stdout=subprocess.PIPE, text=True).stdout
    lines = text.splitlines()
    if source != "stc_api.hip":
        assert sum("global_" in x or "buffer_" in x for x in lines) > 0
    found = too_early(lines)
    assert not found, (len(found), found[:5])
