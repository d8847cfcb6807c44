"""Wait states in the built library's code, read from its listing, and the reader itself on short listings."""
import pytest

import wait_states as W


def code(*lines):
    """A function of these lines; "name:" marks the next one, and a branch names where it goes."""
    marks, rows = {}, []
    for line in lines:
        if line.endswith(":"):
            marks[line[:-1]] = len(rows)
        else:
            rows.append(line)
    out = []
    for line in rows:
        name, _, rest = line.partition(" ")
        out.append(W.Instruction(line, marks[rest] if "branch" in name else None))
    return out


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    """(function, its instructions) of everything in the library."""
    found = []
    for i, obj in enumerate(W.code_objects()):
        found += W.functions(W.listing(obj, str(tmp_path_factory.mktemp(f"code{i}"))))
    return found


def found_in(library, rule):
    return [f"{name}: {i.text} | {j.text} ({states} apart)" for name, code in library for i, j, states in rule(code)]


def test_the_whole_library_is_read(library):
    names = " ".join(name for name, _ in library)
    for kernel in ("latent_attn_kernel", "latent_few_kernel", "attn_stream_kernel", "attn_split_kernel", "attn_few_kernel",
                   "rope_kernel", "argmax_partial_kernel"):
        assert kernel in names
    loads = sum(i.name.startswith("global_load_lds") for _, code in library for i in code)
    assert loads > 1000, loads


def test_registers():
    i = W.Instruction("v_mfma_f32_32x32x16_bf16 a[0:15], v[2:5], v[10:13], a[0:15]")
    assert i.writes == {("a", r) for r in range(16)} and ("v", 13) in i.reads and ("a", 3) in i.reads and ("v", 6) not in i.reads
    i = W.Instruction("global_load_lds_dwordx4 v1, s[2:3] offset:128")
    assert i.writes == set() and i.reads == {("v", 1), ("s", 2), ("s", 3)}
    i = W.Instruction("v_add_co_u32_e32 v4, vcc, s7, v4")
    assert i.writes == {("v", 4), "vcc"} and i.reads == {("s", 7), ("v", 4)}
    assert W.Instruction("s_nop 7").states == 8 and W.Instruction("s_mov_b32 m0, s4").writes == {"m0"}


LOAD, SET = "global_load_lds_dwordx4 v[2:3], off", "s_mov_b32 m0, s4"


@pytest.mark.parametrize("lines, hits", [
    ((SET, LOAD), 1), ((SET, "s_nop 0", LOAD), 0), ((SET, "v_mov_b32_e32 v1, 0", LOAD), 0),
    (("loop:", LOAD, SET, "s_cbranch_scc1 loop", "s_endpgm"), 0), (("loop:", LOAD, "s_nop 0", SET, "s_branch loop"), 0),
    ((SET, "global_load_dwordx4 v[4:7], v[2:3], off"), 0)])
def test_reader_of_direct_loads(lines, hits):
    assert len(list(W.lds_load(code(*lines)))) == hits


@pytest.mark.parametrize("lines, hits", [
    (("v_readfirstlane_b32 s2, v1", "global_load_dword v4, v5, s[2:3]"), 1),
    (("v_readfirstlane_b32 s2, v1", "s_nop 3", "global_load_dword v4, v5, s[2:3]"), 1),
    (("v_readfirstlane_b32 s2, v1", "s_nop 4", "global_load_dword v4, v5, s[2:3]"), 0),
    (("v_readfirstlane_b32 s2, v1", "global_load_dword v4, v5, s[4:5]"), 0),
    (("loop:", "global_load_dword v4, v5, s[2:3]", "v_readlane_b32 s3, v1, 7", "s_cbranch_vccnz loop", "s_endpgm"), 1),
    (("s_mov_b32 s2, s8", "global_load_dword v4, v5, s[2:3]"), 0)])
def test_reader_of_scalar_bases(lines, hits):
    assert len(list(W.scalar_base(code(*lines)))) == hits


def test_direct_loads(library):
    """M0 is written a wait state before a load takes its place in LDS from it."""
    assert found_in(library, W.lds_load) == []


def test_scalar_bases(library):
    """A memory instruction reads scalar registers that a vector instruction wrote five wait states before or earlier."""
    assert found_in(library, W.scalar_base) == []
