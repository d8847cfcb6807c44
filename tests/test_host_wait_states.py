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


BIG, SMALL = "v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]", "v_mfma_f32_16x16x32_bf16 v[0:3], v[20:23], v[24:27], 0"
AGPR = "v_mfma_f32_32x32x16_bf16 a[0:15], v[20:23], v[24:27], a[0:15]"
OTHER = "v_mfma_f32_32x32x16_bf16 a[16:31], v[20:23], v[24:27], a[16:31]"


@pytest.mark.parametrize("lines, hits", [
    ((BIG, "s_nop 10", "v_add_f32_e32 v30, v3, v4"), 1), ((BIG, "s_nop 11", "v_add_f32_e32 v30, v3, v4"), 0),
    ((SMALL, "s_nop 6", "v_add_f32_e32 v30, v3, v4"), 1), ((SMALL, "s_nop 7", "v_add_f32_e32 v30, v3, v4"), 0),
    ((BIG, "v_mov_b32_e32 v15, 0"), 1), ((BIG, "ds_write_b128 v30, v[12:15]"), 1), ((BIG, "v_add_f32_e32 v30, v16, v17"), 0),
    ((BIG, BIG), 0), ((SMALL, SMALL), 0), ((AGPR, OTHER), 0), ((AGPR, "v_accvgpr_read_b32 v30, a7"), 1),
    ((BIG, "v_mfma_f32_32x32x16_bf16 a[0:15], v[4:7], v[24:27], a[0:15]"), 1),
    ((BIG, "v_mfma_f32_16x16x32_bf16 v[0:3], v[20:23], v[24:27], v[0:3]"), 1),
    ((AGPR, OTHER, OTHER, OTHER, "s_nop 3", "v_accvgpr_read_b32 v30, a7"), 1),
    (("loop:", "v_add_f32_e32 v30, v3, v4", "s_nop 7", BIG, "s_cbranch_scc1 loop", "s_endpgm"), 1)])
def test_reader_of_sums(lines, hits):
    assert len(list(W.sums(code(*lines)))) == hits


@pytest.mark.parametrize("lines, hits", [
    (("v_mov_b32_e32 v20, 0", BIG), 1), (("v_mov_b32_e32 v20, 0", "s_nop 0", BIG), 1), (("v_mov_b32_e32 v20, 0", "s_nop 1", BIG), 0),
    (("v_mov_b32_e32 v30, 0", BIG), 0), (("v_mov_b32_e32 v0, 0", BIG), 1), (("v_accvgpr_write_b32 a3, v9", AGPR), 1),
    (("ds_read_b128 v[20:23], v40", BIG), 0), (("v_dot2c_f32_bf16_e32 v20, v30, v31", BIG), 0)])
def test_reader_of_factors(lines, hits):
    assert len(list(W.factors(code(*lines)))) == hits


def test_sums_of_products(library):
    """A matrix product's sums are there when something else than a product that adds to them touches them: the kernels over a
    latent cache write their products in assembly, where the compiler keeps no distance by itself."""
    assert found_in(library, W.sums) == []


def test_factors_of_products(library):
    """A matrix product reads what a vector instruction wrote two wait states before or earlier."""
    assert found_in(library, W.factors) == []
