"""The build's scan of the generated code for a matrix instruction's result that is read too early
(no GPU, text only).  What the compiler itself once wrote for the sums of the fp32 GEMM, and what a
compiler could make of the explicit wait if nothing held it in its place."""
import pytest

from paper_2602_05754_amd.build import mfma_hazards

MFMA = "v_mfma_f32_16x16x4_f32 v[60:63], v17, v51, v[60:63]"
READ = "v_add_f32_e32 v44, v63, v26"
WAIT = "s_nop 15"


def found(*lines):
    return [ins for _, _, ins in mfma_hazards("kernel_a:\n" + "\n".join(lines) + "\ns_endpgm\n")]


def test_waits_and_barriers_are_no_wait_states():
    assert found(MFMA, "s_waitcnt lgkmcnt(0)", "s_barrier", "s_nop 7", READ) == [READ]
    assert found(MFMA, "s_waitcnt lgkmcnt(0)", "s_barrier", "s_nop 9", READ) == []


def test_the_wait_has_to_lie_between():
    assert found(MFMA, WAIT, READ) == []
    assert found(MFMA, READ, WAIT) == [READ]
    assert found(WAIT, MFMA, "v_mov_b32_e32 v1, v2", READ) == [READ]
    assert found(MFMA, WAIT, MFMA, READ) == [READ]
    assert found(MFMA, "ds_write_b128 v69, v[60:63] offset:16") == ["ds_write_b128 v69, v[60:63] offset:16"]
    assert found(MFMA, "v_mov_b32_e32 v63, v1", READ) == []                     # written anew in between


@pytest.mark.parametrize("op,states", [("v_mfma_f32_16x16x32_bf16", 8), ("v_mfma_f32_16x16x4_f32", 10), ("v_mfma_f64_16x16x4_f64", 18)])
def test_every_instruction_has_its_own_number_of_states(op, states):
    lines = f"{op} v[0:7], v[8:9], v[10:11], v[0:7]", "v_mov_b32_e32 v20, v3"
    assert found(lines[0], f"s_nop {states - 1}", lines[1]) == []
    assert found(lines[0], f"s_nop {states - 2}", lines[1]) == [lines[1]]


def test_paths_through_branches_and_loops_are_followed():
    loop = (".LBB0_1:", READ, WAIT, MFMA, "s_cbranch_scc1 .LBB0_1")             # only the second time round
    assert found(*loop) == [READ]
    assert found(".LBB0_1:", READ, MFMA, WAIT, "s_cbranch_scc1 .LBB0_1") == []
    assert found(MFMA, "s_cbranch_scc1 .LBB0_3", WAIT, "s_branch .LBB0_4", ".LBB0_3:", "v_mov_b32_e32 v1, v2", ".LBB0_4:", READ) == [READ]
    assert found(MFMA, "s_branch .LBB0_4", ".LBB0_3:", READ, ".LBB0_4:", "v_mov_b32_e32 v1, v2") == []


SHAPES = {"v_mfma_f32_32x32x16_bf16": (12, 8), "v_mfma_f32_32x32x2_f32": (18, 16), "v_mfma_f32_16x16x4_f32": (10, 8),
          "v_mfma_f32_16x16x32_bf16": (8, 4), "v_mfma_f64_16x16x4_f64": (18, 16)}


def matrix(op, first, last):
    return f"{op} v[{first}:{last}], v[200:203], v[204:207], v[{first}:{last}]"


@pytest.mark.parametrize("op", ["v_mfma_f32_32x32x16_bf16", "v_mfma_f32_32x32x2_f32"])
def test_the_tiles_of_32_rows_have_their_number_of_states(op):
    need, read = SHAPES[op][0], "v_mov_b32_e32 v120, v15"
    assert found(matrix(op, 0, 15), *["s_nop 0"] * need, read) == []
    assert found(matrix(op, 0, 15), *["s_nop 0"] * (need - 1), read) == [read]
    assert found(matrix(op, 0, 15).replace("v[0:15]", "a[0:15]"), "v_accvgpr_read_b32 v9, a7") == ["v_accvgpr_read_b32 v9, a7"]


@pytest.mark.parametrize("second", SHAPES)
@pytest.mark.parametrize("first", SHAPES)
def test_a_matrix_instruction_waits_for_the_one_before(first, second):
    """Right behind another it begins when that one has had the unit for its passes: those states have gone by with it, and no more."""
    need, passes = SHAPES[first]
    read = "v_mov_b32_e32 v120, v15"
    for between in (0, 1, passes // 2, passes - 1, passes, passes + 1):        # states between the two
        gone = max(between + 1, passes)                                        # when the second has been issued
        lines = [matrix(first, 0, 15)] + ["s_nop 0"] * between + [matrix(second, 32, 47)]
        left = max(need - gone, 0)
        assert found(*lines, *["s_nop 0"] * left, read) == []
        if left:
            assert found(*lines, *["s_nop 0"] * (left - 1), read) == [read]


def test_waits_and_barriers_do_not_free_the_unit():
    read, op = "v_mov_b32_e32 v120, v15", "v_mfma_f32_32x32x2_f32"
    assert found(matrix(op, 0, 15), "s_waitcnt lgkmcnt(0)", matrix(op, 32, 47), "s_nop 0", read) == [read]
    assert found(matrix(op, 0, 15), "s_waitcnt lgkmcnt(0)", matrix(op, 32, 47), "s_nop 1", read) == []


def test_a_taken_branch_is_one_state():
    read = "v_mov_b32_e32 v120, v15"
    for need, op in ((12, "v_mfma_f32_32x32x16_bf16"), (18, "v_mfma_f32_32x32x2_f32")):
        for branch in ("s_branch .LBB0_2", "s_cbranch_scc1 .LBB0_2"):
            lines = lambda n: (matrix(op, 0, 15), *["s_nop 0"] * n, branch, "s_nop 15", "s_nop 15", ".LBB0_2:", read)
            assert found(*lines(need - 1)) == [] and found(*lines(need - 2)) == [read]


@pytest.mark.parametrize("swap", [False, True])
def test_where_paths_meet_the_unit_is_the_one_that_is_free_sooner(swap):
    """On one path the first sum's instruction is four states ago, on the other another instruction has the unit for long: the matrix instruction
    behind them waits for no one on the first path."""
    read, short, long = "v_mov_b32_e32 v120, v3", matrix("v_mfma_f32_16x16x4_f32", 0, 3), matrix("v_mfma_f32_32x32x2_f32", 32, 47)
    near = [short, "s_nop 2"]                          # and the branch: four states, four to go for the unit, six for the sum
    busy = [short, "s_nop 15", long]
    one, other = (busy, near) if swap else (near, busy)
    join = [".LBB0_9:", matrix("v_mfma_f32_16x16x4_f32", 64, 67)]
    paths = lambda n: ["s_cbranch_scc1 .LBB0_5", *one, "s_branch .LBB0_9", ".LBB0_5:", *other, "s_branch .LBB0_9", *join, *["s_nop 0"] * n, read]
    assert found(*near, "s_nop 0", join[1], "s_nop 0", read) == [read]         # the first path alone: two states are missing
    assert found(*paths(1)) == [read] and found(*paths(2)) == []


FAKE_HIPCC = """#!/bin/sh
out=
while [ $# -gt 0 ]; do
  if [ "$1" = -o ]; then out=$2; shift; fi
  shift
done
if [ "$out" = - ]; then cat "$FAKE_ASSEMBLY"; exit 0; fi
echo new > "$out"
echo "a.hip:1:1: remark: Function Name: kernel_a [-Rpass-analysis=kernel-resource-usage]" >&2
echo "a.hip:1:1: remark:     ScratchSize [bytes/lane]: $FAKE_SCRATCH [-Rpass-analysis=kernel-resource-usage]" >&2
exit $FAKE_STATUS
"""


@pytest.mark.parametrize("scratch,lines,status,error", [("0", [MFMA, WAIT, READ], "0", None), ("8", [], "0", "scratch memory"), ("0", [MFMA, READ], "0", "too early"),
                                                        ("0", [], "1", "hipcc failed")])
def test_a_library_that_fails_a_check_takes_no_place(tmp_path, monkeypatch, scratch, lines, status, error):
    from paper_2602_05754_amd import build
    compiler, assembly, lib = tmp_path / "hipcc", tmp_path / "a.s", tmp_path / "libtf.so"
    compiler.write_text(FAKE_HIPCC)
    compiler.chmod(0o755)
    assembly.write_text("kernel_a:\n" + "\n".join(lines) + "\ns_endpgm\n")
    lib.write_text("old\n")
    for name, value in (("HIPCC", str(compiler)), ("FAKE_ASSEMBLY", str(assembly)), ("FAKE_SCRATCH", scratch), ("FAKE_STATUS", status)):
        monkeypatch.setenv(name, value)
    monkeypatch.setattr(build, "LIB", str(lib))
    if error is None:
        assert build.build() == str(lib) and lib.read_text() == "new\n"
    else:
        with pytest.raises(RuntimeError, match=error):
            build.build()
        assert lib.read_text() == "old\n"
    assert sorted(p.name for p in tmp_path.iterdir()) == ["a.s", "hipcc", "libtf.so"]
