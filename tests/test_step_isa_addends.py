"""As test_step_isa.py, of the sums that a matrix instruction adds to: none of the
two wait states before one writes them other than by a matrix instruction."""

from __future__ import annotations

from test_step_isa import analyse, kernels, operands, registers  # noqa: F401  (kernels: a fixture)


def test_no_sum_is_written_right_before(kernels):  # noqa: F811
    for name, code in kernels.items():
        _, near = analyse(code)
        for i, (_, text) in enumerate(code):
            if text.startswith("v_mfma"):
                assert not registers(operands(text)[3]) & (near[i][0] | near[i][1]), (name, text)


def test_one_would_be_found():
    """The look itself: the zeroing of a sum one instruction before its matrix instruction, three before, and on
    a path that jumps to it."""
    mma = "v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]"

    def found(lines):
        code = [(4 * n, text) for n, text in enumerate(lines)]
        _, near = analyse(code)
        return any(registers(operands(t)[3]) & (near[i][0] | near[i][1]) for i, (_, t) in enumerate(code) if t.startswith("v_mfma"))

    assert found(["v_accvgpr_write_b32 a2, 0", mma, "s_endpgm"])
    assert found(["v_accvgpr_write_b32 a2, 0", "s_nop 0", mma, "s_endpgm"])
    assert found(["v_accvgpr_write_b32 a2, 0", "s_branch 1", "s_endpgm", mma, "s_endpgm"])
    assert not found(["v_accvgpr_write_b32 a2, 0", "s_nop 1", mma, "s_endpgm"])
    assert not found(["v_accvgpr_write_b32 a4, 0", mma, mma, "s_endpgm"])
