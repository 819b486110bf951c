"""The wait states behind the matrix instruction of 8- and 4-bit elements, on the built instructions: its
result may not be touched by another instruction for its passes of 4 clocks, plus 4. The compiler counts
too few of them behind a branch, so the kernel waits by itself."""
import codeobj
import test_host_matrix_waits as waits
from paper_2008_03602_amd import _lib as L

SCALED = "v_mfma_scale_f32_16x16x128_f8f6f4"


def test_results_of_microscaled_products_are_left_alone_for_their_wait(monkeypatch):
    kernels = checked = 0
    for sym, rows in codeobj.instructions(L.LIB_PATH, "mx_linear_kernel"):
        # kernel<weights, x, exact sums, ...>: with an 8-bit operand 8 passes, of two 4-bit ones 4
        eight = "ILi2E" in sym or "ELi2ELb" in sym
        monkeypatch.setitem(waits.WAITS, SCALED, (8 if eight else 4) + 4)
        kernels += 1
        for i, r in enumerate(rows):
            if r[1] in waits.WAITS:
                checked += 1
                early = list(waits._early_touches(rows, i))
                assert not early, (sym, hex(r[0]), r[1], early)
    assert kernels >= 30 and checked >= 2 * kernels
