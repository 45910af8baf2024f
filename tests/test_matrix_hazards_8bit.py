"""The wait states of the 8-bit matrix instruction, as tests/test_matrix_hazards.py looks for those of the others: planted listings, and the
kernels of 8-bit products in the library as built."""
import re

import pytest

import test_matrix_hazards as hazards
from test_matrix_hazards import library  # noqa: F401 (a fixture)

# v_mfma_i32_16x16x64_i8 takes as long as the 16-bit instruction of half its depth: four passes, results visible as late
hazards.MATRIX.setdefault("16x16x64", (4, True))
I8 = "v_mfma_i32_16x16x64_i8 a[0:3], v[8:11], v[4:7], a[0:3]"
ZERO = "v_mfma_i32_16x16x64_i8 a[0:3], v[8:11], v[4:7], 0"


@pytest.mark.parametrize("code,bad", [
    (["v_mov_b32_e32 v4, v9", I8], 1), (["v_mov_b32_e32 v4, v9", "s_nop 1", I8], 0), (["v_mov_b32_e32 v12, v9", ZERO], 0),
    ([I8, "v_accvgpr_read_b32 v0, a3"], 1), ([I8, "s_nop 7", "v_accvgpr_read_b32 v0, a3"], 0), ([I8, "s_nop 6", "v_accvgpr_read_b32 v0, a3"], 1),
    ([ZERO, "s_nop 6", "v_accvgpr_write_b32 a2, v0"], 1), ([I8, I8, I8], 0), ([ZERO, I8], 0),
    ([I8, "v_mfma_i32_16x16x64_i8 a[2:5], v[8:11], v[4:7], a[2:5]"], 1), ([I8, "ds_write_b128 v0, a[0:3]"], 1),
    ([I8, "v_mov_b32_e32 v4, v9", "s_cbranch_scc1 65533 @0x0", "s_endpgm"], 1),
])
def test_the_check_sees_planted_hazards(code, bad):
    assert len(hazards.hazards(hazards.listing(*code))) == bad


def test_no_8_bit_matrix_instruction_of_the_library_is_too_close(library):  # noqa: F811
    found = {n: f for n, f in library.items() if any("16x16x64_i8" in i.name for i in f)}
    kinds = {re.search(r"q8_[a-z_]+_kernel", n)[0] for n in found}
    assert kinds == {"q8_stream_kernel", "q8_tile_kernel", "q8_small_run_kernel", "q8_gated_small_run_kernel", "q8_run_kernel", "q8_gated_run_kernel"}
    assert all(i.name == "v_mfma_i32_16x16x64_i8" for f in found.values() for i in f if hazards.is_matrix(i))
    bad = {n: h for n, f in found.items() if (h := hazards.hazards(f))}
    assert not bad, "\n".join(f"{n}: {len(h)}, e.g. {h[0][0]} -> {h[0][1]}" for n, h in bad.items())
