"""Which of the norms' kernels in 8 bits hold their rows in registers, read from the library as built (no GPU needed): all for rows up to 8192 and all
in front of the first block; behind a block the wider ones spill, as norm.hip says beside them."""
import re
import shutil
import subprocess

import pytest

import paper_2210_17223_amd as moe

OBJDUMP, READELF = "/opt/rocm/llvm/bin/llvm-objdump", "/opt/rocm/llvm/bin/llvm-readelf"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{(behind a block, threads of a row, columns of a thread): (registers, of them spilled), the most over the types}"""
    moe.lib()                                       # (built if it is not there)
    if shutil.which(OBJDUMP) is None or shutil.which(READELF) is None:
        pytest.skip("no llvm tools")
    where = tmp_path_factory.mktemp("code")
    shutil.copy(moe.lib_path(), where / "libmoe.so")
    subprocess.run([OBJDUMP, "--offloading", "libmoe.so"], cwd=where, check=True, capture_output=True)
    out = {}
    for f in sorted(where.glob("*gfx950")):
        notes = subprocess.run([READELF, "--notes", str(f)], check=True, capture_output=True, text=True).stdout
        for entry in re.split(r"\n  - (?=\.)", notes)[1:]:
            kernel = re.search(r"norm_q8_kernelILi\d+ELi(n?)\d+ELi(\d+)ELi(\d+)E", entry)
            if kernel:
                key = (kernel[1] == "", int(kernel[2]), int(kernel[3]))
                has = [int(re.search(rf"\.{what}: +(\d+)", entry)[1]) for what in ("vgpr_count", "vgpr_spill_count", "private_segment_fixed_size")]
                out[key] = tuple(map(max, zip(out.get(key, (0, 0, 0)), has)))
    return out


def test_rows_that_fit_the_registers_stay_there(kernels):
    few, many = {(256, 4), (512, 4), (1024, 4)}, {(64, 8), (256, 8), (512, 8), (1024, 8)}
    assert {k[1:] for k in kernels} == few | many | {(1024, 16)} and len(kernels) == 16
    for (after, *shape), (registers, spilled, scratch) in kernels.items():
        if tuple(shape) == (1024, 16) and after:
            assert spilled <= 96
        else:
            assert spilled == 0 and scratch == 0 and registers <= 128, (after, shape, registers, spilled)
