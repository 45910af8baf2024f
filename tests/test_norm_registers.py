"""Which of the norms' kernels hold their rows in registers: scratch memory per lane, read from the library as built (no GPU
needed).  Forward kernels for rows up to 8192 spill nothing; backward ones for rows up to 4096 at most what eight bf16 columns a thread
with biases take; the wider ones spill, as norm.hip says beside them."""
import re
import shutil
import subprocess

import pytest

import paper_2210_17223_amd as moe

OBJDUMP, READELF = "/opt/rocm/llvm/bin/llvm-objdump", "/opt/rocm/llvm/bin/llvm-readelf"


@pytest.fixture(scope="module")
def scratch(tmp_path_factory):
    """{(pass, threads of a row, columns of a thread): most bytes of scratch per lane over the types}"""
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
            kernel = re.search(r"norm_(forward|backward)_kernelILi\d+ELin?\d+ELi(\d+)ELi(\d+)E", entry)
            if kernel:
                key = (kernel[1], int(kernel[2]), int(kernel[3]))
                out[key] = max(out.get(key, 0), int(re.search(r"\.private_segment_fixed_size: +(\d+)", entry)[1]))
    return out


def test_rows_that_fit_the_registers_stay_there(scratch):
    forward = {k[1:]: v for k, v in scratch.items() if k[0] == "forward"}
    assert {k: v for k, v in forward.items() if k[0] * k[1] <= 8192} == {(64, 8): 0, (256, 8): 0, (256, 16): 0, (512, 16): 0}
    backward = {k[1:]: v for k, v in scratch.items() if k[0] == "backward" and k[1] * k[2] <= 4096}
    assert set(backward) == {(64, 4), (64, 8), (256, 4), (256, 8), (512, 4), (512, 8), (1024, 4)}
    assert all(v <= 64 for v in backward.values()), backward
