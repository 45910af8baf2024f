"""Rows in 8 bits where there are many: norms whose blocks take several rows, with gates that change among them, and rows to codes and back past a
launch's 2^20 blocks.  As tests/test_gpu_q8.py holds the small ones."""
import pytest
import torch

import paper_2210_17223_amd as moe
import test_gpu_q8 as q8
from gpu_util import DEV

pytestmark = pytest.mark.gpu


# rows enough that every block has three: 4096 wavefronts at a time up to 512 columns, 1024 blocks up to 2048, 512 up to 4096, else 256
@pytest.mark.parametrize("T,d", [(8200, 64), (8195, 512), (2050, 528), (2500, 768), (2049, 2048), (1100, 2064), (1300, 4096), (515, 4112), (600, 8192),
                                 (514, 8208), (520, 16384)])
@pytest.mark.parametrize("kind,res,z,bias,gate_tokens", [("rms", "f32", "f16", False, 2), ("layer", "bf16", "bf16", True, 5),
                                                         ("rms", "bf16", "f32", False, 1), ("layer", "f32", "f32", True, 7),
                                                         ("layer", "f32", "bf16", True, 0), ("rms", "bf16", "f16", False, 4)])
def test_norms_of_several_rows_a_block(T, d, kind, res, z, bias, gate_tokens):
    q8.test_norms_write_the_codes_of_their_fp32_rows(T, d, kind, res, z, bias, gate_tokens)


# (a wavefront a row from 2048 rows of 1040 to 2048 values on)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,K", [(4096, 2048), (2049, 1040), (2048, 1536), (3001, 4096), (2048, 8192)])
def test_many_rows_are_the_rounded_quotients(R, K, dtype):
    q8.test_rows_are_the_rounded_quotients(R, K, dtype)


def repeated(base, R):
    return base.repeat(-(-R // base.shape[0]), *[1] * (base.dim() - 1))[:R].contiguous()


def same_again(got, base):
    """got's rows are base's over and over."""
    n, whole = base.shape[0], got.shape[0] // base.shape[0]
    return torch.equal(got[:whole * n].view(whole, *base.shape), base.expand(whole, *base.shape)) and torch.equal(got[whole * n:], base[:got.shape[0] - whole * n])


@pytest.mark.parametrize("R,K", [((1 << 22) + 9, 16), ((1 << 20) + 5, 2064)])
def test_rows_past_a_launchs_blocks(R, K):
    """A block's second rows: of wavefronts, and of blocks, whose largest values meet in LDS in turn."""
    base = q8.normal(q8.gen(K), 1021, K, std=3.0).bfloat16()
    x = repeated(base, R)
    q, s = torch.full((R, K), 99, dtype=torch.int8, device=DEV), torch.full((R,), -1.0, device=DEV)
    moe.moe_q8_rows(x, q, s)
    code, scale = q8.held(base)
    assert same_again(q, code) and same_again(s, scale)


def test_values_past_a_launchs_blocks():
    R, K = (1 << 20) + 3, 8208
    g = q8.gen(K)
    base, scale = q8.codes(g, 1021, K), q8.scales(g, 1021, of=0.01)
    x = torch.empty(R, K, dtype=torch.float16, device=DEV)
    moe.moe_q8_values(repeated(base, R), repeated(scale, R), x)
    want = (base.float() * scale[:, None]).half()
    at = torch.cat([torch.arange(0, R, 4099, device=DEV), torch.arange(R - 8, R, device=DEV)])
    assert torch.equal(x[at], want[at % 1021])
