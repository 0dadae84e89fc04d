"""hs_kv_attend where the blocks' value scales lie far apart: blocks of zeros,
which hs_kv_append gives the least scale, blocks far larger than the others,
and scales that are no number."""
import numpy as np
import pytest
import torch

import kv_far_testutil as far
import kv_testutil as ref
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu

# Requests of few and of many rows; of the latter several whole ones a block, and ones in parts.
SHAPES = {
    "tokens": ([300, 129, 700], [1, 1, 1]),
    "parts": ([700], [160]),
    "whole": ([200 + i for i in range(50)], [24 + i % 3 for i in range(50)]),
}
ZERO = {
    "first": lambda v, r, pos: torch.where((pos < 128)[:, None, None], 0.0, v),
    "others": lambda v, r, pos: torch.where((pos // 128 % 2 == 1)[:, None, None], 0.0, 1000 * v),
    "last": lambda v, r, pos: torch.where((pos >= 128)[:, None, None], 0.0, 1000 * v),
    "head": lambda v, r, pos: v * torch.tensor([0.0, 1.0], device="cuda")[:, None],
    "all": lambda v, r, pos: 0.0 * v,
}


@pytest.mark.parametrize("which", sorted(ZERO))
@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("d,bt,fmt,dtype", [(64, 16, "e4m3", "bf16"), (128, 128, "e4m3", "fp16"),
                                            (128, 64, "int8", "bf16"), (64, 128, "int8", "fp16")])
def test_blocks_of_zeros(which, shape, d, bt, fmt, dtype):
    lens, n = SHAPES[shape]
    far.check(far.written(lens, n, 2, 4, d, bt, fmt, dtype, ZERO[which], size=3.0))


def wild(lens, n, H, G, d, bt, fmt, spread, seed=1):
    """Random codes, value scales 2^-spread to 2^spread."""
    p = far.written(lens, n, H, G, d, bt, fmt, "bf16", lambda v, r, pos: v, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = p["cache"].v_scale
    s.copy_(torch.exp2(torch.randint(-spread, spread + 1, s.shape, generator=g, device="cuda").float()))
    return p


@pytest.mark.parametrize("shape", ["parts", "whole"])
@pytest.mark.parametrize("d,fmt", [(64, "int8"), (128, "e4m3")])
@pytest.mark.parametrize("spread", [30, 100])
def test_scales_far_apart_many_rows(shape, d, fmt, spread):
    lens, n = SHAPES[shape]
    far.check(wild(lens, n, 2, 4, d, 16, fmt, spread))


@pytest.mark.parametrize("lens,n", [([300, 129, 700], [1, 1, 1]), ([900], [7]), ([9000, 40], [1, 3])])
@pytest.mark.parametrize("d,fmt", [(64, "int8"), (128, "e4m3"), (256, "e4m3")])
@pytest.mark.parametrize("spread", [30, 100])
def test_scales_far_apart_few_rows(lens, n, d, fmt, spread):
    far.check(wild(lens, n, 2, 4, d, 16, fmt, spread))


@pytest.mark.parametrize("n", [4, 8, 160])
@pytest.mark.parametrize("d,fmt", [(64, "int8"), (128, "e4m3"), (256, "int8")])
@pytest.mark.parametrize("up", [28, 32, 90])
def test_a_far_larger_block_that_is_hidden(n, d, fmt, up):
    """The last block is 2^up times the others; its tokens are the last four, which the queries
    before them do not see, nor any query with a window those of the first block."""
    p = far.written([324], [n], 2, 4, d, 16, fmt, "bf16", lambda v, r, pos: v)
    p["cache"].v_scale[p["table"][0, -1].long()] *= 2.0 ** up
    far.check(p)
    p["cache"].v_scale[p["table"][0, 0].long()] *= 2.0 ** up
    far.check(p, window=120)


@pytest.mark.parametrize("n", [1, 160])
@pytest.mark.parametrize("d,fmt", [(64, "int8"), (128, "e4m3"), (256, "int8")])
@pytest.mark.parametrize("up", [28, 32, 60])
def test_a_far_larger_block_of_no_weight(n, d, fmt, up):
    """Every query sees the block that is 2^up times the others, under a score 300 below theirs."""
    p = far.written([400, 90], [n, min(n, 90)], 2, 4, d, 16, fmt, "bf16", lambda v, r, pos: v)
    p["q"].abs_().clamp_(min=0.25)
    c = p["cache"]
    for r in range(2):
        b = p["table"][r, 1].long()
        c.k.view(torch.uint8)[b] = 0xF8 if fmt == "e4m3" else 256 - 64       # -256, -64
        c.k_scale[b] = 300 / (0.25 * (256 if fmt == "e4m3" else 64) * d ** 0.5)
        c.v_scale[b] *= 2.0 ** up
    far.check(p)


@pytest.mark.parametrize("n", [1, 160])
@pytest.mark.parametrize("up", [119, -125])
def test_ends_of_the_range(n, up):
    """Values near the largest and the smallest numbers of bf16."""
    p = far.written([400, 90], [n, min(n, 90)], 2, 4, 128, 16, "e4m3", "bf16", lambda v, r, pos: v)
    p["cache"].v_scale.fill_(2.0 ** up)
    far.check(p)
