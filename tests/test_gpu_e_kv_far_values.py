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


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("n", [1, 7, 160, 300])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", ["k_scale", "v_scale"])
def test_scales_that_are_no_number(what, d, n, value):
    """Queries that see a token of such a block get NaN, the others what they see: those before it,
    and those whose window has left it behind."""
    p = far.written([333, 333], [n, n], 2, 4, d, 16, "e4m3", "bf16", lambda v, r, pos: v)
    L, bad = 333, torch.zeros(333, dtype=torch.bool, device="cuda")
    bad[20 * 16:21 * 16] = True                          # the last block but one of the first request
    bad[9 * 16:10 * 16] = True
    for window in (0, 150, 330):
        want = far.attend(p, window=window)
        t = getattr(p["cache"], what)
        keep = t.clone()
        t[p["table"][0, [9, 20]].long(), 1] = value      # of the second kv head
        got = far.call(p, window=window)
        hs.hs_get_device_error()
        t.copy_(keep)
        hit = torch.zeros(got[1].shape, dtype=torch.bool, device="cuda")
        hit[:n, 4:] = (far.sees(L, n, True, window) & bad).any(1)[:, None]
        assert torch.isnan(got[0][hit].float()).all()
        assert torch.isnan(got[1][hit]).all() or what == "v_scale"
        far.compare(got, want, rows=~hit)


@pytest.mark.parametrize("n,L", [(1, 9000), (5, 300), (160, 700), (300, 333)])
@pytest.mark.parametrize("d", [64, 128])
def test_keys_that_are_no_number_everywhere(d, n, L):
    """Every row of such a request is NaN, in each of its parts; the next one is not touched."""
    p = far.written([L, 333], [n, n], 2, 4, d, 16, "e4m3", "bf16", lambda v, r, pos: v)
    want = far.attend(p)
    p["cache"].k_scale[p["table"][0, :-(-L // 16)].long()] = float("nan")
    got = far.call(p)
    hs.hs_get_device_error()
    assert torch.isnan(got[0][:n].float()).all() and torch.isnan(got[1][:n]).all()
    rows = torch.zeros(got[1].shape, dtype=torch.bool, device="cuda")
    rows[n:] = True
    far.compare(got, want, rows=rows)


@pytest.mark.parametrize("n,lens", [(1, [333, 50]), (7, [333, 50]), (160, [333, 180]), (300, [480, 310]),
                                    (1, [9000, 50]), (90, [2100, 300])])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_values_that_no_query_sees(d, n, lens):
    """NaN among the values that the windows of all of a request's queries have left behind, the
    last of them just now: they change nothing."""
    p = far.written(lens, [n, n], 2, 4, d, 16, "e4m3", "bf16", lambda v, r, pos: v)
    codes = p["cache"].v.view(torch.uint8)
    keep = codes.clone()
    for window in (1, 17, 150):
        first = lens[0] - n - window + 1
        if first < 1:
            continue
        for t in {first - 1, max(first - 9, 0), max(first - 100, 0), 0}:
            codes[p["table"][0, t // 16].long(), :, t % 16, t % d] = 0x7F
        far.check(p, window=window)
        codes.copy_(keep)


@pytest.mark.parametrize("n", [1, 7, 160, 300])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_values_that_are_no_number(d, n):
    """A NaN among the values: its column is NaN for the queries that see it; no other column, no
    lse, no other head and no other request."""
    L, t, col = 333, 332 - n // 2, 37
    p = far.written([L, L], [n, n], 2, 4, d, 16, "e4m3", "bf16", lambda v, r, pos: v)
    want = far.attend(p)
    p["cache"].v.view(torch.uint8)[p["table"][0, t // 16].long(), 1, t % 16, col] = 0x7F
    got = far.call(p)
    hs.hs_get_device_error()
    hit = far.sees(L, n, True, 0)[:, t]
    assert torch.isnan(got[0][:n][hit][:, 4:, col].float()).all()
    may = torch.zeros(p["q"].shape, dtype=torch.bool, device="cuda")
    may[:n, 4:, col] = True
    far.compare(got, want, columns=~may)
