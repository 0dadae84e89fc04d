"""hs_kv_attend at the ends of 31 bits: windows that reach back past the first
token by more than positions can say, and rows of a table that would hold as
many tokens."""
import pytest
import torch

import kv_far_testutil as far

BT = 128
WIDTH = (1 << 31) // BT - 4                            # 2^31 - 512 tokens, the most there may be


@pytest.mark.gpu
@pytest.mark.parametrize("n,lens", [(800, [20, 900]), (3, [2, 40]), (601, [0, 601])])
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_window_of_nearly_all(n, lens, G, d):
    """It hides nothing, whatever stands before the first token."""
    p = far.written(lens, [n, n], 1, G, d, BT, "e4m3", "bf16", lambda v, r, pos: v)
    want = far.attend(p)
    table = torch.full((2, WIDTH), -1, dtype=torch.int32, device="cuda")
    table[:, :p["table"].shape[1]] = p["table"]
    for less in (1, 88, 500, n):
        far.compare(far.call(dict(p, table=table), window=WIDTH * BT - less), want)
