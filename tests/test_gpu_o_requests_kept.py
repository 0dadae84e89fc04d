"""What KvRequests keeps hold of where requests part: tokens of a step that is
not appended yet."""
import pytest
import torch

import pages_testutil as ref
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu
H, D, BT = 2, 64, 16


def begun(lens, most=8, n_blocks=64):
    """Requests whose prompts are appended, and what was."""
    cache = hs.KvCache(n_blocks, BT, H, D, torch.int8)
    req = hs.KvRequests(cache, max_requests=most, max_len=160)
    tokens = torch.arange(len(lens) * max(lens), **ref.INT).view(len(lens), max(lens))
    _, _, unique_idx, inverse = req.begin(tokens, ref.dev(lens))
    kv = torch.randn((tokens.numel(), H, D), generator=ref.gen(1), device="cuda").to(torch.bfloat16)
    req.append(cache, kv, kv)
    return cache, req, unique_idx, inverse, kv


@pytest.mark.parametrize("how", ["fork", "branch"])
@pytest.mark.parametrize("after", ["begin", "extend"])
def test_a_step_that_requests_part_in_cannot_be_appended(how, after):
    """Rows that are made copy the last block as it stands: what is appended later would miss it."""
    cache, req, unique_idx, inverse, kv = begun([20, 20, 7])
    if after == "extend":
        req.extend(torch.ones(8, **ref.INT), 8, 1)
    else:
        _, _, unique_idx, inverse = req.begin(torch.ones((3, 20), **ref.INT), ref.dev([20, 20, 7]))
    if how == "fork":
        req.fork(ref.dev([0]), ref.dev([5]), [cache])
    else:
        req.branch(unique_idx, inverse, [cache])
    hs.hs_get_device_error()
    new = kv[:8 if after == "extend" else 60]
    with pytest.raises(ValueError, match="step"):
        req.append(cache, new, new)
    # A step begun after that is appended as ever.
    slots, _ = req.extend(torch.ones(8, **ref.INT), 8, 1)
    req.append(cache, kv[:8], kv[:8])
    hs.hs_get_device_error()
    assert (slots >= 0).any()
