"""hs_kv_attend where an entry of a request's table is no block: its tokens
count as zeros, its neighbours' do not."""
import pytest
import torch

import kv_far_testutil as far
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 5, 160])
@pytest.mark.parametrize("d,bt", [(64, 16), (128, 16), (128, 32), (64, 128)])
@pytest.mark.parametrize("at", [0, 1, -2, -1])
def test_an_entry_that_is_no_block(n, d, bt, at):
    p = far.written([570], [n], 2, 4, d, bt, "e4m3", "bf16", lambda v, r, pos: v)
    c = p["cache"]
    for t in (c.k, c.v):
        t.view(torch.uint8)[p["table"][0, at].long()] = 0
    want = far.attend(p)
    for entry in (10 ** 6, -1, -2 ** 31, c.n_blocks):
        table = p["table"].clone()
        table[0, at] = entry
        got = far.call(dict(p, table=table))
        with pytest.raises(hs.HsError) as e:
            hs.hs_get_device_error()
        assert e.value.status == hs.HS_ERR_INVALID_ARG
        far.compare(got, want)
