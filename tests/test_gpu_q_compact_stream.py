"""hs_kv_compact on a stream that is not the current one."""
import numpy as np
import pytest
import torch

import pages_testutil as ref
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu


def held(stream):
    """Bytes that the allocator keeps for a stream."""
    return sum(s["total_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == stream.cuda_stream)


@pytest.mark.parametrize("as_number", [False, True])
def test_its_own_workspace_is_that_stream_s(as_number):
    """What is freed when the call returns goes to no other stream, which could write it while the
    kernels still run."""
    n, bt = 400000, 16
    lens = np.array([700, 0, 33, 1599])
    table, shared, _ = ref.requests(list(lens), bt, n, 1, 2)
    args = ref.dev(lens), ref.dev(table), ref.dev(shared), bt
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before = held(side)
    got = hs.hs_kv_compact(*args, stream=side.cuda_stream if as_number else side)
    torch.cuda.synchronize()
    assert held(side) >= before + hs.hs_kv_compact_workspace(n)
    *want, bad = ref.compact(lens, table, shared, bt)
    for a, b in zip(got, want):
        assert (a.cpu().numpy() == b).all()
    hs.hs_get_device_error()
    assert not bad
