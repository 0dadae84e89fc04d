"""KvRequests over several batches: steps of any length in any order, and
blocks that come back."""
import pytest
import torch

import kv_far_testutil as far
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu
D, BT = 64, 16


def prompts(lens, first=0):
    """Prompts of distinct tokens, so that none are merged."""
    t = torch.zeros((len(lens), max(lens)), dtype=torch.int32, device="cuda")
    for i, n in enumerate(lens):
        t[i, :n] = first + 1000 * i + torch.arange(n, device="cuda", dtype=torch.int32)
    return t, far.dev(lens)


def step(req, cache, G, seed):
    """Append and attend of the step's tokens, compared with the definition."""
    H, T = cache.n_kv_heads, len(req.slots)
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v = (torch.randn((T, h, D), generator=g, device="cuda").to(torch.bfloat16)
               for h in (H * G, H, H))
    req.append(cache, k, v)
    got = req.attend(cache, q)
    hs.hs_get_device_error()
    R = int(req.n_req.item())
    starts = req.starts.tolist()[:R + 1]
    p = dict(cache=cache, q=q[:starts[-1]], fmt="e4m3", table=req.table, lens=req.lens.tolist()[:R],
             starts=starts)
    far.compare([x[:starts[-1]] for x in got], far.attend(p))
    return req._ws


def fresh(req, n):
    return far.dev([n] * int(req.n_req.item())
                   + [0] * (req.max_requests - int(req.n_req.item())))


def test_a_long_step_after_a_short_one():
    cache = hs.KvCache(64, BT, 2, D)
    req = hs.KvRequests(cache, max_requests=3, max_len=200)
    req.begin(*prompts([3, 2]))
    step(req, cache, 4, 0)
    for i, n in enumerate((1, 9, 80, 1)):
        req.extend(fresh(req, n), 3 * n, n)
        step(req, cache, 4, 1 + i)
    # as many heads over fewer kv heads: more rows of each
    other = hs.KvCache(64, BT, 1, D)
    more = hs.KvRequests(other, max_requests=3, max_len=200)
    more._ws = req._ws
    more.begin(*prompts([30, 20]))
    step(more, other, 8, 9)


def test_each_stream_has_its_workspace():
    """Calls on two streams may run side by side: their counters are not shared."""
    cache = hs.KvCache(64, BT, 2, D)
    req = hs.KvRequests(cache, max_requests=3, max_len=200)
    req.begin(*prompts([30, 20]))
    q = torch.randn((len(req.slots), 8, D), device="cuda").to(torch.bfloat16)
    kv = torch.randn((len(req.slots), 2, D), device="cuda").to(torch.bfloat16)
    req.append(cache, kv, kv)
    want = req.attend(cache, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = req.attend(cache, q)
    s.synchronize()
    n = int(req.starts[-1].item())
    assert torch.equal(got[0][:n], want[0][:n])
    at = {w.data_ptr() for w in req._ws.values()}
    assert len(at) == 2


def test_a_second_batch_gives_back_the_first_ones_blocks():
    cache = hs.KvCache(24, BT, 2, D)
    req = hs.KvRequests(cache, max_requests=4, max_len=200)
    for batch, lens in enumerate(([100, 17, 40], [5], [160, 150, 30, 1], [200], [16, 16])):
        req.begin(*prompts(lens, first=batch))
        hs.hs_get_device_error()
        held = sum(-(-n // BT) for n in lens)
        taken, given = req.cursor.tolist()
        assert given - taken == 24 - held
        step(req, cache, 4, batch)
        if batch == 1:                                   # some of it given back before
            req.release(torch.tensor([True] * 4, device="cuda"))
            assert req.cursor.tolist()[1] - req.cursor.tolist()[0] == 24
        taken, given = req.cursor.tolist()
        free = req.pool.cpu()[[i % 24 for i in range(taken, given)]].tolist()
        mine = [x for r, n in enumerate(req.lens.tolist()) for x in req.table[r, :-(-n // BT)].tolist()]
        assert sorted(free + mine) == list(range(24))
