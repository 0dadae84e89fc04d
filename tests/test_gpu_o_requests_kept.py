"""What KvRequests keeps hold of where requests part: tokens of a step that is
not appended yet, and rows behind the requests that there were."""
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


def free(req):
    return (req.cursor[1] - req.cursor[0]).item()


def same_blocks(cache, req, a, b, length):
    """Rows a and b hold the same codes and scales of `length` tokens."""
    need = -(-length // BT)
    ia, ib = req.table[a, :need].long(), req.table[b, :need].long()
    assert (ia >= 0).all() and (ib >= 0).all()
    rest = length - (need - 1) * BT
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x, y = codes.view(torch.uint8)[ia], codes.view(torch.uint8)[ib]
        assert torch.equal(x[:-1], y[:-1]) and torch.equal(x[-1, :, :rest], y[-1, :, :rest])
        assert torch.equal(scale[ia], scale[ib])


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


def test_rows_behind_the_requests_keep_their_blocks():
    """Rows made behind n_req are requests from then on: a step, release, compaction and the next
    batch all count what they hold."""
    cache, req, _, _, kv = begun([20, 37, 7])
    assert free(req) == 64 - 2 - 3 - 1
    req.fork(ref.dev([0, 1, 2]), ref.dev([4, 2, -1]), [cache])        # (row 2 has tokens: an error)
    with pytest.raises(hs.HsError):
        hs.hs_get_device_error()
    assert req.n_req.item() == 5 and req.lens.tolist()[:5] == [20, 37, 7, 0, 20]
    same_blocks(cache, req, 0, 4, 20)
    req.fork(ref.dev([1, 4, 0]), ref.dev([6, 3, 0]), [cache])
    hs.hs_get_device_error()
    assert req.n_req.item() == 7 and req.lens.tolist() == [20, 37, 7, 20, 20, 0, 37, 0]
    req.extend(ref.dev([1, 1, 0, 1, 1, 0, 1, 0]), 8, 1)
    req.append(cache, kv[:8], kv[:8])
    assert req.lens.tolist() == [21, 38, 7, 21, 21, 0, 38, 0]
    req.compact([cache])
    hs.hs_get_device_error()
    # 1 + 2 full blocks shared, a rest for each
    assert free(req) == 64 - (1 + 2) - 5 - 1
    done = torch.zeros(8, dtype=torch.bool, device="cuda")
    done[[4, 6]] = True
    req.release(done)
    assert free(req) == 64 - (1 + 2) - 3 - 1
    req.begin(torch.ones((1, 20), **ref.INT), ref.dev([20]))
    hs.hs_get_device_error()
    assert free(req) == 64 - 2 and (req.shared == 0).all()


def test_the_next_batch_gets_back_what_forked_rows_hold():
    cache, req, _, _, _ = begun([20, 37])
    req.fork(ref.dev([0, 1]), ref.dev([2, 7]), [cache])
    req.begin(torch.ones((1, 20), **ref.INT), ref.dev([20]))
    hs.hs_get_device_error()
    assert free(req) == 64 - 2 and (req.shared == 0).all()
    ring = [req.pool[i % 64].item() for i in range(*req.cursor.tolist())]
    assert len(set(ring)) == 62


def test_branch_beside_rows_that_were_forked():
    cache, req, unique_idx, inverse, _ = begun([20, 37, 20])
    tokens = torch.arange(3 * 37, **ref.INT).view(3, 37)
    tokens[2] = tokens[0]
    _, _, unique_idx, inverse = req.begin(tokens, ref.dev([20, 37, 20]))
    kv = torch.randn((tokens.numel(), H, D), generator=ref.gen(2), device="cuda").to(torch.bfloat16)
    req.append(cache, kv, kv)
    assert req.n_req.item() == 2
    req.fork(ref.dev([1]), ref.dev([4]), [cache])
    rows = req.branch(unique_idx, inverse, [cache])
    hs.hs_get_device_error()
    assert rows.tolist() == [0, 1, 5] and req.n_req.item() == 6
    assert req.lens.tolist() == [20, 37, 0, 0, 37, 20, 0, 0]
    same_blocks(cache, req, 0, 5, 20)
    same_blocks(cache, req, 1, 4, 37)


def test_fork_of_nobody_makes_no_requests():
    cache, req, _, _, _ = begun([20, 37])
    none = torch.zeros(0, **ref.INT)
    req.fork(none, none, [cache])
    req.fork(ref.dev([0, 1, 0]), ref.dev([-1, 1, 0]), [cache])
    hs.hs_get_device_error()
    assert req.n_req.item() == 2
    req.fork(ref.dev([0, 0]), ref.dev([8, -2]), [cache])              # no rows of the table
    with pytest.raises(hs.HsError):
        hs.hs_get_device_error()
    assert req.n_req.item() == 2 and (req.shared == 0).all()


def test_a_fork_that_is_refused_changes_nothing():
    cache, req, _, _, kv = begun([20, 37])
    slots, _ = req.extend(torch.ones(8, **ref.INT), 8, 1)
    for src, dst in ((ref.dev([0, 1]), ref.dev([5])), (ref.dev([0]), ref.dev([5]).long())):
        with pytest.raises((TypeError, ValueError)):
            req.fork(src, dst, [cache])
    assert req.slots is slots and req.n_req.item() == 2 and (req.shared == 0).all()
    req.append(cache, kv[:8], kv[:8])
    hs.hs_get_device_error()


@pytest.mark.parametrize("n_req,want", [(3, 9), (9, 9), (10, 10), (12, 12), (13, 12), (0, 9), (-5, 9)])
def test_the_number_of_requests_after_a_fork(n_req, want):
    """The last row that is made counts, not rows that pairs name in vain."""
    table = torch.full((12, 3), -1, **ref.INT)
    table[0, :2], table[1, :1], table[9, :1] = ref.dev([3, 4]), 5, 6
    lens = ref.dev([20, 7, 0, 0, 0, 0, 0, 0, 0, 5, 0, 0])
    shared, pool = torch.zeros(40, **ref.INT), torch.arange(40, **ref.INT)
    cursor = ref.dev([10, 40], torch.int64)
    src, dst = ref.dev([0, 2, 1, 0, 12, 11, 0, 1]), ref.dev([4, 8, 3, 9, 10, 11, 12, -1])
    for out in (False, True):
        given = None
        if out:
            given = tuple(torch.zeros(n, **ref.INT) if n != 2 else torch.zeros_like(cursor)
                          for n in (12, 2, 8, 8, 8, 1))
        got = hs.hs_kv_fork_n(src, dst, lens, ref.dev([n_req]), table.clone(), shared.clone(), pool, cursor, BT,
                              out=given)
        with pytest.raises(hs.HsError):                 # row 9 has tokens, rows 12 are none
            hs.hs_get_device_error()
        plain = hs.hs_kv_fork(src, dst, lens, table.clone(), shared.clone(), pool, cursor, BT)
        with pytest.raises(hs.HsError):
            hs.hs_get_device_error()
        assert got[5].tolist() == [want] and all(torch.equal(a, b) for a, b in zip(got, plain))
    none = torch.zeros(0, **ref.INT)
    got = hs.hs_kv_fork_n(none, none, lens, ref.dev([n_req]), table, shared, pool, cursor, BT)
    assert got[5].tolist() == [min(max(n_req, 0), 12)]
    hs.hs_get_device_error()


def test_the_last_of_many_rows():
    lens = torch.zeros(16384, **ref.INT)
    table = torch.full((16384, 2), -1, **ref.INT)
    lens[0], table[0, 0] = 3, 7
    pool, shared = torch.arange(20000, **ref.INT), torch.zeros(20000, **ref.INT)
    order = 1 + torch.randperm(16380, generator=ref.gen(1), device="cuda").to(torch.int32)
    got = hs.hs_kv_fork_n(torch.zeros_like(order), order, lens, ref.dev([1]), table, shared, pool,
                          ref.dev([8, 20000], torch.int64), BT)
    hs.hs_get_device_error()
    assert got[5].tolist() == [16381] and (got[0] == 3).sum() == 16381
