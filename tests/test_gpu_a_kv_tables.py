"""hs_kv_tables and hs_kv_release against the rule applied request by
request: whole numbers, so everything has to be equal."""
import numpy as np
import pytest
import torch

import kv_testutil as ref
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def ring(rng, n_blocks, used, taken):
    """(pool, cursor): every block that is not in `used`, in a ring that begins at `taken`."""
    free = rng.permutation(np.setdiff1d(np.arange(n_blocks), used))
    pool = np.full(n_blocks, -7)
    pool[(taken + np.arange(len(free))) % n_blocks] = free
    return pool, np.array([taken, taken + len(free)])


def state(rng, have, fresh, bt, width=None, spare=3):
    """Distinct blocks for what the requests have, garbage past them, and a ring of the others."""
    R = len(have)
    width = width or max(1, max((-(-(h + f) // bt) for h, f in zip(have, fresh)), default=1))
    need = [-(-h // bt) for h in have]
    new = sum(-(-(h + f) // bt) for h, f in zip(have, fresh)) - sum(need)
    n_blocks = sum(need) + new + spare
    perm = rng.permutation(n_blocks)
    table = rng.integers(-5, n_blocks + 5, size=(R, width))
    at = 0
    for r in range(R):
        table[r, :need[r]] = perm[at:at + need[r]]
        at += need[r]
    pool, cursor = ring(rng, n_blocks, perm[:at], int(rng.integers(0, 3 * n_blocks)))
    return table, pool, cursor


def call(have, fresh, table, pool, cursor, bt, T, n_req_dev=None):
    t = dev(table)
    slots, starts, lens, after = hs.hs_kv_tables(
        dev(have), dev(fresh), t, dev(pool), dev(cursor, torch.int64), bt, T,
        n_req_dev=None if n_req_dev is None else dev(np.array([n_req_dev])))
    return [x.cpu().numpy() for x in (t, slots, starts, lens, after)]


CASES = [
    # R, most tokens had, most new ones
    (1, 0, 1), (1, 0, 1000), (1, 17, 1), (2, 40, 3), (64, 1500, 1), (64, 1500, 2), (513, 40, 40),
    (1434, 0, 512), (4096, 300, 1), (16384, 5, 2),
]


@pytest.mark.parametrize("bt", [16, 32, 64, 128])
@pytest.mark.parametrize("R,most,new", CASES)
def test_tables(R, most, new, bt):
    rng = np.random.default_rng(R + bt)
    have = rng.integers(0, most + 1, size=R)
    fresh = rng.integers(0, new + 1, size=R)
    have[rng.random(R) < 0.2] = bt * min(1, most)      # whole blocks, and none
    table, pool, cursor = state(rng, have, fresh, bt)
    T = int(fresh.sum()) + int(rng.integers(0, 40))
    got = call(have, fresh, table, pool, cursor, bt, T)
    hs.hs_get_device_error()
    for g, w in zip(got, ref.tables(have, fresh, table, pool, cursor, bt, T)):
        assert np.array_equal(g, w)


def test_no_requests_and_no_tokens():
    rng = np.random.default_rng(1)
    got = call([], [], np.zeros((0, 4), int), np.arange(5), [2, 4], 16, 3)
    hs.hs_get_device_error()
    assert got[1].tolist() == [-1] * 3 and got[2].tolist() == [0] and got[4].tolist() == [2, 4]
    table, pool, cursor = state(rng, [16, 5], [0, 0], 16)
    got = call([16, 5], [0, 0], table, pool, cursor, 16, 0)
    hs.hs_get_device_error()
    assert np.array_equal(got[0], table) and got[3].tolist() == [16, 5]
    assert got[4].tolist() == cursor.tolist()


def test_count_on_the_device():
    """Rows past the merged count are no requests, whatever their lengths say."""
    rng = np.random.default_rng(2)
    have, fresh = np.array([3, 20, -9, 7]), np.array([14, 1, 5, 1 << 30])
    table, pool, cursor = state(rng, have[:2], fresh[:2], 16, width=4)
    table = np.concatenate([table, np.full((2, 4), 99)])
    got = call(have, fresh, table, pool, cursor, 16, 20, n_req_dev=2)
    hs.hs_get_device_error()
    t, slots, starts, lens, after = ref.tables(have[:2], fresh[:2], table, pool, cursor, 16, 20)
    assert np.array_equal(got[0], t) and np.array_equal(got[1], slots)
    assert got[2].tolist() == [0, 14, 15, 15, 15] and got[3].tolist() == [17, 21, 0, 0]
    assert np.array_equal(got[4], after)


def expect_error():
    with pytest.raises(hs.HsError) as e:
        hs.hs_get_device_error()
    assert e.value.status == hs.HS_ERR_INVALID_ARG
    hs.hs_get_device_error()                           # reported once


def test_a_ring_that_runs_out():
    """Requests are served in order; the one that finds too little keeps what it got."""
    bt = 16
    have, fresh = np.array([10, 0, 16, 3]), np.array([30, 33, 40, 2])
    # new blocks: 2 (10 -> 40), 3, 3, 0; six are left
    table = np.full((4, 4), 50)
    table[:, 0] = [0, 50, 1, 2]
    pool, cursor = np.concatenate([np.arange(3, 60), [3, 4, 5]]), np.array([58, 64])
    got = call(have, fresh, table, pool, cursor, bt, int(fresh.sum()))
    expect_error()
    taken = pool[np.arange(58, 64) % 60]
    t = got[0]
    assert t[0].tolist() == [0, taken[0], taken[1], 50]
    assert t[1].tolist() == [taken[2], taken[3], taken[4], 50]
    assert t[2].tolist() == [1, taken[5], -1, -1] and t[3].tolist() == [2, 50, 50, 50]
    assert got[3].tolist() == [40, 33, 32, 5] and got[4].tolist() == [64, 64]
    s = got[1][63:103]                                 # request 2: tokens 16 .. 55
    assert (s[:16] == taken[5] * bt + np.arange(16)).all() and (s[16:] == -1).all()
    assert got[1][103:].tolist() == [2 * bt + 3, 2 * bt + 4]


def test_data_errors():
    """Lengths and entries that cannot be: the request or the token is left out, and said."""
    ok = (np.arange(9), np.array([0, 9]))
    for have, fresh in (([-1], [3]), ([3], [-1]), ([60], [5]), ([2**31 - 1], [2**31 - 1])):
        got = call(have, fresh, np.zeros((1, 4), int), *ok, 16, 4)
        expect_error()
        assert got[1].tolist() == [-1] * 4 and got[3].tolist() == [0] and got[4].tolist() == [0, 9]
    got = call([3], [2], np.full((1, 1), 9), *ok, 16, 2)           # an entry that is no block
    expect_error()
    assert got[1].tolist() == [-1, -1]
    got = call([0], [2], np.full((1, 1), 7), np.full(9, 12), ok[1], 16, 2)
    expect_error()
    assert got[1].tolist() == [-1, -1] and got[0].tolist() == [[-1]]
    got = call([0], [5], np.full((1, 1), 7), *ok, 16, 3)           # more tokens than there is room
    expect_error()
    assert got[1].tolist() == [0, 1, 2] and got[3].tolist() == [5]
    got = call([0], [1], np.full((1, 1), 7), ok[0], [5, 3], 16, 1)  # a ring that ends before it begins
    expect_error()
    assert got[1].tolist() == [-1]


@pytest.mark.parametrize("R", [1, 3, 16, 17, 300])
def test_release_gives_back_what_was_taken(R):
    """Take, give back, take again: the same blocks come round, none twice."""
    rng = np.random.default_rng(R)
    bt, n_blocks = 16, 40 * R
    pool = rng.permutation(n_blocks)
    p, cursor = dev(pool), dev([0, n_blocks], torch.int64)
    fresh = rng.integers(1, 40 * bt, size=R)
    table = torch.full((R, 40), -1, dtype=torch.int32, device="cuda")
    zero = dev(np.zeros(R, int))
    slots, starts, lens, cursor = hs.hs_kv_tables(zero, dev(fresh), table, p, cursor, bt,
                                                  int(fresh.sum()))
    done = rng.random(R) < 0.6
    after = hs.hs_kv_release(torch.where(dev(done, torch.bool), lens, 0), table, p, cursor, bt)
    hs.hs_get_device_error()
    need = -(-fresh // bt)
    t = table.cpu().numpy()
    back = np.concatenate([t[r, :need[r]] for r in range(R) if done[r]] + [np.zeros(0, int)])
    taken, given = after.cpu().numpy()
    assert taken == need.sum() and given == n_blocks + len(back)
    now = p.cpu().numpy()[np.arange(taken, given) % n_blocks]
    assert np.array_equal(now, np.concatenate([pool[need.sum():], back]))
    held = np.concatenate([t[r, :need[r]] for r in range(R) if not done[r]] + [np.zeros(0, int)])
    assert len(np.union1d(now, held)) == n_blocks == len(now) + len(held)


def test_release_errors():
    table = dev([[3, 99, 4], [1, 2, 0]])
    pool, cursor = dev(np.full(8, -1)), dev([6, 9], torch.int64)
    after = hs.hs_kv_release(dev([40, 0]), table, pool, cursor, 16)
    expect_error()                                     # 99 is no block: left out
    assert after.tolist() == [6, 11] and pool.cpu()[[1, 2]].tolist() == [3, 4]
    for lens in ([-1, 0], [49, 0]):
        assert hs.hs_kv_release(dev(lens), table, pool, cursor, 16).tolist() == [6, 9]
        expect_error()
    after = hs.hs_kv_release(dev([0, 48]), table, pool, dev([6, 12], torch.int64), 16)
    expect_error()                                     # room for two
    assert after.tolist() == [6, 14]


def test_on_another_stream():
    rng = np.random.default_rng(3)
    have, fresh = rng.integers(0, 99, size=40), rng.integers(0, 99, size=40)
    table, pool, cursor = state(rng, have, fresh, 32)
    args = [dev(have), dev(fresh), dev(table), dev(pool), dev(cursor, torch.int64)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = hs.hs_kv_tables(*args, 32, int(fresh.sum()), stream=s)
    s.synchronize()
    want = ref.tables(have, fresh, table, pool, cursor, 32, int(fresh.sum()))
    assert np.array_equal(args[2].cpu().numpy(), want[0])
    assert np.array_equal(got[0].cpu().numpy(), want[1])
