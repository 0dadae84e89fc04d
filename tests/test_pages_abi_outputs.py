"""Arrays that lie in one another or where no kernel may read them, refused
before anything touches a device (no GPU needed)."""
import itertools

import pytest
import torch

from paper_2607_22578_gb300 import _lib

A = 1 << 20                                            # an aligned address that nothing reads


def status(fn, *args):
    return getattr(_lib.load(), fn)(*args)


def message():
    return _lib.load().hs_last_error().decode()


def refused(T, H, token, head, dim):
    """Whether out's heads are said to overlap.  (turns is NULL, so that no call goes on.)"""
    got = status("hs_rotary", A, token, head, 2 * A, token, head, 0, T, H, dim, 2, 0, None, 1.0, 0, A,
                 None, None, 0, None, None)
    assert got == _lib.HS_ERR_INVALID_ARG and ("overlap" in message() or "turns" in message())
    return "overlap" in message()


def overlap(T, H, token, head, dim):
    at = sorted(t * token + h * head for t in range(T) for h in range(H))
    return any(b - a < dim for a, b in zip(at, at[1:]))


@pytest.mark.parametrize("T,H", [(1, 1), (1, 5), (4, 1), (2, 2), (3, 2), (2, 7), (5, 4)])
@pytest.mark.parametrize("dim", [2, 3, 8])
def test_heads_of_out_that_overlap(T, H, dim):
    """Every layout with strides of some heads, the equal ones among them, against all pairs."""
    strides = sorted(set(range(dim, 4 * dim + 2)) | {dim * k + j for k in (H, T, H + 1) for j in (-1, 0, 1)})
    for token, head in itertools.product(strides, strides):
        want = overlap(T, H, token, head, dim)
        for a, b in ((token, head), (-token, head), (token, -head), (-token, -head)):
            assert refused(T, H, a, b, dim) == want == overlap(T, H, a, b, dim)


def test_heads_of_out_of_any_size():
    """Counts and strides whose products pass 64 bits, and many steps that nearly meet."""
    most, heads, far = 2 ** 31 - 1, 2 ** 30, 2 ** 62
    assert not refused(most, heads, far, 128, 128) and not refused(most, heads, 128, far, 128)
    assert refused(most, heads, far, far, 128) and refused(2, 2, far, far - 127, 128)
    assert not refused(2, 2, far, far - 128, 128) and not refused(1, 2, 0, -far, 128)
    for T, H, token, head in ((300, 300, 128000, 128128), (300, 300, 1000, 1003), (300, 3, 6400, 3201),
                              (100, 90, 6400, 6465), (100, 100, 6400, 6464), (100, 101, 6400, 6464)):
        assert refused(T, H, token, head, 64) == overlap(T, H, token, head, 64)


def test_more_heads_than_are_counted_in_32_bits():
    """A thread's last heads are followed by two more numbers."""
    for n in (2 ** 30 + 1, 2 ** 31 - 2, 2 ** 31 - 1):
        assert status("hs_rotary", A, 0, 2, 2 * A, 0, 2, 0, 1, n, 2, 2, 0, None, 1.0, 0, A, None, None, 0, None,
                      None) == _lib.HS_ERR_INVALID_ARG and "n_heads" in message()


FORK = ["src", "dst", "lens", "lens_out", "table", "shared", "pool", "cursor", "after", "source", "target",
        "tokens"]


def fork(at, n=3, n_req=4):
    return status("hs_kv_fork", at["src"], at["dst"], n, at["lens"], at["lens_out"], n_req, 16, at["table"], 8,
                  at["shared"], at["pool"], 64, at["cursor"], at["after"], at["source"], at["target"],
                  at["tokens"], None)


def fork_n(at):
    return status("hs_kv_fork_n", at["src"], at["dst"], 3, at["lens"], at["lens_out"], 4, at["n_dev"],
                  at["n_out"], 16, at["table"], 8, at["shared"], at["pool"], 64, at["cursor"], at["after"],
                  at["source"], at["target"], at["tokens"], None)


@pytest.mark.parametrize("other", FORK + ["n_dev"])
def test_the_count_of_requests_is_nothing_else(other):
    at = {name: (i + 1) * A for i, name in enumerate(FORK + ["n_dev"])}
    assert fork_n({**at, "n_out": at[other]}) == _lib.HS_ERR_INVALID_ARG and "output" in message()


@pytest.mark.parametrize("bad,what", [(dict(n_dev=None), "n_req_dev"), (dict(n_out=None), "n_req_dev"),
                                      (dict(n_dev=A + 2), "n_req_dev"), (dict(n_out=A + 2), "misaligned"),
                                      (dict(src=None), "src"), (dict(after=8 * A), "cursor_out")])
def test_fork_n_refuses(bad, what):
    at = {name: (i + 1) * A for i, name in enumerate(FORK + ["n_dev", "n_out"])}
    assert fork_n({**at, **bad}) == _lib.HS_ERR_INVALID_ARG and what in message()


RELEASE = ["lens", "n_dev", "table", "shared", "shared_out", "pool", "cursor", "after"]


def release(at):
    return status("hs_kv_release_shared", at["lens"], 4, at["n_dev"], 16, at["table"], 8, at["shared"],
                  at["shared_out"], at["pool"], 64, at["cursor"], at["after"], None)


COMPACT = ["lens", "n_dev", "table", "table_out", "shared", "shared_out", "pool", "after", "source", "target",
           "moves", "ws"]


def compact(at):
    return status("hs_kv_compact", at["lens"], 4, at["n_dev"], 16, at["table"], at["table_out"], 8, at["shared"],
                  at["shared_out"], 64, at["pool"], at["after"], at["source"], at["target"], at["moves"],
                  at["ws"], 256, None)


def pairs(names, written, allowed=()):
    return [(a, b) for a, b in itertools.combinations(names, 2)
            if (a in written or b in written) and (a, b) not in allowed]


CASES = [(fork, FORK, a, b) for a, b in pairs(FORK, FORK[3:6] + FORK[8:])]
CASES += [(release, RELEASE, a, b) for a, b in pairs(RELEASE, RELEASE[4:6] + RELEASE[7:], [("shared", "shared_out")])]
CASES += [(compact, COMPACT, a, b) for a, b in pairs(COMPACT, COMPACT[3:4] + COMPACT[5:],
                                                     [("table", "table_out"), ("shared", "shared_out")])]


@pytest.mark.parametrize("call,names,a,b", CASES, ids=lambda x: x if isinstance(x, str) else None)
def test_arrays_that_are_written_are_nothing_else(call, names, a, b):
    at = {name: (i + 1) * A for i, name in enumerate(names)}
    at[a] = at[b]
    assert call(at) == _lib.HS_ERR_INVALID_ARG and ("output" in message() or "cursor_out" in message() or
                                                    "lens_out" in message())


def test_rotary_of_a_host_is_not_handed_to_a_kernel():
    x = torch.zeros((2, 1, 64), dtype=torch.bfloat16)
    for r in (_lib.Rotary(64, device="cpu"), _lib.Rotary.of([1.0] * 32, device="cpu")):
        with pytest.raises(TypeError, match="turns"):
            _lib.hs_rotary(x, r, positions=torch.zeros(2, dtype=torch.int32))


def test_compact_with_a_workspace_of_the_host():
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError, match="workspace"):
        _lib.hs_kv_compact(i, i.view(2, 2), i, 16, workspace=torch.zeros(512, dtype=torch.uint8))
