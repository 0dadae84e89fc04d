"""hs_kv_attend against the formula in 64 bits, within what its arithmetic
allows (kv_testutil.attend).  The output is rounded once, and rounding keeps
order: it lies between the rounded ends of what it may have been before."""
import numpy as np
import pytest
import torch

import kv_testutil as ref
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu


def problem(lens, n, H, G, d, bt, fmt, dtype, seed=0, spread=0, pow2=True, spare=3):
    """Requests of `lens` tokens with `n` queries each over random blocks.  Every slot that holds
    no token is a NaN (int8: its largest code), every entry past a request's end is -1, and the
    blocks of no request have NaN for a scale."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    need = [-(-L // bt) for L in lens]
    blocks = sum(need) + spare
    perm, width = rng.permutation(blocks), max(1, max(need))
    table = np.full((len(lens), width), -1)
    at = 0
    codes = torch.randint(0, 256, (2, blocks, H, bt, d), generator=g, device="cuda",
                          dtype=torch.uint8)
    if fmt == "e4m3":
        codes = torch.where((codes & 127) > 0x6F, codes & 0xEF, codes)    # no NaN, at most 120
    else:
        codes = torch.where(codes == 128, 0, codes)
    unit = 2.0 ** -6 if fmt == "e4m3" else 2.0 ** -6
    scale = unit * torch.exp2(torch.randint(-2 - spread, 1 + spread, (2, blocks, H), generator=g,
                                            device="cuda").float())
    if spread:
        scale[0] = unit / 4                               # only the values' blocks differ wildly
    if not pow2:
        scale *= 1 + torch.rand((2, blocks, H), generator=g, device="cuda")
    for r, L in enumerate(lens):
        table[r, :need[r]] = perm[at:at + need[r]]
        at += need[r]
        if L % bt:
            codes[:, table[r, need[r] - 1], :, L % bt:] = 0x7F
    codes[:, perm[at:]] = 0x7F
    scale[:, perm[at:]] = float("nan")
    k, v = (c.contiguous().view(ref.CODES[fmt]) for c in codes)
    T = sum(n)
    q = torch.randn((T, H * G, d), generator=g, device="cuda")
    q = (q * torch.exp(torch.randn((T, H * G, 1), generator=g, device="cuda"))).to(ref.DTYPES[dtype])
    return dict(cache=hs.KvCache.of(k, v, scale[0].contiguous(), scale[1].contiguous()), q=q,
                table=torch.from_numpy(table).int().cuda(), lens=list(lens),
                starts=np.concatenate([[0], np.cumsum(n)]).tolist(), fmt=fmt, dtype=dtype)


def dev(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def call(p, causal=True, window=0, scale=None, **kw):
    n = np.diff(p["starts"])
    kw.setdefault("starts", dev(p["starts"]))
    if kw["starts"] is not None:
        kw.setdefault("max_q", int(n.max()))
    out = hs.hs_kv_attend(p["cache"], p["q"], dev(p["lens"]), p["table"], scale=scale,
                          causal=causal, window=window, **kw)
    hs.hs_get_device_error()
    return out


def check(p, got, causal=True, window=0, scale=None):
    c = p["cache"]
    scale = c.dim ** -0.5 if scale is None else scale
    out, lse, tol, tol_l = ref.attend(p["q"], c.k, c.v, c.k_scale, c.v_scale, p["fmt"], p["table"],
                                      p["lens"], p["starts"], scale, causal, window)
    o, l = (x.double() for x in got)
    assert torch.isfinite(o).all()
    least, most = ((out + x).to(p["q"].dtype).double() for x in (-tol, tol))
    far = torch.maximum(least - o, o - most)
    assert (far <= 0).all(), "out off by %g over its bound" % far.max().item()
    none = lse == -np.inf
    assert torch.equal(none, l == -np.inf)
    assert (o[none] == 0).all()
    far = ((l - lse).abs() - tol_l)[~none]
    assert (far <= 0).all(), "lse off by %g over its bound" % far.max().item()


def both(p, **kw):
    check(p, call(p, **kw), **kw)


LENS = {
    "one_token": ([1], [1]),
    "one": ([33], [1]),
    "ragged": ([1, 700, 16, 17, 128, 129, 31, 2000, 64], [1] * 9),
    "long": ([40003], [1]),
    "drafts": ([5, 900, 130, 64], [5, 5, 5, 5]),
    "mixed": ([300, 40, 77, 1025], [13, 1, 77, 2]),
}


@pytest.mark.parametrize("name", sorted(LENS))
@pytest.mark.parametrize("d,bt", [(64, 16), (64, 128), (128, 16), (128, 32), (128, 64), (256, 16),
                                  (256, 64)])
@pytest.mark.parametrize("fmt,dtype", [("e4m3", "bf16"), ("int8", "fp16")])
def test_lengths(name, d, bt, fmt, dtype):
    lens, n = LENS[name]
    both(problem(lens, n, 2, 4, d, bt, fmt, dtype))


@pytest.mark.parametrize("H,G", [(1, 1), (3, 2), (2, 3), (1, 7), (2, 8), (1, 9), (1, 16), (2, 17),
                                 (1, 48), (8, 4)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_heads(H, G, d):
    both(problem([77, 1, 260], [1, 1, 1], H, G, d, 32, "e4m3", "fp16"))
    both(problem([77, 3, 260], [2, 3, 40], H, G, d, 32, "int8", "bf16"))


@pytest.mark.parametrize("d,bt,H,G", [(128, 16, 2, 4), (64, 32, 3, 1), (128, 128, 1, 8),
                                      (64, 64, 1, 5), (256, 32, 1, 4)])
@pytest.mark.parametrize("fmt,dtype", [("e4m3", "bf16"), ("int8", "fp16")])
def test_prompts(d, bt, H, G, fmt, dtype):
    """Whole prompts, chunks at the end of longer ones, and single tokens beside them."""
    both(problem([513, 300, 1, 64, 129], [513, 300, 1, 64, 129], H, G, d, bt, fmt, dtype))
    both(problem([1500, 1027, 640, 260], [33, 260, 1, 127], H, G, d, bt, fmt, dtype))
    both(problem([700, 45, 0, 390], [1, 200, 64, 257], H, G, d, bt, fmt, dtype), causal=False)


def test_more_prompts_than_sms():
    """Several prompts one after the other on each SM, of one and of two tiles of rows, and more
    requests than threads."""
    rng = np.random.default_rng(8)
    n = rng.integers(0, 130, size=500)
    have = rng.integers(0, 300, size=500)
    both(problem((have + n).tolist(), n.tolist(), 2, 3, 64, 16, "e4m3", "bf16"))
    n = rng.integers(20, 90, size=90)
    both(problem((n + 5).tolist(), n.tolist(), 4, 4, 128, 32, "int8", "bf16"))


@pytest.mark.parametrize("causal,window", [(True, 1), (True, 16), (True, 100), (True, 1000),
                                           (True, 2**31 - 1), (False, 0)])
@pytest.mark.parametrize("n", [1, 7, 150])
def test_masks(causal, window, n):
    lens = [max(n, 5), 260, 1030, 700]
    both(problem(lens, [n] * 4, 2, 4, 128, 16, "e4m3", "bf16"), causal=causal, window=window)
    both(problem(lens, [n] * 4, 2, 1, 64, 64, "int8", "fp16"), causal=causal, window=window)


@pytest.mark.parametrize("n", [1, 6, 70])
def test_rows_that_see_nothing(n):
    """Empty caches, and queries that stand before the first key."""
    p = problem([0, 20, 0, 3, 0], [n, n, 0, n, 1], 2, 4, 128, 16, "e4m3", "bf16")
    both(p)
    both(p, causal=False)
    both(p, window=2)
    p = problem([0, 0], [n, n], 2, 4, 64, 16, "int8", "fp16")
    both(p)


@pytest.mark.parametrize("n", [1, 80])
def test_far_blocks_scales(n):
    """Value blocks whose scales are 2^20 apart, scales that are no powers of two, scores that
    are all alike or all on one key."""
    both(problem([900, 33], [n, min(n, 33)], 2, 4, 128, 16, "e4m3", "bf16", spread=10))
    both(problem([900, 33], [n, min(n, 33)], 2, 2, 64, 32, "int8", "bf16", pow2=False))
    both(problem([900, 33], [n, min(n, 33)], 1, 4, 256, 16, "e4m3", "bf16", pow2=False), scale=3.0)
    both(problem([900, 33], [n, min(n, 33)], 1, 4, 128, 64, "e4m3", "fp16"), scale=1e-6)


@pytest.mark.parametrize("big", [2.0 ** 100, 2.0 ** -100, 0.0])
def test_far_queries(big):
    """Rows of q far from 1: scaled on the way to half."""
    p = problem([400, 90], [1, 90], 2, 4, 128, 16, "e4m3", "bf16")
    p["q"] *= big
    both(p, scale=0.05 / big if big else None)


def test_views_with_strides():
    p = problem([300, 90], [5, 90], 2, 4, 64, 16, "e4m3", "bf16")
    want = call(p)
    T = len(p["q"])
    for pad, at in ((8, 8), (3, 1)):
        wide = torch.full((T, 8 * 64 + 2 * pad), 7.0, dtype=torch.bfloat16, device="cuda")
        view = wide[:, at:at + 512].view(T, 8, 64)
        view.copy_(p["q"])
        got = call(dict(p, q=view))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    heads_first = p["q"].transpose(0, 1).contiguous().transpose(0, 1)
    got = call(dict(p, q=heads_first))
    assert torch.equal(got[0], want[0])


def test_without_starts_and_with_a_count_on_the_device():
    p = problem([300, 90, 17], [3, 3, 3], 2, 4, 128, 16, "e4m3", "bf16")
    want = call(p)
    got = call(p, starts=None)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out = (torch.full_like(want[0], 5.0), torch.full_like(want[1], 5.0))
    call(p, n_req_dev=dev([2]), out=out)
    assert torch.equal(out[0][:6], want[0][:6]) and (out[0][6:] == 5).all()
    assert torch.equal(out[1][:6], want[1][:6]) and (out[1][6:] == 5).all()
    call(p, n_req_dev=dev([0]), out=out)
    got = call(p, out=(torch.empty_like(want[0]), None))
    assert torch.equal(got[0], want[0]) and got[1] is None


def test_many_requests():
    """More requests than threads, most of them short: several a CTA."""
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 200, size=3001).tolist()
    both(problem(lens, [1] * 3001, 1, 4, 64, 16, "e4m3", "bf16"))


def test_the_same_twice_on_one_workspace():
    """Cut requests are merged in the order of their parts, and the workspace is left as found."""
    a = problem([40003, 900], [1, 1], 2, 4, 128, 16, "e4m3", "bf16")
    b = problem([3000] * 7, [3] * 7, 2, 6, 64, 32, "int8", "fp16")
    c = problem([700, 90, 2000, 1], [300, 90, 70, 1], 2, 4, 128, 16, "e4m3", "bf16")
    size = max(hs.hs_kv_attend_workspace(p["cache"], 12, 300) for p in (a, b, c))
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    want = [call(p) for p in (a, b, c)]
    for _ in range(5):
        for p, w in zip((a, b, c), want):
            got = call(p, workspace=ws)
            assert torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])


def test_on_another_stream_and_in_a_graph():
    p = problem([2000, 90], [1, 1], 2, 4, 128, 16, "e4m3", "bf16")
    want = call(p)
    ws = torch.zeros(hs.hs_kv_attend_workspace(p["cache"], 8, 1), dtype=torch.uint8, device="cuda")
    lens, starts = dev(p["lens"]), dev(p["starts"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = hs.hs_kv_attend(p["cache"], p["q"], lens, p["table"], starts=starts, max_q=1,
                          workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0])
    got = hs.hs_kv_attend(p["cache"], p["q"], lens, p["table"], starts=starts, max_q=1, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = hs.hs_kv_attend(p["cache"], p["q"], lens, p["table"], starts=starts, max_q=1,
                              workspace=ws)
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("n", [1, 70])
def test_offsets_past_32_bits(n):
    """Blocks that lie beyond 2^32 values of the cache."""
    H, bt, d = 64, 64, 256
    blocks = (1 << 32) // (H * bt * d) + 4
    p = problem([150], [n], H, 1, d, bt, "int8", "bf16")
    c = p["cache"]
    far = hs.KvCache(blocks, bt, H, d, torch.int8)
    ids = p["table"][0].long()
    to = torch.arange(blocks - len(ids), blocks, device="cuda")
    for x, y in ((far.k, c.k), (far.v, c.v), (far.k_scale, c.k_scale), (far.v_scale, c.v_scale)):
        x[to] = y[ids]
    want = call(p)
    got = call(dict(p, cache=far, table=to.int()[None]))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_no_queries_and_no_requests():
    p = problem([30, 7], [1, 1], 2, 4, 64, 16, "e4m3", "bf16")
    none = p["q"][:0]
    for lens, table in ((dev(p["lens"]), p["table"]), (dev([]), p["table"][:0])):
        out, lse = hs.hs_kv_attend(p["cache"], none, lens, table)
        assert out.shape == none.shape and lse.shape == (0, 8)
    out = (torch.full_like(p["q"], 5.0), torch.full((2, 8), 5.0, device="cuda"))
    hs.hs_kv_attend(p["cache"], p["q"], dev(p["lens"]), p["table"], starts=dev([0, 0, 2]), max_q=2,
                    out=out)
    hs.hs_get_device_error()                           # the first request has none
    assert (out[0] != 5).all()


def expect_error():
    with pytest.raises(hs.HsError) as e:
        hs.hs_get_device_error()
    assert e.value.status == hs.HS_ERR_INVALID_ARG


@pytest.mark.parametrize("n", [1, 70])
def test_data_errors(n):
    """A request whose numbers cannot be is left out, the others are not."""
    p = problem([90, 100, 70], [n, n, n], 1, 4, 64, 16, "e4m3", "bf16")
    want = call(p)
    for bad in (dict(lens=[90, -1, 70]), dict(lens=[90, 113, 70]),
                dict(starts=[0, n, n - 1, 2 * n - 1]), dict(starts=[0, n, 3 * n, 3 * n + n])):
        out = (torch.full_like(want[0], 5.0), torch.full_like(want[1], 5.0))
        s = bad.get("starts", p["starts"])
        hs.hs_kv_attend(p["cache"], p["q"], dev(bad.get("lens", p["lens"])), p["table"],
                        starts=dev(s), max_q=n, out=out)
        expect_error()
        assert torch.equal(out[0][:n - 1], want[0][:n - 1])
        if "lens" in bad:
            assert torch.equal(out[0][:n], want[0][:n]) and torch.equal(out[0][2 * n:], want[0][2 * n:])
            assert (out[0][n:2 * n] == 5).all()
    table = p["table"].clone()
    table[1, 2] = 10 ** 6
    got = hs.hs_kv_attend(p["cache"], p["q"], dev(p["lens"]), table, starts=dev(p["starts"]), max_q=n)
    expect_error()
    assert torch.equal(got[0][:n], want[0][:n]) and torch.equal(got[0][2 * n:], want[0][2 * n:])


def test_refusals():
    p = problem([90, 20], [1, 1], 2, 4, 64, 16, "e4m3", "bf16")
    c, q, lens, t = p["cache"], p["q"], dev(p["lens"]), p["table"]
    for bad in (dict(q=q.float()), dict(lens=lens.long()), dict(t=t.cpu())):
        with pytest.raises(TypeError):
            hs.hs_kv_attend(c, bad.get("q", q), bad.get("lens", lens), bad.get("t", t))
    for bad in (dict(q=q[:, :, :32]), dict(q=q[0]), dict(t=t[0]), dict(t=t[:1]), dict(q=q[:1])):
        with pytest.raises(ValueError):
            hs.hs_kv_attend(c, bad.get("q", q), bad.get("lens", lens), bad.get("t", t))
    with pytest.raises(ValueError):
        hs.hs_kv_attend(c, q, lens, t, out=(q.new_empty(1, 8, 64), None))
    for kw, status in ((dict(window=-1), hs.HS_ERR_INVALID_ARG),
                       (dict(window=4, causal=False), hs.HS_ERR_INVALID_ARG),
                       (dict(scale=0.0), hs.HS_ERR_INVALID_ARG),
                       (dict(scale=float("nan")), hs.HS_ERR_INVALID_ARG),
                       (dict(q=q[:, :7].contiguous()), hs.HS_ERR_INVALID_ARG),
                       (dict(workspace=torch.zeros(256, dtype=torch.uint8, device="cuda")),
                        hs.HS_ERR_WORKSPACE)):
        with pytest.raises(hs.HsError) as e:
            hs.hs_kv_attend(c, kw.pop("q", q), lens, t, **kw)
        assert e.value.status == status
    hs.hs_get_device_error()


SPLIT = {
    "one": ([3000], [150]),
    "odd": ([1153, 4097, 515], [130, 161, 515]),
    "prompt": ([2100], [2100]),
    "mixed": ([900, 5000, 40, 0, 2600], [1, 290, 40, 3, 333]),
}


@pytest.mark.parametrize("name", sorted(SPLIT))
@pytest.mark.parametrize("d,H,G,fmt,dtype", [(128, 1, 4, "e4m3", "bf16"), (64, 2, 2, "int8", "fp16"),
                                             (64, 1, 8, "e4m3", "bf16"), (128, 2, 3, "int8", "bf16")])
def test_many_rows_of_few_requests(name, d, H, G, fmt, dtype):
    """Their tokens are shared out; the parts of a pair of tiles of rows differ in number."""
    lens, n = SPLIT[name]
    p = problem(lens, n, H, G, d, 32, fmt, dtype)
    both(p)
    both(p, window=700)
    both(p, causal=False)
    a, b = call(p), call(p)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_parts_that_see_nothing():
    """More queries than tokens: rows that see nothing beside rows in parts; far scales."""
    p = problem([700, 2000], [900, 400], 1, 4, 128, 16, "e4m3", "bf16", spread=10)
    both(p)
    both(p, window=40)


def test_parts_with_nan():
    """A NaN scale in one part reaches every row that sees its token."""
    p = problem([3000], [200], 1, 4, 128, 16, "e4m3", "bf16")
    out, _ = call(p)
    assert torch.isfinite(out).all()
    p["cache"].k_scale[p["table"][0, 3].item()] = float("nan")
    out, _ = call(p)
    assert torch.isnan(out.float()).all()
    out, _ = call(p, window=500)
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("d,H,G,fmt", [(64, 4, 6, "int8"), (128, 1, 4, "e4m3"), (256, 2, 4, "int8")])
@pytest.mark.parametrize("R,n,most", [(48, 5, 3000), (16, 1, 9000), (100, 2, 1500), (7, 3, 40000)])
def test_a_piece_for_each_block(d, H, G, fmt, R, n, most):
    """Fewer (request, head, group)s than the kernel has blocks, but more tokens than those have in
    one step: lengths that differ much, empty requests and others of no query among them."""
    rng = np.random.default_rng(R)
    lens = rng.integers(1, most, size=R)
    lens[::5] = most
    lens[3::11] = 0
    q = np.full(R, n)
    q[5::9] = 0
    p = problem(lens.tolist(), q.tolist(), H, G, d, 32, fmt, "bf16")
    both(p)
    both(p, window=1024)
