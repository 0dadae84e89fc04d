"""hs_kv_append against the same rule in 64 bits.  Scales are powers of two,
so every quotient is exact and each code is rounded once in both: codes and
scales have to be equal, byte for byte (but for the sign of a NaN)."""
import numpy as np
import pytest
import torch

import kv_testutil as ref
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu


def make(rng, n, H, bt, d, fmt):
    """A cache as an earlier program left it: any codes, scales around 2^-6."""
    codes = [rng.integers(0, 256, size=(n, H, bt, d), dtype=np.uint8) for _ in range(2)]
    if fmt == "int8":
        codes = [np.where(c == 128, 0, c).astype(np.uint8) for c in codes]
    scales = [2.0 ** rng.integers(-9, -3, size=(n, H)) for _ in range(2)]
    t = [torch.from_numpy(c.copy()).cuda().view(ref.CODES[fmt]) for c in codes]
    s = [torch.from_numpy(x.astype(np.float32)).cuda() for x in scales]
    return hs.KvCache.of(t[0], t[1], s[0], s[1]), codes, scales


def same(cache, codes, scales, fmt):
    for t, s, c, x in ((cache.k, cache.k_scale, codes[0], scales[0]),
                       (cache.v, cache.v_scale, codes[1], scales[1])):
        assert np.array_equal(s.cpu().numpy().astype(np.float64), x)
        got = ref.to_bytes(t)
        if fmt == "e4m3":
            nan = (c & 127) == 127
            assert np.array_equal(nan, (got & 127) == 127)
            got, c = np.where(nan, 0, got), np.where(nan, 0, c)
        assert np.array_equal(got, c)


def slots_of(rng, n, bt, counts):
    """Slots of requests with (had, new) tokens, in blocks of a random order; some tokens skipped."""
    perm, at, out = rng.permutation(n), 0, []
    for had, new in counts:
        first = had // bt
        blocks = perm[at:at + -(-(had + new) // bt) - first]
        at += len(blocks)
        p = np.arange(had, had + new)
        out.append(blocks[p // bt - first] * bt + p % bt)
    assert at <= n
    return np.concatenate(out)


def run(rng, counts, H, bt, d, fmt, dtype, make_x, skip=0.0, strided=False, offset=0):
    n = sum(-(-(a + b) // bt) - a // bt for a, b in counts) + 2
    cache, codes, scales = make(rng, n, H, bt, d, fmt)
    slots = slots_of(rng, n, bt, counts)
    slots[rng.random(len(slots)) < skip] = -1
    T = len(slots)
    k, v = (make_x(rng, (T, H, d)) for _ in range(2))
    if strided:
        both = torch.zeros((T, 2 * H * d + offset + 5), dtype=ref.DTYPES[dtype], device="cuda")
        kt, vt = (both[:, o:o + H * d].view(T, H, d) for o in (offset, offset + H * d))
    else:
        kt, vt = (torch.zeros((T, H, d), dtype=ref.DTYPES[dtype], device="cuda") for _ in range(2))
    kt.copy_(torch.from_numpy(k).cuda())
    vt.copy_(torch.from_numpy(v).cuda())
    hs.hs_kv_append(cache, kt, vt, torch.from_numpy(slots.astype(np.int32)).cuda())
    hs.hs_get_device_error()
    for x, c, s in ((kt, codes[0], scales[0]), (vt, codes[1], scales[1])):
        ref.append(x.double().cpu().numpy(), slots, c, s, fmt)
    same(cache, codes, scales, fmt)
    return cache


def normal(rng, shape):
    return rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[-1]))


COUNTS = {
    "one": [(0, 1)],
    "one_more": [(7, 1)],
    "step": [(5 * i, 1) for i in range(64)],
    "prompts": [(0, 300), (0, 1), (0, 128), (0, 77), (0, 256)],
    "chunks": [(3, 200), (15, 1), (16, 17), (127, 130), (64, 64), (1, 9)],
}


@pytest.mark.parametrize("counts", sorted(COUNTS))
@pytest.mark.parametrize("bt,d", [(16, 64), (16, 128), (32, 256), (64, 128), (128, 64), (128, 256)])
@pytest.mark.parametrize("fmt,dtype", [("e4m3", "bf16"), ("int8", "fp16")])
def test_append(counts, bt, d, fmt, dtype):
    rng = np.random.default_rng(bt + d)
    run(rng, COUNTS[counts], 3, bt, d, fmt, dtype, normal)


@pytest.mark.parametrize("fmt,dtype", [("e4m3", "fp16"), ("int8", "bf16")])
@pytest.mark.parametrize("offset", [0, 8, 1])
def test_views_of_a_packed_tensor_with_skipped_tokens(fmt, dtype, offset):
    """Odd strides and offsets: no 16-byte loads.  A skipped token ends its run."""
    rng = np.random.default_rng(offset)
    counts = [(3, 1), (9, 30), (0, 64), (40, 2)] * 5
    n_skip = 0.0 if offset == 8 else 0.02
    run(rng, counts, 1 if n_skip else 5, 128, 64, fmt, dtype, normal, strided=True, offset=offset)
    slots = [0, 1, -1, 16, 17, -1, -1, 32]             # one run a block
    cache, codes, scales = make(rng, 4, 2, 16, 64, fmt)
    x = torch.from_numpy(normal(rng, (8, 2, 64))).cuda().to(ref.DTYPES[dtype])
    hs.hs_kv_append(cache, x, x, torch.tensor(slots, dtype=torch.int32, device="cuda"))
    for c, s in zip(codes, scales):
        ref.append(x.double().cpu().numpy(), np.array(slots), c, s, fmt)
    same(cache, codes, scales, fmt)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_edges_of_the_scale(fmt):
    """Magnitudes on both sides of every bound of the scale, zeros, subnormals, the largest, and
    values that saturate or are no number."""
    top = ref.LARGEST[fmt]
    rows = [0.0, top, top * 2.0 ** -7, 2.0 ** -133, 2.0 ** -126, 3.3895e38, 2.0 ** 100, 1.0]
    above = 450.0 if fmt == "e4m3" else 127.5          # the next bf16 number after it
    rows += [above * 2.0 ** e for e in (-3, 0, 5)]
    x = torch.zeros((len(rows) + 2, 1, 64), dtype=torch.bfloat16)
    for i, r in enumerate(rows):
        x[i, 0] = torch.linspace(-1, 1, 64).double().mul(r).to(torch.bfloat16)
        x[i, 0, 5] = r
    x[len(rows), 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 2.0])
    x[len(rows) + 1, 0, 1] = float("nan")
    x = x.cuda()
    rng = np.random.default_rng(0)
    n = len(x)
    cache, codes, scales = make(rng, n, 1, 16, 64, fmt)
    slots = np.arange(n) * 16
    hs.hs_kv_append(cache, x, x, torch.from_numpy(slots.astype(np.int32)).cuda())
    for c, s in zip(codes, scales):
        ref.append(x.double().cpu().numpy(), slots, c, s, fmt)
    same(cache, codes, scales, fmt)
    # and the next token of each block, from the other end: older codes follow
    y = x.flip(0).contiguous()
    hs.hs_kv_append(cache, y, y, torch.from_numpy((slots + 1).astype(np.int32)).cuda())
    for c, s in zip(codes, scales):
        ref.append(y.double().cpu().numpy(), slots + 1, c, s, fmt)
    same(cache, codes, scales, fmt)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_token_by_token_as_at_once(fmt):
    """Growing magnitudes one token at a time: the scales end as of one call, the values within a
    rounding of each growth (half a step of the last scale each, for the last and a quarter, an
    eighth, ... for those before: less than one step in all)."""
    rng = np.random.default_rng(9)
    bt, d, T = 16, 128, 16
    x = rng.standard_normal((T, 2, d)) * np.exp2(np.arange(T) / 3.0)[:, None, None]
    x = torch.from_numpy(x).cuda().to(torch.bfloat16)
    one = hs.KvCache(3, bt, 2, d, ref.CODES[fmt])
    more = hs.KvCache(3, bt, 2, d, ref.CODES[fmt])
    slots = torch.arange(bt, 2 * bt, dtype=torch.int32, device="cuda")
    hs.hs_kv_append(one, x, x, slots)
    for t in range(T):
        hs.hs_kv_append(more, x[t:t + 1], x[t:t + 1], slots[t:t + 1])
    assert torch.equal(one.k_scale[1], more.k_scale[1])
    s = one.k_scale[1].double().cpu().numpy()[:, None, None]
    for c in (more.k, more.v):
        y = ref.values(ref.to_bytes(c)[1], fmt) * s
        ex = x.double().cpu().numpy().transpose(1, 0, 2)
        step = s if fmt == "int8" else np.maximum(np.exp2(np.floor(np.log2(np.abs(ex) + 1e-300)) - 3),
                                                  s * 2.0 ** -9)
        assert (np.abs(y - ex) <= step).all()


def test_slots_out_of_range_are_left_out():
    rng = np.random.default_rng(4)
    cache, codes, scales = make(rng, 2, 1, 16, 64, "int8")
    x = torch.ones((2, 1, 64), dtype=torch.float16, device="cuda")
    hs.hs_kv_append(cache, x, x, torch.tensor([32, 3], dtype=torch.int32, device="cuda"))
    with pytest.raises(hs.HsError):
        hs.hs_get_device_error()
    for c, s in zip(codes, scales):
        ref.append(np.ones((1, 1, 64)), np.array([3]), c, s, "int8")
    same(cache, codes, scales, "int8")


def test_offsets_past_32_bits():
    """A cache of more than 2^32 values: the last block's codes lie past a 32-bit offset."""
    H, bt, d = 64, 64, 256
    n = (1 << 32) // (H * bt * d) + 2
    cache = hs.KvCache(n, bt, H, d, torch.int8)
    x = torch.randn((3, H, d), device="cuda").to(torch.bfloat16)
    first = (n - 1) * bt
    cache.k[0] = 0
    hs.hs_kv_append(cache, x, x, torch.arange(first, first + 3, dtype=torch.int32, device="cuda"))
    hs.hs_get_device_error()
    codes, scale = np.zeros((1, H, bt, d), np.uint8), np.zeros((1, H))
    ref.append(x.double().cpu().numpy(), np.arange(3), codes, scale, "int8")
    assert np.array_equal(ref.to_bytes(cache.k[n - 1])[:, :3], codes[0, :, :3])
    assert np.array_equal(cache.v_scale[n - 1].cpu().numpy(), scale[0])
    assert not cache.k[0].any()


def test_refusals():
    cache = hs.KvCache(4, 16, 2, 64)
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    s = torch.arange(3, dtype=torch.int32, device="cuda")
    for bad in (x.float(), x.cpu()):
        with pytest.raises(TypeError):
            hs.hs_kv_append(cache, bad, x, s)
    for bad in (x[:, :1], x[..., :32], x.transpose(0, 1), x.to(torch.float16), x[:2]):
        with pytest.raises(ValueError):
            hs.hs_kv_append(cache, x, bad, s)
    with pytest.raises(ValueError):
        hs.hs_kv_append(cache, x, x, s[:2])
    with pytest.raises(TypeError):
        hs.hs_kv_append(cache, x, x, s.long())
    with pytest.raises(TypeError):
        hs.KvCache(4, 16, 2, 64, torch.float16)
    for shape in ((4, 24, 2, 64), (4, 16, 2, 96)):
        c = hs.KvCache(*shape)
        y = torch.zeros((1, 2, shape[3]), dtype=torch.bfloat16, device="cuda")
        with pytest.raises(hs.HsError) as e:
            hs.hs_kv_append(c, y, y, s[:1])
        assert e.value.status == hs.HS_ERR_UNSUPPORTED
