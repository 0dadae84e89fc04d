"""The paged cache of keys and values that the merged model calls of a batch share, as cases that
can be timed and compared.

Workflows are merged before they run, so a model call that several of them ask for runs once, for
one request.  A program that runs those requests keeps their keys and values in blocks of tokens,
8 bits a value with one scale for each block and head, and does three things a step:

  tables   gives every request the blocks that its new tokens need, and every new token its slot
  append   writes the new tokens' keys and values into their slots, rounded to 8 bits; a block
           that was begun earlier keeps one scale, so its codes follow where the scale grows
  attend   attention of the new tokens' queries over all that their request has in the cache

A code c of block b and head h stands for c * scale[b, h].  The scale is the least power of two
(not below 2^-126) that brings the block's largest finite magnitude to at most 448 (e4m3) or 127
(int8), rounding is to nearest even, and what is larger saturates.
"""
import math

import numpy as np
import torch

own = False

LISTED = [
    # One decoding step of 64 workflows' requests: a new token each, a new block for a few.
    dict(name="tables_step", kind="tables", R=64, bt=16, lo=200, hi=1500, nlo=1, nhi=1),
    # A batch of merged prompts, all new: the whole table and a slot for each of 413,000 tokens.
    dict(name="tables_prompts", kind="tables", R=1434, bt=32, lo=0, hi=0, nlo=64, nhi=512),
    # The same decoding step's keys and values, one layer: almost all latency.
    dict(name="append_step", kind="append", R=64, bt=16, lo=200, hi=1500, nlo=1, nhi=1,
         H=8, d=128, fmt="e4m3", dtype="bf16", packed=True),
    # 512 prompts of up to 512 tokens written at once: bound by memory.
    dict(name="append_prompts", kind="append", R=512, bt=64, lo=0, hi=0, nlo=64, nhi=512,
         H=8, d=128, fmt="int8", dtype="bf16", packed=False),
    # Ragged chunks that begin inside a block, an odd number of heads, cut out of a packed tensor.
    dict(name="append_chunks", kind="append", R=37, bt=32, lo=1, hi=700, nlo=1, nhi=333,
         H=5, d=64, fmt="e4m3", dtype="fp16", packed=True),
    # One user with a long context, one new token: the long axis is all the parallelism there is.
    dict(name="attend_one", kind="attend", R=1, bt=16, lo=32771, hi=32771, nlo=1, nhi=1,
         H=8, G=4, d=128, fmt="e4m3", dtype="bf16", causal=True, window=0),
    # A small batch of short answers: latency.
    dict(name="attend_few", kind="attend", R=8, bt=16, lo=100, hi=1500, nlo=1, nhi=1,
         H=8, G=4, d=128, fmt="e4m3", dtype="bf16", causal=True, window=0),
    # A full batch, ragged from a few tokens to 8192: bound by reading the cache.
    dict(name="attend_step", kind="attend", R=256, bt=64, lo=1, hi=8192, nlo=1, nhi=1,
         H=8, G=4, d=128, fmt="e4m3", dtype="bf16", causal=True, window=0),
    # Five drafted tokens checked at once, int8, heads of 64, a sliding window.
    dict(name="attend_draft", kind="attend", R=48, bt=32, lo=5, hi=3001, nlo=5, nhi=5,
         H=4, G=6, d=64, fmt="int8", dtype="fp16", causal=True, window=1024),
    # Prompts of up to 2048 tokens from nothing: bound by the products.
    dict(name="attend_prompts", kind="attend", R=16, bt=64, lo=0, hi=0, nlo=256, nhi=2048,
         H=8, G=4, d=128, fmt="e4m3", dtype="bf16", causal=True, window=0),
    # Chunks of a long document appended to what is there, beside requests that decode.
    dict(name="attend_chunks", kind="attend", R=6, bt=32, lo=1000, hi=12000, nlo=1, nhi=1024,
         H=4, G=8, d=128, fmt="int8", dtype="bf16", causal=True, window=0),
    # Cross attention: queries of one length over an encoder's states of another, nothing hidden.
    dict(name="attend_cross", kind="attend", R=12, bt=16, lo=700, hi=1500, nlo=1, nhi=448,
         H=16, G=1, d=64, fmt="e4m3", dtype="fp16", causal=False, window=0),
]


def listed():
    return [dict(c) for c in LISTED]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "append", "append", "attend", "attend", "attend", "attend"])
    bt = rng.choice([16, 32, 64, 128])
    if kind == "tables":
        R = _log(rng, 1, 4096)
        nhi = min(rng.choice([1, 1, _log(rng, 2, 512)]), 400000 // R + 1)
        hi = _log(rng, 1, 8192)
        return dict(kind=kind, R=R, bt=bt, lo=rng.randint(0, hi), hi=hi,
                    nlo=1 if nhi == 1 else rng.randint(0, nhi - 1), nhi=nhi)
    heads = dict(bt=bt, H=rng.randint(1, 12), d=rng.choice([64, 128, 128, 256]),
                 fmt=rng.choice(["e4m3", "e4m3", "int8"]), dtype=rng.choice(["bf16", "bf16", "fp16"]))
    if kind == "append":
        nhi = rng.choice([1, _log(rng, 2, 512)])
        tokens = 60_000_000 // (heads["H"] * heads["d"])        # 147 M values are the largest listed
        R = _log(rng, 1, max(1, min(512, tokens // nhi)))
        hi = _log(rng, 1, 1000)
        return dict(heads, kind=kind, R=R, lo=rng.randint(0, hi), hi=hi,
                    nlo=1 if nhi == 1 else rng.randint(0, nhi - 1), nhi=nhi,
                    packed=rng.random() < 0.5)
    G = rng.choice([1, 2, 3, 4, 4, 6, 8, 16])
    heads["H"] = min(heads["H"], 64 // G)
    nhi = rng.choice([1, 1, _log(rng, 2, 8), _log(rng, 9, 1024)])
    hi = _log(rng, 16, 16384)
    # At most half of the largest listed case's reads, and of the largest one's products.
    at_most = min(400_000_000 // (heads["H"] * heads["d"] * (hi + G * nhi)),
                  40_000_000_000 // (heads["H"] * G * heads["d"] * (hi + nhi) * nhi))
    R = _log(rng, 1, max(1, min(256, at_most)))
    causal = rng.random() < 0.8
    return dict(heads, kind=kind, R=R, G=G, lo=rng.randint(0, hi), hi=hi,
                nlo=nhi if nhi <= 8 else rng.randint(0, nhi), nhi=nhi, causal=causal,
                window=_log(rng, 16, 4096) if causal and rng.random() < 0.2 else 0)


# ---- lengths: spread evenly over their range, so that the work is the case's and not the seed's ----
def _spread(lo, hi, R):
    return np.floor(lo + (hi - lo + 1) * (np.arange(R) + 0.5) / R).astype(np.int64).clip(lo, hi)


def _counts(case):
    """(tokens in the cache before, new tokens) of each request, in an order of their own."""
    have = _spread(case["lo"], case["hi"], case["R"])
    fresh = _spread(case["nlo"], case["nhi"], case["R"])
    return have, fresh[np.random.RandomState(7).permutation(case["R"])]


def _lens(case):
    """(tokens in the cache, queries) of each request of an attend case: what its new tokens add
    is in the cache already; an encoder's states are as many as they are."""
    have, n = _counts(case)
    if not case["causal"]:
        return have, n
    return (have + n if case["nhi"] > 8 else np.maximum(have, n)), n


DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
LARGEST = {"e4m3": 448.0, "int8": 127.0}


# ---- the 8-bit form in elementary operations ---------------------------------------------------
def _scale(m, fmt):
    """The least power of two s >= 2^-126 with m <= LARGEST * s, for float32 m >= 0."""
    f, e = torch.frexp(m)                                  # m = f * 2^e, 0.5 <= f < 1
    full, bits = (0.875, 9) if fmt == "e4m3" else (0.9921875, 7)
    e = e - bits + (f > full).to(e.dtype)
    e = torch.where(m > 0, e, -126).clamp(min=-126)
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _round(x, fmt):
    """float32 multiples of a scale, rounded to codes."""
    if fmt == "e4m3":
        return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return torch.nan_to_num(x, nan=0.0).round().clamp(-127, 127).to(torch.int8)


def _bytes(codes):
    return codes.view(torch.uint8)


def _finite_max(x):
    return torch.where(x.isfinite(), x.abs(), 0.0)


def _values(codes, scale, ids):
    """What blocks `ids` [R, nb] of codes [n, H, bt, d] stand for: float32 [R, H, nb * bt, d]."""
    R, nb = ids.shape
    _, H, bt, d = codes.shape
    c = _bytes(codes)[ids].view(codes.dtype).to(torch.float32)
    c *= scale[ids][..., None, None]
    return c.transpose(1, 2).reshape(R, H, nb * bt, d)


# ---- inputs ------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


def _normal(shape, g, dtype):
    """Keys or values as a model has them: normal, with a few channels that are larger."""
    x = torch.randn(shape, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(shape[-1], generator=g, device="cuda"))
    return x.to(dtype)


def _blocks(lens, width, bt, g, spare):
    """A table [R, width] of distinct blocks for `lens` tokens a request (-1 past them), the number
    of blocks, and the others in an order of their own."""
    need = -(-lens // bt)
    n = int(need.sum()) + spare
    perm = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
    col = torch.arange(width, device="cuda")[None]
    need_d = _dev(need, torch.int64)
    at = (need_d.cumsum(0) - need_d)[:, None] + col
    table = torch.where(col < need_d[:, None], perm[at.clamp(max=n - 1)], -1).to(torch.int32)
    return table.contiguous(), n, perm[int(need.sum()):]


def _cache(case, n, g):
    """Codes and scales of n blocks, as an earlier program left them."""
    H, bt, d = case["H"], case["bt"], case["d"]
    got = []
    for _ in range(2):
        codes = torch.empty((n, H, bt, d), dtype=CODES[case["fmt"]], device="cuda")
        scale = torch.empty((n, H), device="cuda")
        step = max(1, (1 << 27) // (H * bt * d))
        for i in range(0, n, step):
            x = _normal((min(step, n - i), H, bt, d), g, torch.float32)
            scale[i:i + step] = _scale(x.abs().amax((2, 3)), case["fmt"])
            codes[i:i + step] = _round(x / scale[i:i + step, :, None, None], case["fmt"])
        got += [codes, scale]
    return got


def _stale(case, s, lens):
    """What no token was written to yet: a NaN (int8: the largest code) in every slot past a
    request's end."""
    bt = case["bt"]
    r = np.nonzero(lens % bt)[0]
    if not len(r):
        return
    ids = s["table"][_dev(r, torch.int64), _dev(lens[r] // bt, torch.int64)].long()
    past = torch.arange(bt, device="cuda")[None] >= _dev(lens[r] % bt)[:, None]
    for c in (s["k_codes"], s["v_codes"]):
        b = _bytes(c)
        b[ids] = torch.where(past[:, None, :, None], 0x7F, b[ids])


def prepare(case, seed):
    g = _gen(seed)
    R, bt = case["R"], case["bt"]
    order = torch.randperm(R, generator=g, device="cuda").cpu().numpy()
    s = {"case": case}
    if case["kind"] == "attend":
        lens, n = (x[order] for x in _lens(case))
        width = max(1, int(-(-lens.max() // bt)))
        s["table"], blocks, _ = _blocks(lens, width, bt, g, 16)
        s["k_codes"], s["k_scale"], s["v_codes"], s["v_scale"] = _cache(case, blocks, g)
        _stale(case, s, lens)
        T = int(n.sum())
        s["q"] = _normal((T, case["H"] * case["G"], case["d"]), g, DTYPES[case["dtype"]])
        s["lens"], s["max_q"] = _dev(lens), int(n.max())
        s["starts"] = _dev(np.concatenate([[0], np.cumsum(n)]))
        return s
    have, fresh = (x[order] for x in _counts(case))
    T, lens = int(fresh.sum()), have + fresh
    width = max(1, int(-(-lens.max() // bt)))
    s["have"], s["fresh"], s["tokens"] = _dev(have), _dev(fresh), T
    if case["kind"] == "tables":
        need = int((-(-lens // bt) - -(-have // bt)).sum())
        s["table"], n, rest = _blocks(have, width, bt, g, need + 64)
        s["pool"] = torch.zeros(n, dtype=torch.int32, device="cuda")
        taken = int(torch.randint(n, (1,), generator=g, device="cuda"))
        at = (taken + torch.arange(len(rest), device="cuda")) % n        # the free blocks, in a ring
        s["pool"][at] = rest
        s["cursor"] = _dev(np.array([taken, taken + len(rest)]), torch.int64)
        return s
    table, n, _ = _blocks(lens, width, bt, g, 8)
    s["k_codes"], s["k_scale"], s["v_codes"], s["v_scale"] = _cache(case, n, g)
    r = np.repeat(np.arange(R), fresh)
    pos = _dev(have[r] + np.arange(T) - np.repeat(np.cumsum(fresh) - fresh, fresh), torch.int64)
    s["slots"] = (table[_dev(r, torch.int64), pos // bt] * bt + pos % bt).to(torch.int32)
    H, d, dtype = case["H"], case["d"], DTYPES[case["dtype"]]
    if case["packed"]:                                  # queries, keys and values in one tensor
        qkv = _normal((T, 3 * H, d), g, dtype)
        s["k"], s["v"] = qkv[:, H:2 * H], qkv[:, 2 * H:]
    else:
        s["k"], s["v"] = _normal((T, H, d), g, dtype), _normal((T, H, d), g, dtype)
    return s


# ---- the plain forms ---------------------------------------------------------------------------
def _plain_tables(s):
    bt, table, T = s["case"]["bt"], s["table"], s["tokens"]
    have, fresh = s["have"].long(), s["fresh"].long()
    first, last = -(-have // bt), -(-(have + fresh) // bt)
    need = last - first
    zero = have.new_zeros(1)
    starts = torch.cat([zero, fresh.cumsum(0)])
    taken = s["cursor"][:1]
    col = torch.arange(table.shape[1], device="cuda")[None]
    at = taken + (need.cumsum(0) - need - first)[:, None] + col
    new = (col >= first[:, None]) & (col < last[:, None])
    table = torch.where(new, s["pool"][at % len(s["pool"])], table)
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    pos = have[r] + t - starts[r]
    slots = table[r, pos // bt] * bt + (pos % bt).to(torch.int32)
    return {"table": table, "slots": slots, "starts": starts.to(torch.int32),
            "lens": (have + fresh).to(torch.int32),
            "cursor": s["cursor"] + torch.cat([need.sum()[None], zero])}


def _plain_append(x, codes, scale, slots, fmt):
    """Writes x [T, H, d] to the slots, in place."""
    n, H, bt, d = codes.shape
    x = x.to(torch.float32)
    block, off = slots.long() // bt, slots.long() % bt
    m = torch.zeros((n, H), device="cuda")
    m.index_reduce_(0, block, _finite_max(x).amax(2), "amax")
    begin = torch.full((n,), bt, device="cuda").index_reduce_(0, block, off, "amin")
    touched = begin < bt
    grown = torch.where((begin > 0)[:, None], torch.maximum(scale, _scale(m, fmt)), _scale(m, fmt))
    new = torch.where(touched[:, None], grown, scale)
    # The codes that a block had before follow its scale.
    ids = block[(off == begin[block])]                  # one token of each touched block
    b = _bytes(codes)
    old = b[ids].view(codes.dtype).to(torch.float32) * (scale[ids] / new[ids])[..., None, None]
    before = torch.arange(bt, device="cuda")[None] < begin[ids][:, None]
    b[ids] = torch.where(before[:, None, :, None], _bytes(_round(old, fmt)), b[ids])
    b[block, :, off] = _bytes(_round(x / new[block][..., None], fmt))
    scale.copy_(new)
    return codes, scale


def _plain_attend(s):
    c, lens, starts, n = s["case"], s["lens"].long(), s["starts"].long(), s["max_q"]
    H, G, d, bt = c["H"], c["G"], c["d"], c["bt"]
    R, L, T = len(lens), s["table"].shape[1] * bt, len(s["q"])
    ids = s["table"].clamp(min=0).long()
    key = torch.arange(L, device="cuda")
    gone = (key[None] >= lens[:, None])[:, None, :, None]
    K = _values(s["k_codes"], s["k_scale"], ids).masked_fill_(gone, 0.0)
    V = _values(s["v_codes"], s["v_scale"], ids).masked_fill_(gone, 0.0)
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    i = t - starts[r]
    q = torch.zeros((R, n, H, G, d), device="cuda")
    q[r, i] = s["q"].to(torch.float32).view(T, H, G, d)
    q = q.permute(0, 2, 1, 3, 4).reshape(R, H, n * G, d)
    S = (q @ K.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(R, H, n, G, L)
    pos = (lens - starts.diff())[:, None] + torch.arange(n, device="cuda")        # of each query
    seen = (key < lens[:, None, None]).expand(R, n, L)
    if c["causal"]:
        seen = seen & (key <= pos[..., None])
    if c["window"]:
        seen = seen & (key > pos[..., None] - c["window"])
    S.masked_fill_(~seen[:, None, :, None], -math.inf)
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    S.sub_(m).exp_()
    total = S.sum(-1, keepdim=True)
    o = (S.view(R, H, n * G, L) @ V).view(R, H, n, G, d)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (m + total.log())[..., 0]                                               # R, H, n, G
    return {"out": o[r, :, i].reshape(T, H * G, d).to(s["q"].dtype),
            "lse": lse[r, :, i].reshape(T, H * G)}


# ---- one pass ----------------------------------------------------------------------------------
def _handle(s):
    """The cache as the framework has it and its workspace, kept with the state."""
    if "handle" not in s:
        import paper_2607_22578_gb300 as hs
        cache = hs.KvCache.of(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"])
        c, ws = s["case"], None
        if c["kind"] == "attend":
            ws = torch.zeros(hs.hs_kv_attend_workspace(cache, c["H"] * c["G"], s["max_q"]),
                             dtype=torch.uint8, device="cuda")
        s["handle"] = (hs, cache, ws)
    return s["handle"]


def run(s):
    c = s["case"]
    if c["kind"] == "tables":
        if own:
            import paper_2607_22578_gb300 as hs
            slots, starts, lens, cursor = hs.hs_kv_tables(s["have"], s["fresh"], s["table"], s["pool"],
                                                          s["cursor"], c["bt"], s["tokens"])
            return {"table": s["table"], "slots": slots, "starts": starts, "lens": lens,
                    "cursor": cursor}
        return _plain_tables(s)
    if c["kind"] == "append":
        if own:
            hs, cache, _ = _handle(s)
            hs.hs_kv_append(cache, s["k"], s["v"], s["slots"])
        else:
            _plain_append(s["k"], s["k_codes"], s["k_scale"], s["slots"], c["fmt"])
            _plain_append(s["v"], s["v_codes"], s["v_scale"], s["slots"], c["fmt"])
        # The updated cache: e4m3 or int8 values, each with its block's scale.
        return {k: s[k] for k in ("k_codes", "k_scale", "v_codes", "v_scale")}
    if own:
        hs, cache, ws = _handle(s)
        out, lse = hs.hs_kv_attend(cache, s["q"], s["lens"], s["table"], starts=s["starts"],
                                   max_q=s["max_q"], causal=c["causal"], window=c["window"],
                                   workspace=ws)
        return {"out": out, "lse": lse}
    return _plain_attend(s)


# ---- what a pass cannot do without -------------------------------------------------------------
def _seen(case, L, n):
    """(tokens of the cache that some query sees, pairs of a query and a key that it sees)."""
    if n == 0 or L == 0:
        return 0, 0
    if not case["causal"]:
        return L, L * n
    p = L - n + np.arange(n)                                # the queries' positions
    p = p[p >= 0]
    w = case["window"] or L + 1
    return (int(L - max(0, p[0] - w + 1)), int(np.minimum(p + 1, w).sum())) if len(p) else (0, 0)


def work(case):
    bt = case["bt"]
    if case["kind"] == "tables":
        have, fresh = _counts(case)
        new = int((-(-(have + fresh) // bt) - -(-have // bt)).sum())
        # lengths read and written, the free list read, new entries and slots written
        return {"bytes": 4 * (4 * case["R"] + 2 * new + int(fresh.sum())), "flops": 0}
    if case["kind"] == "append":
        have, fresh = _counts(case)
        T, touched = int(fresh.sum()), int((-(-(have + fresh) // bt) - have // bt).sum())
        # 16-bit values read, codes written, a slot for each token and a scale for each block
        return {"bytes": T * (2 * case["H"] * case["d"] * 3 + 4) + 16 * touched * case["H"],
                "flops": 0}
    lens, n = _lens(case)
    seen = [_seen(case, int(a), int(b)) for a, b in zip(lens, n)]
    keys, pairs = (sum(x) for x in zip(*seen))
    Hq = case["H"] * case["G"]
    tokens = int(n.sum())
    return {"bytes": keys * 2 * case["H"] * case["d"] + keys // bt * (4 + 8 * case["H"])
            + tokens * Hq * (4 * case["d"] + 4),
            "flops": 4 * pairs * Hq * case["d"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------
def _exact_cache(x, codes, scale, slots, fmt):
    codes, scale = codes.to(torch.float32).double(), scale.double()
    n, H, bt, d = codes.shape
    x = x.double()
    top = LARGEST[fmt]

    def rounded(y):
        y = y.clamp(-top, top)
        if fmt == "int8":
            return y.round()
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        return (y / step).round() * step

    slots = slots.cpu().numpy().astype(np.int64)
    cut = np.nonzero(np.diff(slots // bt, prepend=-1))[0]          # where a block's tokens begin
    for a, b in zip(cut, np.append(cut[1:], len(slots))):
        at, o = int(slots[a]) // bt, int(slots[a]) % bt
        m = x[a:b].abs().amax((0, 2)).clamp(min=top * 2.0 ** -126)
        new = torch.exp2(torch.round(torch.log2(m / top)))         # then to the side that holds m
        new = torch.where(m > top * new, 2 * new, new)
        if o:
            new = torch.maximum(new, scale[at])
            codes[at, :, :o] = rounded(codes[at, :, :o] * (scale[at] / new)[:, None, None])
        scale[at] = new
        codes[at, :, o:o + b - a] = rounded(x[a:b] / new[:, None]).transpose(0, 1)
    return (codes if fmt == "e4m3" else None), scale


def exact(case, seed):
    if case["kind"] == "tables":
        return None
    s = prepare(case, seed)
    if case["kind"] == "append":
        if case["R"] * -(-case["nhi"] // case["bt"]) > 3000:
            return None
        kc, ks = _exact_cache(s["k"], s["k_codes"], s["k_scale"], s["slots"], case["fmt"])
        vc, vs = _exact_cache(s["v"], s["v_codes"], s["v_scale"], s["slots"], case["fmt"])
        return {"k_codes": kc, "k_scale": ks, "v_codes": vc, "v_scale": vs}
    if work(case)["flops"] > 4e12:
        return None
    H, G, d, bt = case["H"], case["G"], case["d"], case["bt"]
    lens, starts = s["lens"].tolist(), s["starts"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for r, L in enumerate(lens):
        a, b = starts[r], starts[r + 1]
        n = b - a
        if n == 0 or L == 0:
            continue
        ids = s["table"][r, :-(-L // bt)].long()
        k, v = ((c.view(torch.uint8)[ids].view(c.dtype).to(torch.float32).double()
                 * f[ids].double()[..., None, None]).transpose(0, 1).reshape(H, -1, d)[:, :L]
                for c, f in ((s["k_codes"], s["k_scale"]), (s["v_codes"], s["v_scale"])))
        pos = torch.arange(L - n, L, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None]
        hidden = torch.zeros((n, L), dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= j > pos
        if case["window"]:
            hidden |= j <= pos - case["window"]
        for h in range(H):
            q = s["q"][a:b, h * G:(h + 1) * G].double().transpose(0, 1)
            z = (q @ k[h].T / math.sqrt(d)).masked_fill(hidden, -math.inf)
            e = torch.logsumexp(z, -1)
            p = torch.where(e[..., None] == -math.inf, 0.0, torch.exp(z - e[..., None]))
            out[a:b, h * G:(h + 1) * G] = (p @ v[h]).transpose(0, 1)
            lse[a:b, h * G:(h + 1) * G] = e.T
    return {"out": out, "lse": lse}
