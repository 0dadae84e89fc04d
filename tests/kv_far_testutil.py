"""Attention over the paged cache in 64 bits with bounds that follow a row's
own keys: what a query does not see, or sees with no weight, allows no error."""
from __future__ import annotations

import math

import numpy as np
import torch

import kv_testutil as ref
import paper_2607_22578_gb300 as hs


def dev(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def layout(lens, bt, rng, spare=3):
    """(table int32 [n_req, width], number of blocks): blocks of a random order."""
    need = [-(-L // bt) for L in lens]
    perm = rng.permutation(sum(need) + spare)
    table, at = np.full((len(lens), max(1, max(need))), -1), 0
    for r, m in enumerate(need):
        table[r, :m] = perm[at:at + m]
        at += m
    return table, len(perm)


def queries(T, heads, d, dtype, g, size=1.0):
    return (size * torch.randn((T, heads, d), generator=g, device="cuda")).to(ref.DTYPES[dtype])


def written(lens, n, H, G, d, bt, fmt, dtype, values, seed=0, size=1.0):
    """Requests whose keys and values hs_kv_append wrote: normal, the values changed by
    values(v float32 [T, H, d], request [T], position [T])."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    table, blocks = layout(lens, bt, rng)
    r = np.repeat(np.arange(len(lens)), lens)
    pos = np.concatenate([np.arange(L) for L in lens]).astype(np.int64)
    slots = table[r, pos // bt] * bt + pos % bt
    k, v = (torch.randn((len(r), H, d), generator=g, device="cuda") for _ in range(2))
    v = values(v, torch.from_numpy(r).cuda(), torch.from_numpy(pos).cuda())
    cache = hs.KvCache(blocks, bt, H, d, ref.CODES[fmt])
    cache.k.view(torch.uint8).fill_(0x7F)                 # what no token is written to
    cache.v.view(torch.uint8).fill_(0x7F)
    hs.hs_kv_append(cache, k.to(ref.DTYPES[dtype]), v.to(ref.DTYPES[dtype]), dev(slots.tolist()))
    hs.hs_get_device_error()
    return dict(cache=cache, q=queries(sum(n), H * G, d, dtype, g, size), fmt=fmt,
                table=dev(table.tolist()), lens=list(lens),
                starts=np.concatenate([[0], np.cumsum(n)]).tolist())


def call(p, causal=True, window=0, **kw):
    return hs.hs_kv_attend(p["cache"], p["q"], dev(p["lens"]), p["table"], starts=dev(p["starts"]),
                           max_q=int(np.diff(p["starts"]).max()), causal=causal, window=window, **kw)


def sees(L, n, causal, window, device="cuda"):
    """bool [n, L]: which keys each query sees."""
    i = torch.arange(n, device=device)[:, None] + (L - n)
    j = torch.arange(L, device=device)[None]
    see = torch.ones((n, L), dtype=torch.bool, device=device)
    if causal:
        see &= j <= i
    if window:
        see &= j > i - window
    return see


def attend(p, causal=True, window=0):
    """(out, lse, tol_out, tol_lse) in float64.  Hidden keys and values are not looked at, whatever
    they hold.  With p the normalised weights, vs a token's value scale and c its codes, a row's
    bounds over the keys that it sees:
      scores: fp32 sums of up to 256 products and q to 2^-24 of its row's largest: 2^-18 S, with S
        the largest sum of magnitudes of a score; for lse too, and 2^-20 of itself for exp and log
      weights: 2^-11 each as half, 2 * 2^-18 S from the score, 2^-14 for exponents, sums and the
        division, all of p |v|
      what is small as half: weights p vs are taken relative to their largest, which is at least
        2^7, and half's least step is 2^-24: 2^-32 max(p vs) |c| each
      weights under 2^-126 of the largest may be dropped: 2^-126 |v| each
    (the output's own rounding is the caller's to add)."""
    c = p["cache"]
    T, Hq, d = p["q"].shape
    H, bt = c.n_kv_heads, c.block_tokens
    G = Hq // H
    lut = torch.from_numpy(ref.e4m3_values()).cuda()
    out = torch.zeros((T, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    tol, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    for r, L in enumerate(p["lens"]):
        a, b = p["starts"][r], p["starts"][r + 1]
        n = b - a
        if n == 0 or L == 0:
            continue
        ids = p["table"][r, :-(-L // bt)].long()
        see = sees(L, n, causal, window)
        used = see.any(0)

        def of(codes, scale):
            x = lut[codes.view(torch.uint8)[ids].long()] if p["fmt"] == "e4m3" else codes[ids].double()
            x = x.transpose(0, 1).reshape(H, -1, d)[:, :L]
            s = scale[ids].double().T.repeat_interleave(bt, 1)[:, :L]
            return torch.where(used[:, None], x, 0.0), torch.where(used, s, 0.0)

        kc, ks = of(c.k, c.k_scale)
        vc, vs = of(c.v, c.v_scale)
        for h in range(Hq):
            x = p["q"][a:b, h].double()
            K, C, s_v = kc[h // G] * ks[h // G][:, None], vc[h // G], vs[h // G]
            s = (x @ K.T * d ** -0.5).masked_fill(~see, -math.inf)
            m = s.amax(1, keepdim=True)
            w = torch.where(see, torch.exp(s - torch.where(m == -math.inf, 0.0, m)), 0.0)
            l = w.sum(1, keepdim=True)
            w = torch.where(l > 0, w / l, 0.0)
            V = C * s_v[:, None]
            out[a:b, h] = w @ V
            lse[a:b, h] = torch.where(l > 0, m + l.log(), -math.inf)[:, 0]
            S = torch.where(see, x.abs() @ K.abs().T * d ** -0.5, 0.0).amax(1, keepdim=True)
            one = see.double()
            tol[a:b, h] = (2.0 ** -11 + 2.0 ** -17 * S + 2.0 ** -14) * (w @ V.abs()) + \
                2.0 ** -32 * (w * s_v).amax(1, keepdim=True) * (one @ C.abs()) + \
                2.0 ** -126 * (one @ V.abs())
            tol_l[a:b, h] = (2.0 ** -18 * S[:, 0] + 2.0 ** -20 * (1 + lse[a:b, h].abs())).nan_to_num()
    return out, lse, tol, tol_l


def compare(got, want, rows=None, columns=None):
    """The call's (out, lse) within the bounds of attend(), or that of bool masks `rows` of the
    queries and heads (and `columns` of the outputs)."""
    out, lse, tol, tol_l = want
    o, l = (x.double() for x in got)
    at = torch.ones_like(lse, dtype=torch.bool) if rows is None else rows
    full = at[..., None].expand(out.shape) if columns is None else at[..., None] & columns
    least, most = ((out + x).to(got[0].dtype).double() for x in (-tol, tol))
    assert torch.isfinite(o[full]).all()
    far = torch.maximum(least - o, o - most)[full]
    assert (far <= 0).all(), "out off by %g over its bound" % far.max().item()
    none = lse == -math.inf
    assert torch.equal(none[at], (l == -math.inf)[at])
    far = ((l - lse).abs() - tol_l)[~none & at]
    assert (far <= 0).all(), "lse off by %g over its bound" % far.max().item()


def check(p, **kw):
    got = call(p, **kw)
    hs.hs_get_device_error()
    compare(got, attend(p, **kw))
