"""Plain forms of the paged cache's operators in 64 bits, written from their
definitions with numpy, and the inputs of their tests."""
from __future__ import annotations

import math

import numpy as np
import torch

LARGEST = {"e4m3": 448.0, "int8": 127.0}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def e4m3_values() -> np.ndarray:
    """What each of the 256 e4m3 codes stands for."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    x[(b & 127) == 127] = np.nan
    return np.where(b & 128, -x, x)


def values(codes: np.ndarray, fmt: str) -> np.ndarray:
    """Stored bytes as the numbers they are."""
    return e4m3_values()[codes] if fmt == "e4m3" else codes.view(np.int8).astype(np.float64)


def rounded(x: np.ndarray, fmt: str) -> np.ndarray:
    """Numbers to stored bytes: to nearest even, saturating; NaN is NaN, or 0 in int8."""
    if fmt == "int8":
        y = np.nan_to_num(x, nan=0.0, posinf=1e9, neginf=-1e9)
        return np.rint(np.clip(y, -127, 127)).astype(np.int8).view(np.uint8)
    y = np.minimum(np.abs(x), 448.0)
    with np.errstate(invalid="ignore", divide="ignore"):
        step = np.exp2(np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3)
        y = np.rint(y / step) * step
    order = e4m3_values()[:127]
    code = np.searchsorted(order, np.nan_to_num(y)).astype(np.uint8)
    code = np.where(np.isnan(x), 127, code)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_of(m: float, fmt: str) -> float:
    """The least power of two s >= 2^-126 with m <= LARGEST * s."""
    e = -126
    if m > LARGEST[fmt] * 2.0 ** -126:
        e = math.frexp(m / LARGEST[fmt])[1] - 1
        while m > LARGEST[fmt] * 2.0 ** e:
            e += 1
    return 2.0 ** e


def append(x, slots, codes, scale, fmt):
    """x float64 [T, H, d] into codes uint8 [n, H, bt, d], scale float64 [n, H], in place."""
    bt = codes.shape[2]
    a = 0
    while a < len(slots):
        if slots[a] < 0:
            a += 1
            continue
        b = a + 1
        while b < len(slots) and slots[b] == slots[b - 1] + 1 and slots[b] // bt == slots[a] // bt:
            b += 1
        block, o = int(slots[a]) // bt, int(slots[a]) % bt
        for h in range(codes.shape[1]):
            y = x[a:b, h]
            fin = np.abs(y[np.isfinite(y)])
            s = scale_of(fin.max() if fin.size else 0.0, fmt)
            if o > 0:
                old = scale[block, h]
                s = max(s, old)
                if s > old:
                    codes[block, h, :o] = rounded(values(codes[block, h, :o], fmt) * (old / s), fmt)
            scale[block, h] = s
            codes[block, h, o:o + b - a] = rounded(y / s, fmt)
        a = b


def tables(have, fresh, table, pool, cursor, bt, max_tokens):
    """(table, slots, starts, lens, cursor) of valid inputs, request by request."""
    table = table.copy()
    taken, given = int(cursor[0]), int(cursor[1])
    slots, starts, lens = [], [0], []
    for r in range(len(have)):
        for p in range(have[r], have[r] + fresh[r]):
            b = p // bt
            if b >= -(-have[r] // bt) and p % bt == 0 or (b >= -(-have[r] // bt) and p == have[r]):
                table[r, b] = pool[taken % len(pool)]
                taken += 1
            slots.append(table[r, b] * bt + p % bt)
        starts.append(len(slots))
        lens.append(have[r] + fresh[r])
    assert taken <= given
    slots += [-1] * (max_tokens - len(slots))
    return (table, np.array(slots, np.int64), np.array(starts), np.array(lens, np.int64),
            np.array([taken, given]))


def to_bytes(t: torch.Tensor) -> np.ndarray:
    return t.view(torch.uint8).cpu().numpy()


def attend(q, k, v, ks, vs, fmt, table, lens, starts, scale, causal, window):
    """(out, lse, tol_out, tol_lse) in float64 on q's device, one request after the other.

    The tolerances bound what the arithmetic of 16-bit products with fp32 sums
    may differ by.  With a = sum_j p_j |v_j| (p normalised) and S the largest
    scale * sum_t |q_t k_jt| of a row:
      scores: fp32 sums of up to 256 products, q to 2^-24 of its row's largest
              -> 2^-18 S; the same for lse, with 2^-20 of itself for exp and log
      weights: rounded to half, 2^-11 each, and what is below 2^-31 of the
              largest is dropped -> (2^-11 + 2 * 2^-18 S) a + L 2^-31 max|v|,
              and 2^-14 a for block scales, sums and the division
    (the output's own rounding is the caller's to add)."""
    dev = q.device
    T, Hq, d = q.shape
    H = k.shape[1]
    G = Hq // H
    lut = torch.from_numpy(e4m3_values()).to(dev)

    def val(c, s, ids):
        x = lut[c.view(torch.uint8)[ids].long()] if fmt == "e4m3" else c[ids].double()
        return (x * s[ids].double()[..., None, None]).transpose(0, 1).reshape(H, -1, d)

    out = torch.zeros((T, Hq, d), dtype=torch.float64, device=dev)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=dev)
    tol, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    bt = k.shape[2]
    for r, L in enumerate(lens):
        a, b = starts[r], starts[r + 1]
        n = b - a
        if n == 0 or L == 0:
            continue
        ids = table[r, :-(-L // bt)].long()
        K, V = val(k, ks, ids)[:, :L], val(v, vs, ids)[:, :L]
        i = torch.arange(n, device=dev)[:, None] + (L - n)
        j = torch.arange(L, device=dev)[None]
        see = torch.ones((n, L), dtype=torch.bool, device=dev)
        if causal:
            see &= j <= i
        if window:
            see &= j > i - window
        for h in range(Hq):
            x = q[a:b, h].double()
            s = (x @ K[h // G].T * scale).masked_fill(~see, -math.inf)
            m = s.amax(1, keepdim=True)
            p = torch.where(see, torch.exp(s - torch.where(m == -math.inf, 0.0, m)), 0.0)
            l = p.sum(1, keepdim=True)
            p = torch.where(l > 0, p / l, 0.0)
            vh = torch.where(see.any(0)[:, None], V[h // G], 0.0)
            out[a:b, h] = p @ vh
            lse[a:b, h] = torch.where(l > 0, m + l.log(), -math.inf)[:, 0]
            S = torch.where(see, x.abs() @ K[h // G].abs().T * abs(scale), 0.0).amax(1, keepdim=True)
            A = p @ vh.abs()
            tol[a:b, h] = (2.0 ** -11 + 2.0 ** -17 * S + 2.0 ** -14) * A + \
                L * 2.0 ** -31 * vh.abs().amax()
            tol_l[a:b, h] = (2.0 ** -18 * S[:, 0] + 2.0 ** -20 * (1 + lse[a:b, h].abs())).nan_to_num()
    return out, lse, tol, tol_l
