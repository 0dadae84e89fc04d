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
