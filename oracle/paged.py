"""Oracle of the paged K/V cache: writing rows, reading them back, attention over them (numpy float64, loops over rows).

A cache is a dict: k, v [pages, kv heads, slots, head_dim] float64 (the values that are held), table [batch, width] int,
lengths [batch] int. Rows are given per sequence by offsets; None: one row per sequence.
"""
import numpy as np


def e4m3_values():
    """Value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities, 0x7f and 0xff NaN."""
    out = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, c >> 3 & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = np.nan if c & 127 == 127 else -x if s else x
    return out


_CODES = e4m3_values()
_POSITIVE = _CODES[:127]


def round_e4m3(x):
    """Nearest e4m3 value of magnitudes up to 448, ties to the even code."""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    below, above = a - _POSITIVE[lo], _POSITIVE[hi] - a
    pick = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(np.isnan(x), np.nan, np.copysign(_POSITIVE[pick], x))


def quantise(x):
    """Rows [..., n] -> (values held, exponents of their scales)."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x)
    a = np.where(fine, np.abs(x), 0.0).max(-1, initial=0.0)
    # the smallest exponent that brings the row to at most 448
    e = -110 + np.searchsorted(448.0 * 2.0 ** np.arange(-110, 120, dtype=np.float64), a)
    scale = (2.0 ** e)[..., None]
    y = np.where(fine, x, 0.0) / scale
    y = np.where((e == 120)[..., None], np.clip(y, -240.0, 240.0), y)
    return np.where(fine, round_e4m3(y) * scale, np.nan), e


def e2m1_values():
    """Value of each of the 16 codes: sign, 2 exponent bits (bias 1), 1 mantissa bit; neither infinities nor NaN."""
    a = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    return np.concatenate([a, -a])


def round_e2m1(x):
    """Nearest e2m1 value of magnitudes up to 6, ties to the even code."""
    a, v = np.abs(x), e2m1_values()[:8]
    hi = np.clip(np.searchsorted(v, a), 1, 7)
    lo = hi - 1
    below, above = a - v[lo], v[hi] - a
    return np.copysign(v[np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))], x)


def quantise_e2m1(x):
    """Rows [..., n] -> (values held, exponents of their scales [..., n / 32]; 128: NaN)."""
    x = np.asarray(x, dtype=np.float64)
    y = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    fine = np.isfinite(y).all(-1)
    y = np.where(fine[..., None], y, 0.0)
    # the smallest exponent that brings the 32 to at most 6
    e = -110 + np.searchsorted(6.0 * 2.0 ** np.arange(-110, 126, dtype=np.float64), np.abs(y).max(-1))
    scale = (2.0 ** e)[..., None]
    most = np.where(e == 126, 3.0, 6.0)[..., None]
    held = np.where(fine[..., None], round_e2m1(np.clip(y / scale, -most, most)) * scale, np.nan)
    return held.reshape(x.shape), np.where(fine, e, 128)


def round_bf16(x):
    import torch
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


def hold(x, dtype):
    """Rows as a cache of this type holds them."""
    if dtype == "e2m1":
        return quantise_e2m1(x)[0]
    return quantise(x)[0] if dtype == "e4m3" else round_bf16(x) if dtype == "bf16" else np.asarray(x, np.float32).astype(np.float64)


def place(cache, b, p):
    """(page, slot) of a position, or None."""
    pages, _, slots, _ = cache["k"].shape
    if not 0 <= p < cache["table"].shape[1] * slots:
        return None
    page = int(cache["table"][b, p // slots])
    return (page, p % slots) if 0 <= page < pages else None


def rows_of(cache, off, rows):
    """(row, sequence) of the rows that belong to a sequence."""
    batch = cache["table"].shape[0]
    if off is None:
        return [(r, r) for r in range(batch)]
    return [(r, b) for b in range(batch) for r in range(off[b], min(off[b + 1], rows))]


def store(cache, k_new, v_new, positions, off, dtype):
    k, v = hold(k_new, dtype), hold(v_new, dtype)
    for r, b in rows_of(cache, off, len(positions)):
        at = place(cache, b, int(positions[r]))
        if at:
            cache["k"][at[0], :, at[1]], cache["v"][at[0], :, at[1]] = k[r], v[r]


def load(cache, positions, off, k_out, v_out):
    for r, b in rows_of(cache, off, len(positions)):
        at = place(cache, b, int(positions[r]))
        k_out[r] = cache["k"][at[0], :, at[1]] if at else 0.0
        v_out[r] = cache["v"][at[0], :, at[1]] if at else 0.0


def seen(cache, b):
    """Places of the positions that the rows of a sequence attend to."""
    n = min(int(cache["lengths"][b]), cache["table"].shape[1] * cache["k"].shape[2])
    return [at for at in (place(cache, b, p) for p in range(n)) if at]


def attn(cache, q, off):
    """(result, sum of p |v| / sum of p, largest sum of |q| |k| / sqrt(head_dim)) of every row and head; rows of no sequence: NaN."""
    R, Hq, dh = q.shape
    out, spread, most = np.full(q.shape, np.nan), np.full(q.shape, np.nan), 0.0
    group = Hq // cache["k"].shape[1]
    mine = {}
    for r, b in rows_of(cache, off, R):
        mine.setdefault(b, []).append(r)
    for b, r in mine.items():
        at = seen(cache, b)
        pages, slots = [a[0] for a in at], [a[1] for a in at]
        if not at:
            out[r] = spread[r] = 0.0
            continue
        K, V = cache["k"][pages, :, slots], cache["v"][pages, :, slots]          # [keys, kv heads, dh]
        for h in range(Hq):
            k, v = K[:, h // group], V[:, h // group]
            s = q[r, h] @ k.T / np.sqrt(dh)
            m = s.max(-1, keepdims=True)
            nothing = m == -np.inf
            p = np.where(nothing, 0.0, np.exp(s - np.where(nothing, 0.0, m)))
            total = p.sum(-1, keepdims=True)
            total = np.where(nothing, 1.0, total)
            out[r, h] = np.where(nothing, 0.0, p @ v / total)
            spread[r, h] = np.where(nothing, 0.0, p @ np.abs(v) / total)
            finite = np.abs(k).max(-1) < np.inf
            if finite.any():
                most = max(most, float((np.abs(q[r, h]) @ np.abs(k[finite]).T).max() / np.sqrt(dh)))
    return out, spread, most
