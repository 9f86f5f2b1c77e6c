"""CPU oracle of the 8-bit key / value cache, its attention and eviction, and of rotary positions with several axes:
numpy float64 from the definitions in include/vvs.h, plain loops over sequences, heads and rows.  Nothing here is
shared with the CUDA path.

No counterpart in the paper: there is nothing to be unpinned against.  Pins: tests/test_oracle_quant_cache.py."""
from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0


def e4m3_decode(codes: np.ndarray) -> np.ndarray:
    """uint8 codes -> float64: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    c = codes.astype(np.int64)
    exp, man = (c >> 3) & 15, c & 7
    mag = np.where(exp == 0, man * 2.0 ** -9, (8 + man) * 2.0 ** (exp - 10.0))
    mag = np.where((c & 127) == 127, np.nan, mag)
    return np.where(c & 128, -mag, mag)


_POSITIVE = e4m3_decode(np.arange(127, dtype=np.uint8))          # 0 .. 448, ascending


def e4m3_encode(x: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one, magnitudes beyond 448 to 448, NaN to 0."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.where(np.isnan(x), 0.0, np.minimum(np.abs(x), E4M3_MAX))
    hi = np.clip(np.searchsorted(_POSITIVE, mag, side="left"), 1, 126)
    lo = hi - 1
    to_lo, to_hi = mag - _POSITIVE[lo], _POSITIVE[hi] - mag
    code = np.where(to_lo < to_hi, lo, np.where(to_lo > to_hi, hi, np.where(lo % 2 == 0, lo, hi)))
    negative = np.signbit(x) & ~np.isnan(x)
    return (code + np.where(negative, 128, 0)).astype(np.uint8)


def block_scale(amax: float) -> float:
    """The smallest power of two, 2^-60 at least, by which amax is at most 448."""
    s = 2.0 ** -60
    while amax > E4M3_MAX * s:
        s *= 2.0
    return s


def rotate_axes(x: np.ndarray, inv_freq, axis, pos, halves: bool) -> np.ndarray:
    """x [B, T, H, hd], pos [axes, B, T]; the angle is a float32 number, everything else float64."""
    out = np.array(x, dtype=np.float64)
    n = len(inv_freq)
    for i in range(n):
        angle = (pos[axis[i]].astype(np.float32) * np.float32(inv_freq[i])).astype(np.float64)       # [B, T]
        c, s = np.cos(angle)[..., None], np.sin(angle)[..., None]
        e0, e1 = (i, i + n) if halves else (2 * i, 2 * i + 1)
        x0, x1 = np.array(x[..., e0], dtype=np.float64), np.array(x[..., e1], dtype=np.float64)
        out[..., e0], out[..., e1] = x0 * c - x1 * s, x1 * c + x0 * s
    return out


def append_rows(codes, scales, x, base: int, block: int) -> None:
    """One head of one sequence: x [rows, hd] goes to slots base .. of codes [cap, hd], scales [cap / block], in place."""
    x = np.asarray(x, dtype=np.float64)
    end = base + x.shape[0]
    for b in range(base // block, -(-end // block) if x.shape[0] else 0):
        lo, hi = max(base, b * block), min(end, (b + 1) * block)
        rows = x[lo - base:hi - base]
        fine = np.abs(rows[np.isfinite(rows)])
        now = block_scale(fine.max() if fine.size else 0.0)
        if b * block < base:
            was = float(scales[b])
            now = max(now, was)
            if now > was:
                codes[b * block:base] = e4m3_encode(e4m3_decode(codes[b * block:base]) * (was / now))
        codes[lo:hi] = e4m3_encode(rows / now)
        scales[b] = now


def attend(k_codes, v_codes, k_scale, v_scale, q, cache_len, block: int, scale=None, row_count=None, first_slot=None, visible=None,
           mass=None, mass_rows: int = 0, mass_decay: float = 1.0):
    """codes [B, Hkv, cap, hd], q [B, T, H, hd] -> out, lse, mass, and the sum of p |v| of each output element."""
    b_n, t_n, heads, hd = q.shape
    kv_heads = k_codes.shape[1]
    share = heads // kv_heads
    scale = 1.0 / np.sqrt(hd) if scale is None else scale
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full((b_n, t_n, heads), -np.inf)
    mass = None if mass is None else np.array(mass, dtype=np.float64)
    for b in range(b_n):
        length = int(cache_len[b])
        n = t_n if row_count is None else int(row_count[b])
        first = 0 if first_slot is None else int(first_slot[b])
        end = length + n
        for h in range(kv_heads):
            each = np.arange(end) // block
            k = e4m3_decode(k_codes[b, h, :end]) * k_scale[b, h][each][:, None]
            v = e4m3_decode(v_codes[b, h, :end]) * v_scale[b, h][each][:, None]
            got = np.zeros(end)
            for t in range(n):
                seen = [j for j in range(first, length)]
                if visible is None:
                    seen += [length + j for j in range(t + 1)]
                else:
                    seen += [length + j for j in range(n) if int(visible[b, t]) >> j & 1]
                if not seen:
                    continue
                for g in range(h * share, (h + 1) * share):
                    s = scale * (k[seen] @ np.asarray(q[b, t, g], dtype=np.float64))
                    top = s.max()
                    w = np.exp(s - top)
                    p = w / w.sum()
                    out[b, t, g] = p @ v[seen]
                    spread[b, t, g] = p @ np.abs(v[seen])
                    lse[b, t, g] = top + np.log(w.sum())
                    if t < mass_rows:
                        got[seen] += p
            if mass_rows:
                mass[b, h, :end] = (0.0 if mass_decay == 0 else mass_decay * mass[b, h, :end]) + got
    return out, lse, mass, spread


def evict(k_codes, v_codes, k_scale, v_scale, mass, age, cache_len, next_age, keep: int, n_sink: int, n_recent: int, block: int):
    """Everything [B, H, ...]; codes and scales in place.  Returns kept [B, H, keep], new mass, new age, new_len; slots from
    new_len on are 0 and -1."""
    b_n, heads, cap = mass.shape
    kept = np.full((b_n, heads, keep), -1, dtype=np.int32)
    mass_out, age_out = np.zeros_like(mass), np.full_like(age, -1)
    new_len = np.minimum(cache_len, keep).astype(np.int32)
    for b in range(b_n):
        length = int(cache_len[b])
        for h in range(heads):
            m, a = mass[b, h, :length], age[b, h, :length]

            def worth(j):
                guarded = a[j] < n_sink or a[j] >= next_age[b] - n_recent
                return (0 if guarded else 1, 0.0 if guarded else (np.inf if np.isnan(m[j]) else -float(m[j])),
                        1 if not guarded and np.isnan(m[j]) else 0, j)

            stays = set(sorted(range(length), key=worth)[:keep])
            source = np.arange(min(length, keep))
            movers = iter(sorted(j for j in stays if j >= keep))
            for d in range(len(source)):
                if d not in stays:
                    source[d] = next(movers)
            kept[b, h, :len(source)] = source
            mass_out[b, h, :len(source)] = m[source]
            age_out[b, h, :len(source)] = a[source]
            moved = [d for d in range(len(source)) if source[d] != d]
            for codes, scales in ((k_codes[b, h], k_scale[b, h]), (v_codes[b, h], v_scale[b, h])):
                was_codes, was = codes.copy(), scales.copy()
                for d in moved:
                    scales[d // block] = max(scales[d // block], was[source[d] // block])
                for n in {d // block for d in moved}:
                    if scales[n] > was[n]:
                        rows = slice(n * block, (n + 1) * block)
                        codes[rows] = e4m3_encode(e4m3_decode(was_codes[rows]) * (was[n] / scales[n]))
                for d in moved:
                    f = was[source[d] // block] / scales[d // block]
                    codes[d] = was_codes[source[d]] if f == 1.0 else e4m3_encode(e4m3_decode(was_codes[source[d]]) * f)
    return kept, mass_out, age_out, new_len
