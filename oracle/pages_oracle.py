"""fp64 oracle of decoding from 8-bit pages: rotary positions with several axes, rows into pages, attention over pages, pages
onto pages.  numpy only; written from the definitions in include/ifkv.h's terms, page by page and row by row.

A pool is a dict of arrays: k uint8 [P, H, 64, d], v uint8 [P, H, d, 64], k_scale and v_scale float64 [P, H]; bytes are e4m3.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 64
NAN_BYTE = 0x7F


def _decode_table() -> np.ndarray:
    out = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = math.nan if (b & 0x7F) == 0x7F else m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[b] = -v if b & 0x80 else v
    return out


E4M3 = _decode_table()


def to_e4m3(x) -> np.ndarray:
    """Bytes of the nearest e4m3 numbers, ties to the even one; |x| <= 448 or not finite (then NaN)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    bad = ~np.isfinite(x)
    a = np.where(bad, 0.0, a)
    assert a.size == 0 or a.max() <= 448.0
    grid = E4M3[:0x7F]                                   # 0 .. 448, ascending; the byte's last bit says odd or even
    hi = np.clip(np.searchsorted(grid, a), 0, 0x7E)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    byte = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    byte = np.where(grid[hi] == a, hi, byte)
    return np.where(bad, NAN_BYTE, byte | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def value_byte(t: int) -> int:
    """Where token t of a page lies in a value row: bits 3:2 of t, then bit 5, bit 4, bits 1:0."""
    return (t >> 2 & 3) * 16 + (t >> 5) * 8 + (t >> 4 & 1) * 4 + (t & 3)


ORDER = np.array([value_byte(t) for t in range(PAGE)])


def scale_for(x) -> float:
    """2^e with the smallest e >= -100 for which no finite |x| exceeds 448 * 2^e."""
    a = np.abs(np.asarray(x, dtype=np.float64))
    a = a[np.isfinite(a)]
    top = float(a.max()) if a.size else 0.0
    e = -100
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def rope_rows_axes(x: np.ndarray, pos: np.ndarray, axes, inv_freq, pairing: str = "half") -> np.ndarray:
    x, d = np.array(x, dtype=np.float64), x.shape[-1]
    for j in range(d // 2):
        ang = pos[:, axes[j]].astype(np.float64) * inv_freq[j]
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
        i0, i1 = (j, j + d // 2) if pairing == "half" else (2 * j, 2 * j + 1)
        a, b = x[..., i0].copy(), x[..., i1].copy()
        x[..., i0], x[..., i1] = a * c - b * s, a * s + b * c
    return x


def rows_of(row_start, s, n_rows):
    return (s, s + 1) if row_start is None else (int(row_start[s]), int(row_start[s + 1]))


def store_pages(pool: dict, table, kv_len, row_pos, k_new, v_new, row_start=None) -> dict:
    pool = {name: a.copy() for name, a in pool.items()}
    n_pages, heads = pool["k"].shape[:2]
    for s in range(len(table)):
        lo, hi = rows_of(row_start, s, len(row_pos))
        by_page = {}
        for r in range(lo, hi):
            if 0 <= row_pos[r] < PAGE * table.shape[1] and 0 <= table[s][row_pos[r] // PAGE] < n_pages:
                by_page.setdefault(int(row_pos[r]) // PAGE, []).append(r)
        for logical, rows in by_page.items():
            page, slots = int(table[s][logical]), [int(row_pos[r]) % PAGE for r in rows]
            kept = [t for t in range(PAGE) if logical * PAGE + t < kv_len[s] and t not in slots]
            for h in range(heads):
                for name, new in (("k", k_new), ("v", v_new)):
                    x = np.stack([new[r, h] for r in rows]).astype(np.float64)
                    old, scale = float(pool[name + "_scale"][page, h]), scale_for(x)
                    tile = pool[name][page, h] if name == "k" else pool[name][page, h].T[ORDER]   # [token, d]
                    if kept:
                        scale = max(scale, old)
                        if scale != old:
                            tile = to_e4m3(E4M3[tile] * (old / scale))
                        tile = tile.copy()
                    else:
                        tile = np.zeros_like(tile)
                    tile[slots] = to_e4m3(x / scale)
                    if name == "k":
                        pool[name][page, h] = tile
                    else:
                        back = np.empty_like(tile)
                        back[ORDER] = tile
                        pool[name][page, h] = back.T
                    pool[name + "_scale"][page, h] = scale
    return pool


def tokens(pool: dict, table_row, n: int, h: int):
    """Which of the first n tokens a sequence's pages hold, their keys and their values (kv head h)."""
    n_pages = pool["k"].shape[0]
    k, v, there = [], [], []
    for logical in range(-(-n // PAGE)):
        page, take = int(table_row[logical]), min(PAGE, n - logical * PAGE)
        if not 0 <= page < n_pages:
            there += [False] * take
            continue
        there += [True] * take
        k.append(E4M3[pool["k"][page, h]][:take] * pool["k_scale"][page, h])
        v.append(E4M3[pool["v"][page, h].T[ORDER]][:take] * pool["v_scale"][page, h])
    d = pool["k"].shape[3]
    return np.array(there, dtype=bool), np.concatenate(k + [np.zeros((0, d))]), np.concatenate(v + [np.zeros((0, d))])


def attend_pages(q, row_pos, pool: dict, table, sm_scale: float, row_start=None):
    """(out, lse, mass, size): mass = sum_j w_j |v_j|, size = max_j sum_c |q_c k_jc| * sm_scale (for error bounds); rows that belong
    to no sequence are NaN in all."""
    n, hq, d = q.shape
    hkv = pool["k"].shape[1]
    grp = hq // hkv
    out, mass = np.full((n, hq, d), np.nan), np.full((n, hq, d), np.nan)
    lse, size = np.full((n, hq), np.nan), np.full((n, hq), np.nan)
    for s in range(len(table)):
        lo, hi = rows_of(row_start, s, n)
        for h in range(hkv):
            inside = [int(p) for p in row_pos[lo:hi] if 0 <= p < PAGE * table.shape[1]]
            there, k, v = tokens(pool, table[s], max(inside, default=-1) + 1, h)
            at = np.flatnonzero(there)
            for r in range(lo, hi):
                p, cols = int(row_pos[r]), slice(h * grp, (h + 1) * grp)
                seen = int(np.searchsorted(at, p, side="right")) if 0 <= p < PAGE * table.shape[1] else 0
                if seen == 0:
                    out[r, cols], mass[r, cols], lse[r, cols], size[r, cols] = 0.0, 0.0, -np.inf, 0.0
                    continue
                qr = q[r, cols].astype(np.float64)
                logits = qr @ k[:seen].T * sm_scale
                top = logits.max(axis=1, keepdims=True)
                w = np.exp(logits - top)
                z = w.sum(axis=1, keepdims=True)
                out[r, cols], mass[r, cols] = w / z @ v[:seen], w / z @ np.abs(v[:seen])
                lse[r, cols] = (top + np.log(z))[:, 0]
                size[r, cols] = (np.abs(qr) @ np.abs(k[:seen]).T).max(axis=1) * abs(sm_scale)
    return out, lse, mass, size


def copy_pages(pool: dict, src, dst) -> dict:
    new = {name: a.copy() for name, a in pool.items()}
    for a, b in zip(src, dst):
        for name in new:
            new[name][b] = pool[name][a]
    return new
