"""Paged-cache operators in 64 bits, by their definitions (numpy)."""
from __future__ import annotations

import numpy as np

import parity

FLT_MAX = 3.4028234663852886e38


def scale_of(a) -> np.ndarray:
    """2^e, e the smallest whole number >= -126 with a <= 127 * 2^e."""
    a = np.asarray(a, dtype=np.float64)
    m, x = np.frexp(a)                        # a = m 2^x, 0.5 <= m < 1
    e = np.where(a > 0, np.where(m <= 127.0 / 128.0, x - 7, x - 6), -126)
    return np.ldexp(1.0, np.maximum(e, -126))


def bounds(codes, scales, keys, table, start, first, page):
    """The boxes (int64 codes [pages, heads, 2, d], float64 scales) after the new keys, row by row groups."""
    codes, scales = codes.astype(np.int64), scales.astype(np.float64)
    pages, heads, _, d = codes.shape
    for s in range(len(start)):
        by_col = {}
        for i in range(max(int(first[s]), 0), min(int(first[s + 1]), len(keys))):
            pos = int(start[s]) + i - int(first[s])
            if 0 <= pos < table.shape[1] * page:
                by_col.setdefault(pos // page, []).append((pos % page, i))
        for col, rows in by_col.items():
            p = int(table[s, col])
            if not 0 <= p < pages:
                continue
            x = keys[[i for _, i in rows]]    # [rows, heads, d]
            fresh = any(o == 0 for o, _ in rows)
            for h in range(heads):
                v = x[:, h]
                if not np.isfinite(v).all() or (not fresh and np.isinf(scales[p, h])):
                    codes[p, h, 0], codes[p, h, 1], scales[p, h] = -127, 127, np.inf
                    continue
                new = scale_of(np.abs(v).max())
                lo, hi = np.full(d, np.inf), np.full(d, -np.inf)
                if not fresh:
                    old = scales[p, h] if scales[p, h] > 0 else 2.0**-126
                    new = max(new, old)
                    lo, hi = np.floor(codes[p, h, 0] * (old / new)), np.ceil(codes[p, h, 1] * (old / new))
                codes[p, h, 0] = np.minimum(lo, np.floor(v.min(axis=0) / new))
                codes[p, h, 1] = np.maximum(hi, np.ceil(v.max(axis=0) / new))
                scales[p, h] = new
    return codes, scales


def select(q, codes, scales, table, lengths, page, budget, keep_first=1, keep_last=1):
    """(selected, counts) for q [seqs, heads * group, d] float64."""
    pages, heads, _, d = codes.shape
    seqs = len(lengths)
    group = q.shape[1] // heads
    out = np.full((seqs, heads, budget), -1, dtype=np.int32)
    counts = np.zeros((seqs, heads), dtype=np.int32)
    q = np.where(np.isfinite(q), q, 0.0)
    for s in range(seqs):
        n = -(-min(max(int(lengths[s]), 0), table.shape[1] * page) // page)
        take = min(n, budget)
        counts[s] = take
        if take == 0:
            continue
        col = table[s, :n].astype(np.int64)
        ok = (col >= 0) & (col < pages)
        at = np.where(ok, col, 0)
        for h in range(heads):
            best = np.full(n, -np.inf)
            for a in range(group):
                x = q[s, h * group + a]
                st = scale_of(np.abs(x).max())
                c = np.rint(x / st)
                lo, hi = codes[at, h, 0].astype(np.float64), codes[at, h, 1].astype(np.float64)
                dot = np.maximum(c * lo, c * hi).sum(axis=1)
                with np.errstate(invalid="ignore"):
                    sc = np.clip(dot * st * scales[at, h], -FLT_MAX, FLT_MAX)
                best = np.maximum(best, np.where(np.isinf(scales[at, h]), FLT_MAX, sc))
            best = np.where(ok, best, -np.inf)
            order = sorted(range(n), key=lambda j: (not (j < keep_first or j >= n - keep_last), -best[j], j)) if n > budget else range(n)
            out[s, h, :take] = np.sort(list(order)[:take])
    return out, counts


def pool_rows(orc, cache):
    """The rows [slots, d] (float64) that a pool's records stand for, by the oracle."""
    cfg = cache.cfg
    k, c, hdr = parity.gpu_codes(orc, cache, cache.capacity)
    if hdr is None:
        hdr = np.zeros((cache.capacity, 2), dtype=np.float32)
    return orc.decode(k, c, hdr, parity.signs_pm1(cfg.signs, cfg.d), cfg.n_angle, cfg.norm_bits, cfg.norm_mode)


def tokens_of(s, h, table, lengths, page, pages, selected=None, counts=None):
    """(position, page) of the tokens that (sequence s, head h) attends to."""
    n = min(max(int(lengths[s]), 0), table.shape[1] * page)
    cols = range(-(-n // page)) if selected is None else selected[s, h, : min(max(int(counts[s, h]), 0), selected.shape[2])]
    got = []
    for c in cols:
        if 0 <= c < table.shape[1] and 0 <= table[s, c] < pages:
            got += [(t, int(table[s, c])) for t in range(int(c) * page, min((int(c) + 1) * page, n))]
    return got


def attend(orc, q, krows, vrows, table, lengths, page, heads, scale, selected=None, counts=None):
    """(out [seqs, heads * group, d], tolerances' ingredients: max ||k^||, max ||v^|| of each row) in 64 bits."""
    seqs, qh, d = q.shape
    group, pages = qh // heads, len(krows) // (heads * page)
    out = np.zeros((seqs, qh, d))
    kmax, vmax, vel = np.zeros((seqs, qh)), np.zeros((seqs, qh)), np.zeros((seqs, qh))
    for s in range(seqs):
        for h in range(heads):
            tok = tokens_of(s, h, table, lengths, page, pages, selected, counts)
            if not tok:
                continue
            slot = np.array([(p * heads + h) * page + t % page for t, p in tok])
            k, v = krows[slot], vrows[slot]
            r = slice(h * group, (h + 1) * group)
            out[s, r] = orc.attend(np.ascontiguousarray(q[s, r]), np.ascontiguousarray(k), np.ascontiguousarray(v), scale)
            kmax[s, r] = np.linalg.norm(k, axis=1).max()
            vmax[s, r] = np.linalg.norm(v, axis=1).max()
            vel[s, r] = np.abs(v).max()
    return out, kmax, vmax, vel
