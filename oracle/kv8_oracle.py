"""fp64 oracle of the 8-bit key/value cache and of the scores read off a step's logits (numpy, loops and definitions; test infrastructure only).

A cache is a dict of numpy arrays in the library's layout: k [B, H, cap, D] and v [B, H, cap / 32, D, 32] uint8 codes, ks and vs [B, H, cap / 32] scales (float64).
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32
TOP = 448.0
FLOOR = 2.0 ** -100
NAN_CODE = 0x7f


def _values() -> np.ndarray:
    """The 256 e4m3 values by code: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities, 0x7f and 0xff are NaN."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.nan if e == 15 and m == 7 else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        out[c] = -x if c & 0x80 else x
    return out


VALUES = _values()


def encode(x: np.ndarray) -> np.ndarray:
    """Nearest code of each value (|x| <= 448 where finite), ties to the even code; what is not finite becomes the NaN code.  The sign of a zero is kept."""
    x = np.asarray(x, np.float64)
    mags = VALUES[:0x7f]                                        # ascending
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(mags, a), 0, 0x7e)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - mags[lo], mags[hi] - a
    c = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    c = np.where(hi == 0, 0, c)
    c = np.where(np.signbit(x), c | 0x80, c)
    return np.where(np.isfinite(x), c, NAN_CODE).astype(np.uint8)


def scale_of(x: np.ndarray) -> float:
    """The smallest power of two s >= FLOOR with 448 s >= the largest finite magnitude."""
    f = np.abs(x[np.isfinite(x)])
    top = float(f.max()) if f.size else 0.0
    s = FLOOR
    while s * TOP < top:
        s *= 2
    return s


def v_rows(v: np.ndarray) -> np.ndarray:
    """V codes [.., blocks, D, 32] as rows [.., cap, D]."""
    w = np.swapaxes(v, -1, -2)
    return w.reshape(*w.shape[:-3], -1, w.shape[-1])


def v_blocks(rows: np.ndarray) -> np.ndarray:
    w = rows.reshape(*rows.shape[:-2], -1, BLOCK, rows.shape[-1])
    return np.ascontiguousarray(np.swapaxes(w, -1, -2))


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """Values of codes [.., cap, D] with scales [.., cap / 32]."""
    return VALUES[codes] * np.repeat(scales, BLOCK, -1)[..., None]


def _write(codes, scales, rows, first):
    """codes [cap, D], scales [cap / 32], in place: rows [n, D] at `first`, block by block together with the committed rows of each block."""
    end = min(first + len(rows), len(codes))
    for j in range(first // BLOCK, -(-end // BLOCK)):
        r0, r1 = j * BLOCK, min(end, (j + 1) * BLOCK)
        at = max(r0, first)
        x = np.concatenate([VALUES[codes[r0:at]] * scales[j], rows[at - first:r1 - first]])
        scales[j] = scale_of(x)
        codes[r0:r1] = encode(x / scales[j])


def append(cache: dict, k_new, v_new, lens, counts) -> dict:
    """k_new, v_new [B, G, H, D].  Returns the cache after the call."""
    k, v, ks, vs = cache["k"].copy(), v_rows(cache["v"]).copy(), cache["ks"].copy(), cache["vs"].copy()
    for b in range(k.shape[0]):
        if counts[b]:
            for h in range(k.shape[1]):
                _write(k[b, h], ks[b, h], k_new[b, :counts[b], h], lens[b])
                _write(v[b, h], vs[b, h], v_new[b, :counts[b], h], lens[b])
    return {"k": k, "v": v_blocks(v), "ks": ks, "vs": vs}


def attend(cache: dict, q, lens, counts, acc_in=None):
    """q [B, G, Hq, D].  Returns (out [B, G, Hq, D], acc [B, H, cap] or None, spread [B, G, Hq, D] = sum_j p_j |v_j|, reach [B, G, Hq] = max_j |q| . |k_j|):
    rows of padding tokens are NaN in out.  spread and reach are what bounds of rounding errors are made of."""
    B, G, Hq, D = q.shape
    H, cap = cache["k"].shape[1], cache["k"].shape[2]
    group = Hq // H
    out, spread, reach = np.full(q.shape, np.nan), np.zeros(q.shape), np.zeros(q.shape[:3])
    acc = np.full((B, H, cap), np.nan)
    for b in range(B):
        n = min(lens[b] + counts[b], cap)
        for h in range(H):
            k = (VALUES[cache["k"][b, h]] * np.repeat(cache["ks"][b, h], BLOCK)[:, None])[:n]
            v = (VALUES[v_rows(cache["v"][b, h])] * np.repeat(cache["vs"][b, h], BLOCK)[:, None])[:n]
            w = np.zeros(n)
            for t in range(counts[b]):
                for hq in range(h * group, (h + 1) * group):
                    if n == 0:
                        out[b, t, hq] = 0
                        continue
                    s = k @ q[b, t, hq] / math.sqrt(D)
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[b, t, hq], spread[b, t, hq], reach[b, t, hq] = p @ v, p @ np.abs(v), (np.abs(k) @ np.abs(q[b, t, hq])).max()
                    w += p
            if acc_in is not None:
                acc[b, h, :n] = w
                m = min(lens[b], n)
                acc[b, h, :m] += acc_in[b, h, :m]
    return out, (acc if acc_in is not None else None), spread, reach


def evict(cache: dict, acc, lens, keep: int, recent: int, dst: dict, acc_dst):
    """Returns (dst cache, acc, lens, rows [B, H, keep]) after the call; what the call leaves alone is as in dst, acc_dst."""
    B, H = acc.shape[:2]
    k, v, ks, vs = dst["k"].copy(), v_rows(dst["v"]).copy(), dst["ks"].copy(), dst["vs"].copy()
    src_v = v_rows(cache["v"])
    out, rows = acc_dst.copy(), np.full((B, H, keep), -1, np.int32)
    for b in range(B):
        for h in range(H):
            n = int(lens[b])
            old = max(0, n - min(recent, keep)) if n > keep else 0
            score = [-math.inf if math.isnan(x) else float(x) for x in acc[b, h, :old]]
            nan = [math.isnan(x) for x in acc[b, h, :old]]
            first = sorted(range(old), key=lambda i: (nan[i], -score[i], i))[:keep - (n - old)] if n > keep else []
            kept = sorted(first) + list(range(old, n))
            rows[b, h, :len(kept)] = kept
            out[b, h, :len(kept)] = acc[b, h, kept]
            for j in range(-(-len(kept) // BLOCK)):
                r = np.array(kept[j * BLOCK:(j + 1) * BLOCK])
                for c, s, src, ss in ((k, ks, cache["k"], cache["ks"]), (v, vs, src_v, cache["vs"])):
                    x = VALUES[src[b, h, r]] * ss[b, h, r // BLOCK, None]
                    s[b, h, j] = scale_of(x)
                    c[b, h, j * BLOCK:j * BLOCK + len(r)] = encode(x / s[b, h, j])
    return {"k": k, "v": v_blocks(v), "ks": ks, "vs": vs}, out, np.minimum(lens, keep), rows


def token_scores(logits, tokens, exclude: int, top_k: int):
    """logits [rows, vocab] float64.  Returns (logprob, entropy, top_ids, top_logprobs)."""
    R, V = logits.shape
    lp, en = np.empty(R), np.empty(R)
    ids, tops = np.full((R, top_k), -1, np.int64), np.full((R, top_k), -math.inf)
    for r in range(R):
        x = logits[r].astype(np.float64).copy()
        if 0 <= exclude < V:
            x[exclude] = -math.inf
        ok = 0 <= tokens[r] < V and tokens[r] != exclude
        if np.isnan(x).any() or np.isposinf(x).any():
            lp[r] = en[r] = math.nan
            order = [v for v in sorted(range(V), key=lambda i: (-x[i] if not math.isnan(x[i]) else math.inf, i)) if x[v] > -math.inf][:top_k]
            ids[r, :len(order)] = order
            tops[r] = math.nan
            continue
        live = np.flatnonzero(x > -math.inf)
        if not live.size:
            lp[r], en[r] = -math.inf, 0.0
            continue
        m = x.max()
        q = (x - m) - math.log(np.exp(x[live] - m).sum())
        lp[r] = q[tokens[r]] if ok else -math.inf
        en[r] = -(np.exp(q[live]) * q[live]).sum()
        order = live[np.argsort(-x[live], kind="stable")][:top_k]
        ids[r, :len(order)], tops[r, :len(order)] = order, q[order]
    return lp, en, ids, tops
