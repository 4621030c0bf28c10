"""Oracle of the serving operators (include/keep_serve.h): rotary positions, 8-bit pages, attention of new tokens over
pages, sampling.  numpy, 64 bits, plain loops over sequences, heads and rows; written from the definitions."""
import math

import numpy as np


# ---- rotary positions ----
def rope_frequencies(rot_dim, theta, scaling="plain", factor=1.0, trained_len=1, fast=32.0, slow=1.0):
    freq, magnitude = [], 1.0
    for j in range(rot_dim // 2):
        base = theta
        if scaling == "base" and rot_dim > 2:
            base = theta * factor ** (rot_dim / (rot_dim - 2))
        f = 1.0 / base ** (2 * j / rot_dim)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            turns = trained_len / (2 * math.pi / f)
            share = min(1.0, max(0.0, (turns - slow) / (fast - slow)))      # of the unscaled frequency
            f = share * f + (1 - share) * f / factor
            magnitude = 0.1 * math.log(factor) + 1
        freq.append(f)
    return np.array(freq), magnitude


def rope(x, positions, freq, interleaved=False, magnitude=1.0):
    """x [rows, heads, head_dim]"""
    y = np.array(x, dtype=np.float64)
    h = len(freq)
    for r, p in enumerate(positions):
        for j, f in enumerate(freq):
            c, s = magnitude * math.cos(float(p) * f), magnitude * math.sin(float(p) * f)
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + h)
            x1, x2 = np.float64(x[r, :, a]), np.float64(x[r, :, b])
            y[r, :, a], y[r, :, b] = x1 * c - x2 * s, x2 * c + x1 * s
    return y


# ---- 8-bit pages ----
TOP = {"fp8": np.float32(448), "int8": np.float32(127)}
# the non-negative 8-bit floats of 4 exponent and 3 mantissa bits (the last pattern is NaN)
FP8 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])


def quantise(x, fmt):
    """rows of binary32 values -> (the code values, scales): one scale per row, both exactly as defined"""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(all="ignore"):
        amax = np.abs(x).max(-1)
        scale = np.maximum(amax * (np.float32(1) / TOP[fmt]), np.float32(2.0 ** -126))
        bad = ~np.isfinite(x).all(-1)
        u = np.clip(x / scale[..., None], -TOP[fmt], TOP[fmt])
    u[bad] = 0
    scale[bad] = np.nan
    if fmt == "int8":
        return np.rint(u).astype(np.float32), scale
    mag = np.abs(u).astype(np.float64)
    lo = np.clip(np.searchsorted(FP8, mag, side="right") - 1, 0, 126)
    hi = np.minimum(lo + 1, 126)
    d_lo, d_hi = mag - FP8[lo], FP8[hi] - mag
    up = (d_hi < d_lo) | ((d_hi == d_lo) & (lo % 2 == 1))                  # ties to the even pattern
    return np.copysign(FP8[np.where(up, hi, lo)], u).astype(np.float32), scale


def dequantise(codes, scale):
    return codes * scale[..., None]                                        # (one binary32 rounding)


# ---- attention over pages ----
def gather(pages, table_row, n):
    """pages [n_pages, heads, page_size, dh] (numbers) -> [n, heads, dh] of one sequence"""
    size = pages.shape[2]
    return np.stack([pages[min(max(int(table_row[t // size]), 0), len(pages) - 1), :, t % size] for t in range(n)]) \
        if n else np.zeros((0, pages.shape[1], pages.shape[3]))


def paged_attention(q, k_pages, v_pages, q_start, kv_len, table, window=0, scale=None):
    """q [rows, Hq, dh]; returns (out, lse, absum): absum = sum of probability * |value|, what errors are relative to.  Rows of
    no sequence are NaN."""
    rows, hq, dh = q.shape
    rep = hq // k_pages.shape[1]
    scale = dh ** -0.5 if scale is None else scale
    out, absum = np.full((2, rows, hq, dh), np.nan)
    lse = np.full((rows, hq), np.nan)
    for s in range(len(kv_len)):
        n = int(q_start[s + 1] - q_start[s])
        k, v = gather(k_pages, table[s], kv_len[s]), gather(v_pages, table[s], kv_len[s])
        for i in range(n):
            r, pos = q_start[s] + i, int(kv_len[s]) - n + i
            lo = max(0, pos - window + 1) if window else 0
            if pos < 0:
                out[r], absum[r], lse[r] = 0, 0, -np.inf
                continue
            for h in range(hq):
                x = (k[lo:pos + 1, h // rep] @ np.float64(q[r, h])) * scale
                p = np.exp(x - x.max())                # (a difference from lse would lose log(sum) beside scores of 2^50)
                lse[r, h] = x.max() + math.log(p.sum())
                p /= p.sum()
                out[r, h] = p @ v[lo:pos + 1, h // rep]
                absum[r, h] = p @ np.abs(v[lo:pos + 1, h // rep])
    return out, lse, absum


# ---- sampling ----
ONE = 2 ** 40


def weights(x, temperature):
    """whole numbers as Python ints, None where the row has no number above -infinity"""
    x = np.asarray(x, dtype=np.float64)
    real = x[~np.isnan(x)]
    if len(real) == 0 or real.max() == -np.inf:
        return None
    top = real.max()
    w = []
    for v in x:
        d = 0.0 if v == top else top - v
        w.append(0 if math.isnan(v) or d == math.inf else int(np.rint(math.exp(-(d / temperature)) * ONE)))
    return w


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, probability) of one row"""
    x = np.asarray(x, dtype=np.float64)
    greedy = not temperature > 0
    w = weights(x, 1.0 if greedy else temperature)
    if w is None:
        return -1, 0.0
    if greedy:
        return int(np.nanargmax(x)), 1.0
    least = max(1, math.ceil(min(min_p, 1.0) * ONE)) if min_p > 0 else 1
    rank = sorted((i for i in range(len(x)) if w[i] >= least), key=lambda i: (-x[i], i))
    if top_k >= 1:
        rank = rank[:top_k]
    if top_p < 1:
        goal = math.ceil(top_p * float(sum(w[i] for i in rank)))
        kept, mass = [], 0
        for i in rank:
            if mass >= max(goal, 1):
                break
            kept.append(i)
            mass += w[i]
        rank = kept
    total = sum(w[i] for i in rank)
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    goal = min(math.floor(u * float(total)), total - 1)
    for i in rank:
        if goal < w[i]:
            return i, w[i] / total
        goal -= w[i]
    raise AssertionError
