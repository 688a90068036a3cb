"""Plain 64-bit forms of answering from a compacted cache, and inputs for its tests: appending to a paged cache with the
position rotation, and attention over shared prefixes and paged tails.  numpy only; nothing here comes from the package."""
from __future__ import annotations

import math

import numpy as np

EPS = {"f32": 2.0 ** -23, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}         # spacing at one; a rounding is off by half of it
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}     # smallest subnormal


def rotate(x, positions, inv_freq, interleaved):
    """x (..., 128) float64 turned by positions (...) times inv_freq (rot / 2)."""
    rot = 2 * len(inv_freq)
    a = np.asarray(positions, np.float64)[..., None] * np.asarray(inv_freq, np.float64)
    u, v = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y = x.copy()
    y[..., u] = x[..., u] * np.cos(a) - x[..., v] * np.sin(a)
    y[..., v] = x[..., v] * np.cos(a) + x[..., u] * np.sin(a)
    return y


def append(q, k, v, new_lens, past_lens, pos_base, inv_freq, interleaved, K_pages, V_pages, table, q_out):
    """Token by token.  Returns q_out, K_pages, V_pages (float64, changed copies), kv_lens and, shaped like them, how much a pair
    may be off in units of its own length (zero where values are only copied)."""
    q_out, Kp, Vp = q_out.copy(), K_pages.copy(), V_pages.copy()
    eq, ek = np.zeros_like(q_out), np.zeros_like(Kp)
    n_pages, _, page, _ = Kp.shape
    cap = table.shape[1] * page
    kv = np.zeros(len(new_lens), np.int64)
    half = len(inv_freq)

    def length(x):                                            # of the pair that a dimension belongs to
        r = np.zeros_like(x)
        if half:
            rot = 2 * half
            i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
            r[..., i] = r[..., j] = np.hypot(x[..., i], x[..., j])
        return r

    for b, n in enumerate(new_lens):
        n = min(max(int(n), 0), k.shape[1])
        past = min(max(int(past_lens[b]), 0), cap)
        kv[b] = min(past + n, cap)
        for t in range(n):
            slot = past + t
            x = int(pos_base[b]) + slot
            if q is not None:
                q_out[b, t] = rotate(q[b, t], np.full(q.shape[2], x), inv_freq, interleaved)
                eq[b, t] = length(q[b, t])
            if slot >= cap:
                continue
            p = int(table[b, slot // page])
            if 0 <= p < n_pages:
                Kp[p, :, slot % page] = rotate(k[b, t], np.full(k.shape[2], x), inv_freq, interleaved)
                ek[p, :, slot % page] = length(k[b, t])
                Vp[p, :, slot % page] = v[b, t]
    return q_out, Kp, Vp, kv, eq, ek


def prompt_of(b, B, P, row_start):
    if P == 0:
        return -1
    if row_start is None:
        return b // (B // P)
    for p in range(P):
        if row_start[p] <= b < row_start[p + 1]:
            return p
    return -1


def attention(q, G, new_lens, prefix=None, pages=None):
    """q (B, T, H*G, 128) float64; prefix = dict(K, V, lens, row_start), pages = dict(K, V, table, kv_lens).  Only keys that a query
    sees are touched.  Returns out, lse (NaN where there is no token) and the bounds of tolerance()."""
    B, T, HG, d = q.shape
    H = HG // G
    out, lse = np.full(q.shape, np.nan), np.full(q.shape[:3], np.nan)
    spread, worst, small = np.zeros(q.shape), np.zeros(q.shape[:3]), np.zeros(q.shape)
    for b in range(B):
        n = T if new_lens is None else min(max(int(new_lens[b]), 0), T)
        p = -1 if prefix is None else prompt_of(b, B, prefix["K"].shape[0], prefix["row_start"])
        slots, where = [], []
        if pages is not None:
            n_pages, _, page, _ = pages["K"].shape
            kv = min(max(int(pages["kv_lens"][b]), 0), pages["table"].shape[1] * page)
            for j in range(kv):
                g = int(pages["table"][b, j // page])
                if 0 <= g < n_pages:
                    slots.append(j)
                    where.append((g, j % page))
            slots = np.array(slots, np.int64)
            gi, gj = (np.array([w[i] for w in where], np.int64) for i in (0, 1))
        for h in range(H):
            L = 0
            if p >= 0:
                cap = prefix["K"].shape[2]
                L = cap if prefix["lens"] is None else min(max(int(prefix["lens"][p, h]), 0), cap)
            for t in range(n):
                K = prefix["K"][p, h, :L] if p >= 0 else np.zeros((0, d))
                V = prefix["V"][p, h, :L] if p >= 0 else np.zeros((0, d))
                if pages is not None:
                    see = slots <= kv - n + t
                    K = np.concatenate([K, pages["K"][gi[see], h, gj[see]]])
                    V = np.concatenate([V, pages["V"][gi[see], h, gj[see]]])
                for g in range(G):
                    x = q[b, t, h * G + g]
                    if len(K) == 0:
                        out[b, t, h * G + g], lse[b, t, h * G + g] = 0.0, -np.inf
                        continue
                    s = K @ x / math.sqrt(d)
                    top = s.max()
                    w = np.exp(s - top)
                    total = w.sum()
                    out[b, t, h * G + g] = w @ V / total
                    lse[b, t, h * G + g] = top + math.log(total)
                    spread[b, t, h * G + g] = w @ np.abs(V) / total
                    small[b, t, h * G + g] = np.abs(V).sum(axis=0) / total
                    # fp32 sums of 128 products: 128 half steps of the sum of the products' sizes; as many half steps as keys for
                    # the sums of weights and weighted values; eight for exponentials, scales and the division
                    worst[b, t, h * G + g] = (128 * (np.abs(K) @ np.abs(x)).max() / math.sqrt(d) + len(K) + 8) * 2.0 ** -24
    return out, lse, (spread, worst, small)


def tolerance(dtype, out, lse, bounds):
    """How far out and lse may be off.  Weights are rounded to dtype (half a step each, so half a step of the weighted sizes;
    below the normal range half of the smallest step each), the result once more; scores are off by `worst`, twice for
    weight and sum."""
    spread, worst, small = bounds
    half = EPS[dtype] / 2
    weights = half if dtype != "f32" else 0.0
    o = (weights + 2 * worst)[..., None] * spread + (TINY[dtype] / 2 * small if dtype == "f16" else 0.0)
    o = o * (1 + EPS[dtype]) + half * np.abs(out) + TINY[dtype]
    return o, worst + 2.0 ** -22 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0.0)))


def scattered_pages(rng, B, kv_lens, page, extra=2):
    """A page table over a pool in random order; entries behind a row's last page are -1.  Returns (table, n_pages)."""
    used = [-(-int(n) // page) for n in kv_lens]
    order = rng.permutation(sum(used) + extra)
    table = np.full((B, max(used + [0]) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(used) + extra
