"""fp64 oracle for the operators around a paged key/value cache.  TEST INFRASTRUCTURE ONLY.

The paper caches the keys and values of accepted tokens and feeds position-encoded queries and keys to the attention of
Algorithm 2; it says nothing about how either is stored or made.  Written out row by row here:

  norm_rope   y = x / sqrt(mean(x^2) + eps) * w;  columns (u, v) of a pair turned by  pos * inv_freq[j]
  append      row j of a sequence goes to slot len + j: page table[b][slot // ps], row slot % ps; 8-bit pages carry an exponent
              per page and head, a byte q standing for decode(q) * 2^(e - 127)
  gather      the rows a sequence's table spells out, for oracle.tree_attention
"""
from __future__ import annotations

import math

import numpy as np

from oracle.tree_attention import tree_verify_attention


def turn(x, pos, inv_freq, interleaved):
    """x [..., D] at position pos."""
    y = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    for j in range(half):
        i0, i1 = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        c, s = math.cos(float(pos) * inv_freq[j]), math.sin(float(pos) * inv_freq[j])
        u, v = np.array(x[..., i0], dtype=np.float64), np.array(x[..., i1], dtype=np.float64)
        y[..., i0], y[..., i1] = u * c - v * s, u * s + v * c
    return y


def norm_rope(x, pos, inv_freq, weight=None, eps=1e-6, interleaved=False):
    """x [B,H,n,D] float64, pos [B,n]; returns the same shape."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * weight
    for b in range(x.shape[0]):
        for i in range(x.shape[2]):
            y[b, :, i] = turn(y[b, :, i], int(pos[b, i]), inv_freq, interleaved)
    return y


def needed_exponent(top):
    """Smallest byte e >= 1 with top <= 448 * 2^(e - 127)."""
    e = 1
    while top > 448.0 * 2.0 ** (e - 127):
        e += 1
    return e


def stored_rows(cache_len, count, table, ps, num_pages):
    """Rows that an append of `count` rows stores: up to the capacity and to the first page that is none."""
    cap = len(table) * ps
    L = min(max(int(cache_len), 0), cap)
    end = min(L + max(int(count), 0), cap)
    for p in range(L // ps, -(-end // ps) if end > L else L // ps):
        if not 0 <= table[p] < num_pages:
            end = max(L, p * ps)
            break
    return L, end - L


def append(pool, exps, K, table, cache_len, count, rows=None, inv_freq=None, interleaved=False, shift=0, decode=None):
    """One of K / V.  pool: float64 values [P,H,ps,D] (16-bit pages) or bytes (decode given, exps [P,H]); K [B,H,n,D] float64.
    Returns (want, exps): want float64 [P,H,ps,D], the exact value that every row written should be nearest to (8-bit: in
    units of the page's factor), NaN where nothing is written; exps the new exponents."""
    want = np.full(pool.shape, np.nan)
    new_exps = None if exps is None else exps.copy()
    P, H, ps, D = pool.shape
    lens = []
    for b in range(K.shape[0]):
        L, m = stored_rows(cache_len[b], min(max(int(count[b]), 0), K.shape[2]), table[b], ps, P)
        lens.append(L + m)
        for p in range(L // ps, -(-(L + m) // ps) if m else L // ps):
            page = table[b][p]
            lo, hi = max(L, p * ps), min(L + m, p * ps + ps)
            x = np.zeros((H, hi - lo, D))
            for r in range(lo, hi):
                i = r - L if rows is None else int(rows[b][r - L])
                if 0 <= i < K.shape[2]:
                    x[:, r - lo] = K[b, :, i] if inv_freq is None else turn(K[b, :, i], r + shift, inv_freq, interleaved)
            at = slice(lo - p * ps, hi - p * ps)
            if exps is None:
                want[page, :, at] = x
                continue
            for h in range(H):
                fin = np.abs(x[h])[np.isfinite(x[h])]
                e = needed_exponent(float(fin.max()) if fin.size else 0.0)
                if lo > p * ps:
                    e = max(e, int(exps[page, h]))
                    old = slice(0, lo - p * ps)
                    want[page, h, old] = decode(pool[page, h, old]) * 2.0 ** (int(exps[page, h]) - e)
                new_exps[page, h] = e
                want[page, h, at] = np.where(np.isinf(x[h]), np.sign(x[h]) * 448.0, x[h] / 2.0 ** (e - 127))
    return want, new_exps, np.array(lens, dtype=np.int32)


def gather(pool, exps, table, length, decode=None):
    """Rows 0 .. length - 1 of a sequence: (values [H, rows, D], which of them lie in pages)."""
    P, H, ps, D = pool.shape
    out, there = np.zeros((H, length, D)), np.zeros(length, dtype=bool)
    for r in range(length):
        page = int(table[r // ps])
        if not 0 <= page < P:
            continue
        there[r] = True
        row = pool[page, :, r % ps]
        out[:, r] = row if exps is None else decode(row) * np.exp2(exps[page].astype(np.float64) - 127)[:, None]
    return out, there


def attention(Q, pools, exps, table, prefix_len, K_tree=None, V_tree=None, mask=None, decode=None, scale=None):
    """pools (k, v), exps (k, v) or (None, None).  Returns (O, A, S): the output, per output the sum of weight * |value| and
    per (b, h, i) the largest sum of |q k| (times scale) over visible keys -- what rounding errors are measured in."""
    B, Hq, n, D = Q.shape
    H, cap = pools[0].shape[1], table.shape[1] * pools[0].shape[2]
    g = Hq // H
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    O, A, S = np.zeros(Q.shape), np.zeros(Q.shape), np.zeros((B, Hq, n))
    for b in range(B):
        L = min(max(int(prefix_len[b]), 0), cap)
        k, there = gather(pools[0], exps[0], table[b], L, decode)
        v, _ = gather(pools[1], exps[1], table[b], L, decode)
        keep = np.flatnonzero(there)
        Kp, Vp = k[None][:, :, keep], v[None][:, :, keep]
        m, Kt, Vt = np.zeros((1, n, 1), dtype=np.uint64), np.zeros((1, H, 1, D)), np.zeros((1, H, 1, D))
        if K_tree is not None:
            m, Kt, Vt = mask[b:b + 1], K_tree[b:b + 1].copy(), V_tree[b:b + 1].copy()
            bits = np.unpackbits(np.ascontiguousarray(m[0]).view(np.uint8), axis=-1, bitorder="little")[:, :Kt.shape[2]]
            unseen = ~bits.any(0).astype(bool)
            Kt[0][:, unseen] = 0.0                       # rows that nobody sees may hold anything
            Vt[0][:, unseen] = 0.0
        args = (np.array([len(keep)]), m, scale)
        O[b] = tree_verify_attention(Q[b:b + 1], Kp, Vp, Kt, Vt, *args)[0]
        A[b] = tree_verify_attention(Q[b:b + 1], Kp, np.abs(Vp), Kt, np.abs(Vt), *args)[0]
        for h in range(Hq):
            allk = np.concatenate([Kp[0, h // g], Kt[0, h // g]], 0)
            S[b, h] = scale * (np.abs(Q[b, h]) @ np.abs(allk).T).max(-1)
    return O, A, S
