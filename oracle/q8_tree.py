"""Float64 oracle of the 8-bit cache rows and of the drafted token tree."""
from __future__ import annotations

from typing import Optional

import numpy as np

from .h2o_oracle import bottomk, selection_keys

F64 = np.float64


def quantize(x):
    """(codes int8, scales float32) of the rows of x (last axis): scale =
    float32(max|x| / 127), 0 below the smallest normal float32, NaN for a row with
    an Inf or NaN; code = x / scale to the nearest integer, ties to even."""
    x = np.asarray(x, np.float32).astype(F64)
    bad = ~np.isfinite(x).all(-1)
    a = np.abs(np.where(np.isfinite(x), x, 0.0)).max(-1)
    scales = (a / 127).astype(np.float32)
    scales[scales < np.finfo(np.float32).tiny] = 0
    s = scales.astype(F64)
    ok = (s > 0) & ~bad
    # np.rint rounds ties to even; the float64 quotient of two float32 values never
    # rounds onto a tie that it is not (the two differ by more than 2^-33 of it)
    codes = np.where(ok[..., None], np.rint(x / np.where(ok, s, 1.0)[..., None]), 0.0)
    scales[bad] = np.nan
    return codes.astype(np.int8), scales


def dequantize(codes, scales):
    """The values that codes stand for, in float64 (the product is exact there)."""
    return codes.astype(F64) * np.asarray(scales, F64)[..., None]


def ancestors(parents):
    """seen [B,T,T]: node i sees node j (its ancestors and itself). A parent that is
    not in [-1, i) counts as -1."""
    parents = np.asarray(parents)
    B, T = parents.shape
    seen = np.zeros((B, T, T), bool)
    for b in range(B):
        for i in range(T):
            p = int(parents[b, i])
            if 0 <= p < i:
                seen[b, i] = seen[b, p]
            seen[b, i, i] = True
    return seen


def sdpa_tree(q, k_cache, v_cache, k_new, v_new, parents, scale: Optional[float] = None):
    """(out, lse) of every node over [cache || its ancestors and itself]. Only what a
    node sees enters its sums."""
    q = np.asarray(q)
    B, Hq, T, d = q.shape
    Hkv, M = k_cache.shape[1], k_cache.shape[2]
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(d) if scale is None else float(scale)
    seen = ancestors(parents)
    out, lse = np.zeros((B, Hq, T, d)), np.zeros((B, Hq, T))
    for b in range(B):
        for hq in range(Hq):
            h = hq // G
            for i in range(T):
                K = np.concatenate([k_cache[b, h], k_new[b, h, seen[b, i]]]).astype(F64)
                V = np.concatenate([v_cache[b, h], v_new[b, h, seen[b, i]]]).astype(F64)
                s = scale * (K @ q[b, hq, i].astype(F64))
                lam = s.max() + np.log(np.exp(s - s.max()).sum())
                lse[b, hq, i] = lam
                out[b, hq, i] = np.exp(s - lam) @ V
    return out, lse


def tree_accept(q, k_cache, k_new, v_new, lse, path, scale: Optional[float] = None):
    """(wsum [B,Hkv,M+A], k_acc, v_acc) of the path's nodes; entries outside [0, T)
    are no rows and no keys."""
    q = np.asarray(q)
    path = np.asarray(path)
    B, Hq, T, d = q.shape
    Hkv, M, A = k_cache.shape[1], k_cache.shape[2], path.shape[1]
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(d) if scale is None else float(scale)
    wsum = np.zeros((B, Hkv, M + A))
    k_acc, v_acc = (np.zeros((B, Hkv, A, d), np.asarray(x).dtype) for x in (k_new, v_new))
    for b in range(B):
        for h in range(Hkv):
            for a, n in enumerate(path[b]):
                if not 0 <= n < T:
                    continue
                k_acc[b, h, a], v_acc[b, h, a] = k_new[b, h, n], v_new[b, h, n]
                cols = [c for c in range(a + 1) if 0 <= path[b, c] < T]
                K = np.concatenate([k_cache[b, h], k_new[b, h, path[b, cols]]]).astype(F64)
                at = np.concatenate([np.arange(M), M + np.asarray(cols, int)])
                for hq in range(h * G, (h + 1) * G):
                    s = scale * (K @ q[b, hq, n].astype(F64))
                    wsum[b, h, at] += np.exp(s - lse[b, hq, n])
    return wsum, k_acc, v_acc


def tree_insert(k_cache, v_cache, scores, token_pos, k_acc, v_acc, wsum, path, pos0, T,
                policy: str = "h2o"):
    """Eviction and insert of a path's tokens (entries in [0, T)), whose number may differ
    between batch entries: (k_cache, v_cache, scores, token_pos, evict_idx), new copies;
    evict_idx is -1 at entries that are no token. pos0 [B]."""
    path = np.asarray(path)
    B, A = path.shape
    Hkv, M = scores.shape[1:]
    kc, vc, sc = k_cache.copy(), v_cache.copy(), np.asarray(scores, np.float32).copy()
    tp = None if token_pos is None else token_pos.copy()
    idx = np.full((B, Hkv, A), -1, np.int32)
    for b in range(B):
        at = [a for a in range(A) if 0 <= path[b, a] < T]
        if not at:
            continue
        one = slice(None) if policy == "h2o_orig" else slice(b, b + 1)
        keys = selection_keys(scores[one], None if token_pos is None else token_pos[one], policy,
                              int(pos0[b]) + len(at))
        slots = np.broadcast_to(bottomk(keys, len(at)), (1, Hkv, len(at)))[0]
        for h in range(Hkv):
            idx[b, h, at] = slots[h]
            kc[b, h, slots[h]], vc[b, h, slots[h]] = k_acc[b, h, at], v_acc[b, h, at]
            sc[b, h, slots[h]] = wsum[b, h, M + np.asarray(at)]
            if tp is not None:
                tp[b, h, slots[h]] = pos0[b] + np.arange(len(at), dtype=np.int32)
    return kc, vc, sc, tp, idx
