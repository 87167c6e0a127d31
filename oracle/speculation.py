"""Float64 definitions of the operators of a speculative decoding step (see include/ooco.h for their statements).

TEST INFRASTRUCTURE ONLY -- the product path never imports this file.  Written out node by node; values come as float64.
"""
from __future__ import annotations

import math

import numpy as np


def ancestors(parents):
    """For each node of one tree the list of nodes from its root to itself.  A parent that is no earlier node counts as none."""
    paths = []
    for t, p in enumerate(parents):
        p = int(p)
        paths.append((paths[p] if 0 <= p < t else []) + [t])
    return paths


def tree_masks(parents, query_start_loc, ctx_lens, words):
    T = int(query_start_loc[-1])
    masks, positions = np.zeros((T, words), np.uint64), np.zeros(T, np.int32)
    for i in range(len(ctx_lens)):
        q0, q1 = int(query_start_loc[i]), int(query_start_loc[i + 1])
        for t, path in enumerate(ancestors(parents[q0:q1])):
            positions[q0 + t] = ctx_lens[i]
            if t < 64 * words:
                positions[q0 + t] += len(path) - 1
                for j in path:
                    masks[q0 + t, j // 64] |= np.uint64(1 << (j % 64))
    return masks, positions


def rotate(x, positions, frequencies, interleaved, factor=1.0):
    """x [rows][heads][hd] rotated, float64, and the sum of the magnitudes that each value is made of."""
    n = 2 * len(frequencies)
    angle = np.asarray(positions, np.float64)[:, None, None] * np.asarray(frequencies)
    c, s = factor * np.cos(angle), factor * np.sin(angle)
    a, b = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    y, size = x.copy(), np.abs(x)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = abs(factor) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, size


def attn_tree(q, k, v, query_start_loc, ctx_lens, masks, scale=None):
    """k, v: per sequence [tokens][Hkv][hd].  Returns the output and sum(weight * |v|), both [T][Hq][hd]."""
    T, Hq, hd = q.shape
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    out, size = np.zeros((T, Hq, hd)), np.zeros((T, Hq, hd))
    for i in range(len(ctx_lens)):
        g = Hq // k[i].shape[1]
        for t in range(int(query_start_loc[i + 1] - query_start_loc[i])):
            row, ctx = int(query_start_loc[i]) + t, int(ctx_lens[i])
            n = min(len(k[i]) - ctx, 64 * masks.shape[1])
            seen = list(range(ctx)) + [ctx + j for j in range(n) if (int(masks[row, j // 64]) >> (j % 64)) & 1]
            if not seen:
                continue
            for h in range(Hq):
                s = scale * (k[i][seen, h // g] @ q[row, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                out[row, h] = p @ v[i][seen, h // g]
                size[row, h] = p @ np.abs(v[i][seen, h // g])
    return out, size


def _weights(p):
    return np.where(np.isfinite(p) & (p > 0), p, 0.0)


def verify_drafts(target, draft, tokens, parents, uniforms, final_uniforms, query_start_loc, max_path):
    """target, draft: float64 [T][vocab] (draft may be None); parents None: chains."""
    B, V = len(query_start_loc) - 1, target.shape[1]
    counts, path = np.zeros(B, np.int32), np.full((B, max_path), -1, np.int32)
    out = np.full((B, max_path + 1), -1, np.int32)
    for i in range(B):
        q0, n = int(query_start_loc[i]), min(int(query_start_loc[i + 1] - query_start_loc[i]), 256)
        if n == 0:
            continue
        par = [t - 1 if parents is None else (int(parents[q0 + t]) if 0 <= parents[q0 + t] < t else -1) for t in range(n)]
        at, taken, refused = 0, [], []
        while len(taken) < max_path:
            refused, rest, went = [], 1.0, None
            seen = []
            for c in range(n):
                if par[c] != at:
                    continue
                x = int(tokens[q0 + c])
                known = 0 <= x < V
                p = float(target[q0 + at, x]) if known and x not in seen else 0.0
                q = float(draft[q0 + c, x]) if draft is not None and known else 1.0
                if float(uniforms[q0 + c]) * q * rest < p:
                    went = c
                    break
                refused.append(c)
                seen.append(x)
                rest -= p
            if went is None:
                break
            taken.append(went)
            at, refused = went, []
        full = _weights(target[q0 + at])
        left = full.copy()
        if draft is not None and refused:
            left = _weights(full - draft[q0 + refused[0]])
        for c in refused:
            if draft is None and 0 <= tokens[q0 + c] < V:
                left[tokens[q0 + c]] = 0.0
        if not left.sum() > 0:
            left = full
        drawn = -1
        if left.sum() > 0:
            run = np.cumsum(left)
            past = np.flatnonzero((run > float(final_uniforms[i]) * run[-1]) & (left > 0))
            drawn = past[0] if len(past) else np.flatnonzero(left > 0)[-1]
        counts[i] = len(taken) + 1
        path[i, :len(taken)] = taken
        out[i, :len(taken) + 1] = [tokens[q0 + c] for c in taken] + [drawn]
    return counts, path, out


def kv_compact(k_cache, v_cache, block_tables, ctx_lens, path, counts, BS=16):
    """Pools [blocks][Hkv][hd/8][BS][8] and [blocks][Hkv][hd][BS], changed in place; the nodes move one after the other."""
    for i in range(len(ctx_lens)):
        for d in range(int(counts[i]) - 1):
            src, dst = int(ctx_lens[i]) + int(path[i, d]), int(ctx_lens[i]) + 1 + d
            if path[i, d] <= d + 1 or max(src, dst) // BS >= block_tables.shape[1]:
                continue
            sb, db = int(block_tables[i, src // BS]), int(block_tables[i, dst // BS])
            if not (0 <= sb < len(k_cache) and 0 <= db < len(k_cache)):
                continue
            k_cache[db, :, :, dst % BS] = k_cache[sb, :, :, src % BS]
            v_cache[db, :, :, dst % BS] = v_cache[sb, :, :, src % BS]


def rope_frequencies(kind, d, base, s=1.0, original=0.0, low=1.0, high=2.0):
    """Written from the statement in include/ooco.h, pair by pair."""
    out = []
    if kind == "base":
        base = base * s ** (d / (d - 2.0))
    for i in range(d // 2):
        f = base ** (-2.0 * i / d)
        if kind == "linear":
            f = f / s
        if kind == "wavelength":
            n = original * f / (2 * math.pi)
            w = 1.0 if n > high else 0.0 if n < low else (n - low) / (high - low)
            f = w * f + (1 - w) * f / s
        if kind == "ramp":
            c = lambda n: d * math.log(original / (2 * math.pi * n)) / (2 * math.log(base))
            a, b = (min(max(x, 0), d - 1) for x in (math.floor(c(high)), math.ceil(c(low))))
            w = 1.0 if i <= a else 0.0 if i >= b else 1.0 - (i - a) / (b - a)
            f = w * f + (1 - w) * f / s
        out.append(f)
    return np.array(out), 0.1 * math.log(s) + 1.0 if kind == "ramp" else 1.0
