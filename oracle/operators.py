"""CPU oracle of the operators on the caller's own tensors: rotary positions, attention of a chunk over a paged cache, logit rules.

THIS IS TEST INFRASTRUCTURE, NOT THE PRODUCT.  Only tests/ may import it.  It shares no code with the HIP path.  Everything is float64, row by row, from
the definitions in include/eagle.h; beside a result it returns what the result's rounding is bounded by."""
from __future__ import annotations

import math

import numpy as np


def chunk_rows(row_start, key_len, tree_base=None, tree_mask=None):
    """(row, sequence, token, position, path) of every row that a sequence owns; path: the tree nodes on the row's path, None for consecutive tokens."""
    out = []
    for s in range(len(key_len)):
        for r in range(int(row_start[s]), int(row_start[s + 1])):
            if tree_mask is None:
                t = int(key_len[s]) - int(row_start[s + 1]) + r
                out.append((r, s, t, t, None))
            else:
                path = [u for u in range(64) if int(tree_mask[r]) >> u & 1]
                out.append((r, s, int(tree_base[s]) + path[-1], int(tree_base[s]) + len(path) - 1, path))
    return out


def frequencies(rot, theta=10000.0, scaling="none", factor=1.0, low=1.0, high=4.0, trained_len=4096):
    """Radians a position, pair by pair."""
    L, out = trained_len, []
    if scaling == "base":
        theta = theta * factor ** (rot / (rot - 2))
    for p in range(rot // 2):
        f = theta ** (-2.0 * p / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "bands":
            w = 2 * math.pi / f
            if w > L / low:
                f /= factor
            elif w >= L / high:
                s = (L / w - low) / (high - low)
                f *= s + (1 - s) / factor
        elif scaling == "ramp":
            def pair(n):
                return rot * math.log(L / (2 * math.pi * n)) / (2 * math.log(theta))
            a, b = max(0, math.floor(pair(high))), min(rot - 1, math.ceil(pair(low)))
            t = min(1.0, max(0.0, (p - a) / max(b - a, 0.001)))
            f = f * (1 - t) + f / factor * t
        out.append(f)
    return np.array(out)


def rotate(x, positions, freqs, rot, interleaved, mscale=1.0, inverse=False):
    """x [rows, heads, dim] -> rotated, and per element the sum of absolute values that were added up."""
    x = np.asarray(x, dtype=np.float64)
    y, size = x.copy(), np.abs(x)
    for r in range(x.shape[0]):
        # the angle modulo a turn from whole turns in exact integer arithmetic would be the same to 1e-10: positions here stay below 2^22
        ang = float(positions[r]) * freqs * (-1 if inverse else 1)
        for p in range(rot // 2):
            i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + rot // 2)
            c, s = mscale * math.cos(ang[p]), mscale * math.sin(ang[p])
            a, b = x[r, :, i], x[r, :, j]
            y[r, :, i], y[r, :, j] = a * c - b * s, b * c + a * s
            size[r, :, i] = size[r, :, j] = abs(mscale) * (np.abs(a) + np.abs(b))
    return y, size


def attention(q, k_cache, v_cache, table, rows, n_rows_out, key_len, *, page, scale, softcap=0.0, slopes=None, window=0, prefix=None, tree_base=None):
    """rows: chunk_rows().  k_cache, v_cache [pages, kv heads, page tokens, dim].  -> out [rows, heads, dim] (nan: rows nobody owns), weighted mean of |v|, largest
    scale * sum |q k| of a visible token, number of visible tokens."""
    q = np.asarray(q, dtype=np.float64)
    R, H, D = q.shape
    KVH = k_cache.shape[1]
    out, mean = np.full((R, H, D), np.nan), np.zeros((R, H, D))
    big, count = np.zeros((R, H)), np.zeros(R, dtype=np.int64)
    for r, s, t, pos, path in rows:
        K = int(key_len[s])
        seen, dist = [], []
        for j in range(K):
            pj = j
            if path is None:
                ok = j <= t
            else:
                base = int(tree_base[s])
                ok = j < base or (j - base) in path
                if j >= base:
                    pj = base + sum(u < j - base for u in path)
            if window > 0 and pos - pj >= window:
                ok = False
            if prefix is not None and j < (int(prefix[s]) if path is None else min(int(prefix[s]), int(tree_base[s]))):
                ok = True
            if ok and 0 <= table[s][j // page] < k_cache.shape[0]:
                seen.append(j)
                dist.append(abs(pos - pj))
        count[r] = len(seen)
        if not seen:
            out[r] = 0.0
            continue
        pages = np.array([table[s][j // page] for j in seen])
        slots = np.array([j % page for j in seen])
        for h in range(H):
            kv = h // (H // KVH)
            k, v = k_cache[pages, kv, slots].astype(np.float64), v_cache[pages, kv, slots].astype(np.float64)
            x = k @ q[r, h] * scale
            big[r, h] = (np.abs(k) @ np.abs(q[r, h])).max() * abs(scale)
            if softcap > 0:
                x = softcap * np.tanh(x / softcap)
            if slopes is not None:
                x = x - float(slopes[h]) * np.array(dist)
            w = np.exp(x - x.max())
            w /= w.sum()
            out[r, h], mean[r, h] = w @ v, w @ np.abs(v)
    return out, mean, big, count


def logit_rules(x, row_start, *, tokens=None, n_tokens=None, n_prompt=None, repetition=None, presence=None, frequency=None, bias=None, path_token=None, path_mask=None,
                allowed=None, allowed_row=None):
    """x [rows, vocab] -> after the rules, and per element the sum of absolute values on the way."""
    y = np.asarray(x, dtype=np.float64).copy()
    size = np.abs(y)
    R, V = y.shape
    for s in range(len(row_start) - 1):
        for r in range(int(row_start[s]), int(row_start[s + 1])):
            seen, count = set(), {}
            text = [] if tokens is None else [(int(t), i >= (0 if n_prompt is None else int(n_prompt[s]))) for i, t in enumerate(tokens[s][:int(n_tokens[s])])]
            if path_mask is not None:
                text += [(int(path_token[int(row_start[s]) + u]), True) for u in range(64)
                         if int(path_mask[r]) >> u & 1 and int(row_start[s]) + u < int(row_start[s + 1])]
            for t, new in text:
                if 0 <= t < V:
                    seen.add(t)
                    count[t] = count.get(t, 0) + new
            rep = 1.0 if repetition is None or not repetition[s] > 0 else float(repetition[s])
            for t in seen:
                y[r, t] = y[r, t] / rep if y[r, t] > 0 else y[r, t] * rep
                size[r, t] = abs(y[r, t])
                if count[t] > 0:
                    off = (0.0 if presence is None else float(presence[s])) + (0.0 if frequency is None else float(frequency[s])) * count[t]
                    y[r, t] -= off
                    size[r, t] += abs(off)
            if bias is not None:
                last = {}
                for i in range(int(bias[0][s]), int(bias[0][s + 1])):
                    last[int(bias[1][i])] = float(bias[2][i])
                for t, b in last.items():
                    if 0 <= t < V:
                        y[r, t] += b
                        size[r, t] += abs(b)
            m = r if allowed_row is None else int(allowed_row[r])
            if allowed is not None and 0 <= m < len(allowed):
                for t in range(V):
                    if not int(allowed[m][t // 32]) >> (t % 32) & 1:
                        y[r, t] = -math.inf
    return y, size
