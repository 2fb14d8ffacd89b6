"""float64 oracle of the operators around a drafted tree: rotary rows with head norms, tree attention, sampling and
the accepted path.  Written from the definitions, one element or one row at a time; test infrastructure only."""
import math

import numpy as np


def rope_frequencies(rot, theta, scaling="plain", factor=1.0, trained_len=32768, beta_fast=32.0, beta_slow=1.0):
    """(angle per position of each pair, factor on cosine and sine)."""
    theta, factor = float(np.float32(theta)), float(np.float32(factor))
    f, m = [], 1.0
    for i in range(rot // 2):
        t = theta * factor ** (rot / (rot - 2.0)) if scaling == "ntk" else theta
        v = t ** (-2.0 * i / rot)
        if scaling == "linear":
            v /= factor
        if scaling == "yarn":
            lo = math.floor(rot * math.log(trained_len / (2 * math.pi * beta_fast)) / (2 * math.log(theta)))
            hi = math.ceil(rot * math.log(trained_len / (2 * math.pi * beta_slow)) / (2 * math.log(theta)))
            lo, hi = max(lo, 0), min(hi, rot - 1)
            r = min(max((i - lo) / (hi - lo if hi > lo else 0.001), 0.0), 1.0)
            v = v / factor * r + v * (1.0 - r)
        f.append(v)
    if scaling == "yarn" and factor > 1.0:
        m = 0.1 * math.log(factor) + 1.0
    return np.array(f), m


def norm_rope(x, pos, f, m, interleaved, weight=None, eps=1e-6):
    """x [rows, heads, d], pos [rows].  Returns the rows and, for tolerances, the size of what each was added up from."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt(np.mean(y * y, axis=-1, keepdims=True) + float(np.float32(eps))) * weight
    out, size = y.copy(), np.abs(y)
    half = len(f)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        t = (np.asarray(pos, dtype=np.float64) * f[i])[:, None]
        out[..., a] = m * (y[..., a] * np.cos(t) - y[..., b] * np.sin(t))
        out[..., b] = m * (y[..., b] * np.cos(t) + y[..., a] * np.sin(t))
        size[..., a] = size[..., b] = m * (np.abs(y[..., a]) + np.abs(y[..., b]))
    return out, size


def tree_path(parent, j):
    """Node j and the nodes it hangs from, a parent that is not an earlier node being the history."""
    path = []
    while True:
        path.append(j)
        up = int(parent[j])
        if not 0 <= up < j:
            return path
        j = up


def tree_attention(q, k_cache, v_cache, k_tree, v_tree, parent, scale):
    """One sequence: q [n, Hq, d], caches [len, Hkv, d], tree [n, Hkv, d].  Returns out and sum_t p_t |v_t|."""
    n, hq, d = q.shape
    hkv = k_tree.shape[1]
    out, size = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    for j in range(n):
        path = tree_path(parent, j)
        for h in range(hq):
            g = h // (hq // hkv)
            k = np.concatenate([k_cache[:, g], k_tree[path, g]])
            v = np.concatenate([v_cache[:, g], v_tree[path, g]])
            s = k @ q[j, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[j, h], size[j, h] = p @ v, p @ np.abs(v)
    return out, size


def tree_walk(parent, draft, decided, nodes):
    """Accepted nodes of one tree, in order."""
    if nodes == 0:
        return []
    path = [0]
    while True:
        for c in range(path[-1] + 1, nodes):
            if parent[c] == path[-1] and draft[c] == decided[path[-1]]:
                path.append(c)
                break
        else:
            return path


def sample(l, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row (float32 values): token, prob, entropy, kept, and how near the decision was (share of the weight
    between a border and the number it was compared with; inf where nothing was compared)."""
    l = np.asarray(l, dtype=np.float32).copy()
    l[np.isnan(l)] = -np.inf
    able = np.flatnonzero(l > -np.inf)
    if not len(able):
        return -1, 0.0, 0.0, 0, math.inf
    z = l[able].astype(np.float64)
    order = np.lexsort((able, -z))
    able, z = able[order], z[order]
    if not temperature > 0:
        return int(able[0]), 1.0, 0.0, 1, math.inf
    z = (z - z[0]) / float(np.float32(temperature))
    w = np.exp(z)
    near = math.inf
    if 0 < top_k < len(w):
        w, able = w[:top_k], able[:top_k]
    if top_p < 1.0:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        goal = max(float(np.float32(top_p)), 0.0) * w.sum()
        keep = before < goal
        keep[0] = True
        near = min(near, float(np.min(np.abs(before[1:] - goal))) / w.sum() if len(w) > 1 else math.inf)
        w, able = w[keep], able[keep]
    if min_p > 0.0:
        keep = w >= min(float(np.float32(min_p)), 1.0)
        w, able = w[keep], able[keep]
    total = w.sum()
    by_index = np.argsort(able)
    c = np.cumsum(w[by_index])
    goal = float(np.float32(u)) * total
    if len(w) > 1:
        near = min(near, float(np.min(np.abs(c[:-1] - goal))) / total)
    at = by_index[min(int(np.searchsorted(c, goal, side="right")), len(w) - 1)]
    p = w / total
    live = p[p > 0]
    return int(able[at]), float(p[at]), float(-np.sum(live * np.log(live))), len(w), near
