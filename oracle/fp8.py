"""64-bit definitions of the operators around the cache held in 8 bits, and of those on its blocks (numpy, plain loops where order matters).

TEST INFRASTRUCTURE ONLY, like the rest of this package.  bf16 arrays are uint16 bit patterns, as everywhere in the oracle.
"""
from __future__ import annotations

import numpy as np

from .packed import E4M3, bf16, nearest

GROUP = 32


def decode(codes: np.ndarray) -> np.ndarray:
    """Values of e4m3 bytes."""
    grid = np.concatenate([E4M3, [np.nan]])
    return np.where(codes >> 7, -1.0, 1.0) * grid[codes & 0x7F]


def encode(x: np.ndarray) -> np.ndarray:
    """e4m3 bytes of the values nearest to x (float64); what is no finite number: NaN."""
    odd = ~np.isfinite(x)
    code = nearest(np.abs(np.where(odd, 0.0, x)), E4M3)
    return np.where(odd, 0x7F, code | (np.signbit(x).astype(np.int64) << 7)).astype(np.uint8)


def least_scale(most: float) -> float:
    e = -64
    while e < 64 and most > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def put(codes, scales, blk, off, x):
    """Rows x [rows][Hkv][128] (bits) of one plane to rows `off` of blocks `blk`: codes [blocks][Hkv][128][128] and scales [blocks][Hkv][4] are
    changed; the kept values [rows][Hkv][128] come back."""
    value = np.empty(x.shape)
    groups = {}
    for r, (b, o) in enumerate(zip(blk, off)):
        groups.setdefault((int(b), int(o) // GROUP), []).append(r)
    for (b, g), rows in groups.items():
        at = np.asarray(off)[rows]
        for h in range(x.shape[1]):
            y = bf16(x[rows, h])
            finite = np.where(np.isfinite(y), np.abs(y), 0.0)
            s = least_scale(finite.max())
            old = float(scales[b, h, g])
            if not (at % GROUP == 0).any():
                old = min(max(old, 2.0 ** -64), 2.0 ** 64) if old == old else 2.0 ** -64
                s = max(s, 2.0 ** np.ceil(np.log2(old)))
                if s != old:
                    lines = np.s_[b, h, g * GROUP:(g + 1) * GROUP]
                    codes[lines] = encode(decode(codes[lines]) * (old / s))
            scales[b, h, g] = s
            c = encode(y / s)
            codes[b, h, at] = c
            value[rows, h] = decode(c) * s
    return value


def append(codes, scales, table, tree_kv, path, n_acc, prefix_len):
    """The accepted rows of every layer behind the prefixes: codes, scales changed; the kept values at the nodes' places (NaN elsewhere)."""
    out = np.full(tree_kv.shape, np.nan)
    layers, _, B = tree_kv.shape[:3]
    for layer in range(layers):
        for plane in (0, 1):
            for b in range(B):
                n = int(n_acc[b])
                if n:
                    pos, node = int(prefix_len[b]) + np.arange(n), path[b, :n]
                    v = put(codes[layer, plane], scales[layer, plane], table[b, pos // 128], pos % 128, np.swapaxes(tree_kv[layer, plane, b][:, node], 0, 1))
                    out[layer, plane, b][:, node] = np.swapaxes(v, 0, 1)
    return out


def rows_of(codes, scales, layer, plane, table, h, L):
    """Values of the first L rows of one sequence (its row of the block table) and kv head [L][128], and their rows' scales [L]."""
    blocks = table[:(L + 127) // 128]
    s = np.repeat(np.float64(scales[layer, plane, blocks, h].reshape(-1)), GROUP)[:L]
    return decode(codes[layer, plane, blocks, h].reshape(-1, 128)[:L]) * s[:, None], s


def tree_attn(q, codes, scales, layer, table, tree_k, tree_v, parent, prefix_len, scale=None):
    """Attention over the 8-bit cache: out [B][N][Hq][128] float64, and of every row what its roundings are relative to, in a dict: `mass` =
    sum_j p_j |v_j| [B][N][Hq][128]; `size`, the largest sum of magnitudes of a score, and `far`, the score's change where each element of the query
    changes by the row's largest [B][N][Hq]; `small` = (max_j p_j s_j) sum_j |code_j| over the cached keys, s_j the scale of V's row [B][N][Hq][128]."""
    B, N, hq, _ = q.shape
    hkv = tree_k.shape[1]
    scale = 1 / np.sqrt(128.0) if scale is None else scale
    out, mass, small, size, far = np.empty(q.shape), np.empty(q.shape), np.zeros(q.shape), np.empty(q.shape[:3]), np.zeros(q.shape[:3])
    for b in range(B):
        L = int(prefix_len[b])
        see = np.zeros((N, L + N), bool)
        see[:, :L] = True
        for i in range(N):
            at = i
            while at >= 0:
                see[i, L + at] = True
                at = parent[b, at]
        for u in range(hq):
            h = u // (hq // hkv)
            ck, _ = rows_of(codes, scales, layer, 0, table[b], h, L)
            cv, sv = rows_of(codes, scales, layer, 1, table[b], h, L)
            k, v = np.concatenate([ck, bf16(tree_k[b, h])]), np.concatenate([cv, bf16(tree_v[b, h])])
            x = bf16(q[b, :, u])
            with np.errstate(invalid="ignore"):
                s = np.where(see, x @ k.T * scale, -np.inf)
                size[b, :, u] = np.where(see, np.abs(x) @ np.abs(k).T * scale, 0).max(-1)
                p = np.exp(s - s.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                if L:
                    far[b, :, u] = np.abs(x).max(-1) * np.abs(ck).sum(-1).max() * scale
                    small[b, :, u] = (p[:, :L] * sv).max(-1)[:, None] * np.abs(cv / sv[:, None]).sum(0)
                for i in range(N):                       # (a row that is not seen has no part in it, whatever it holds)
                    out[b, i, u] = p[i, see[i]] @ v[see[i]]
                    mass[b, i, u] = p[i, see[i]] @ np.abs(v[see[i]])
    return out, dict(mass=mass, size=size, far=far, small=small)


# ---- blocks: state (table, held, shares, free, n_free), arrays that are copied; None where something does not fit ---------------------------------


def _copies(table, held, shares, free, n_free):
    return table.copy(), held.copy(), shares.copy(), free.copy(), int(n_free)


def fork(src, dst, length, table, held, shares, free, n_free):
    """(pairs, length, state) after the sequences dst go on from src's rows."""
    t, h, s, f, n = _copies(table, held, shares, free, n_free)
    ln, nb, pairs = length.copy(), len(free), []
    if not 0 <= n <= nb or len(set(dst.tolist())) != len(dst) or set(dst.tolist()) & set(src.tolist()):
        return None
    for a, b in zip(src, dst):
        if not (0 <= a < len(h) and 0 <= b < len(h)) or h[b] != 0 or not 0 <= h[a] <= t.shape[1] or not 0 <= ln[a] <= h[a] * 128:
            return None
        L = int(ln[a])
        for j in range((L + 127) // 128):
            if not 0 <= t[a, j] < nb:
                return None
            if (j + 1) * 128 <= L:
                s[t[a, j]] += 1
                t[b, j] = t[a, j]
            else:
                if n == 0 or not 0 <= f[n - 1] < nb:
                    return None
                n -= 1
                t[b, j] = f[n]
                pairs.append((t[a, j], f[n]))
        h[b], ln[b] = (L + 127) // 128, L
    out = np.full((len(src), 2), -1, np.int32)
    out[:len(pairs)] = np.array(pairs, np.int32).reshape(-1, 2)
    return out, ln, (t, h, s, f, n)


def drop(which, table, held, shares, free, n_free):
    """The state after the sequences with which[b] != 0 have given back their blocks."""
    t, h, s, f, n = _copies(table, held, shares, free, n_free)
    nb, freed = len(f), []
    if not 0 <= n <= nb:
        return None
    for b in np.flatnonzero(which):
        if not 0 <= h[b] <= t.shape[1]:
            return None
        for x in t[b, :h[b]]:
            if not 0 <= x < nb or x in freed:
                return None
            s[x] -= 1
            if s[x] < 0:
                freed.append(x)
                s[x] = 0
        h[b] = 0
    if n + len(freed) > nb:
        return None
    for x in sorted(freed, reverse=True):
        f[n] = x
        n += 1
    return t, h, s, f, n


def compact(table, held, shares, free, n_free, max_pairs=None):
    """(pairs, state): the blocks in use at the lowest numbers among those in use or free."""
    t, h, s, f, n = _copies(table, held, shares, free, n_free)
    nb = len(f)
    if not 0 <= n <= nb or (h < 0).any() or (h > t.shape[1]).any():
        return None
    idle, live = f[:n].tolist(), sorted({int(x) for b in range(len(h)) for x in t[b, :h[b]]})
    if any(not 0 <= x < nb for x in idle + live) or len(set(idle)) != n or set(idle) & set(live):
        return None
    low = set(sorted(idle + live)[:len(live)])
    pairs = list(zip([x for x in live if x not in low], [x for x in sorted(idle) if x in low]))
    max_pairs = max(1, nb // 2) if max_pairs is None else max_pairs
    if len(pairs) > max_pairs:
        return None
    to = dict(pairs)
    for b in range(len(h)):
        t[b, :h[b]] = [to.get(int(x), int(x)) for x in t[b, :h[b]]]
    for x, y in pairs:
        s[y], s[x] = s[x], 0
    f[:n] = sorted(set(idle + live) - low, reverse=True)
    out = np.full((max_pairs, 2), -1, np.int32)
    out[:len(pairs)] = np.array(pairs, np.int32).reshape(-1, 2)
    return out, (t, h, s, f, n)
