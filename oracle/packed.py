"""64-bit definitions of the operators around the cache held in 4 bits (numpy, plain loops where order matters).

TEST INFRASTRUCTURE ONLY, like the rest of this package.  bf16 arrays are uint16 bit patterns, as everywhere in the oracle.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# e4m3 values of the bytes 0 .. 126 (127 is NaN)
E4M3 = np.array([(1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 7) if b >> 3 else (b & 7) * 2.0 ** -9 for b in range(127)])


def bf16(bits: np.ndarray) -> np.ndarray:
    with np.errstate(invalid="ignore"):
        return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def nearest(x: np.ndarray, grid: np.ndarray) -> np.ndarray:
    """Index of the value of `grid` nearest to x >= 0; a tie goes to the even index, beyond the last value to that."""
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    below, above = x - grid[lo], grid[hi] - x
    return np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def quantise(bits: np.ndarray):
    """Rows [..., 128] -> codes [..., 64], scales [..., 8] (uint8) and the values that are kept (float64)."""
    x = bf16(bits).reshape(bits.shape[:-1] + (8, 16))
    odd = ~np.isfinite(x).all(-1)
    y = np.where(odd[..., None], 0.0, x)
    scale = nearest(np.abs(y).max(-1) / 6.0, E4M3)
    s = E4M3[scale][..., None]
    code = nearest(np.divide(np.abs(y), s, out=np.zeros_like(y), where=s > 0), E2M1)
    neg = (bits.reshape(x.shape) >> 15).astype(bool)
    code = np.where(odd[..., None], 0, code + 8 * neg).astype(np.uint8)
    scale = np.where(odd, 0x7F, scale).astype(np.uint8)
    code = code.reshape(bits.shape)
    codes = code[..., 0::2] | (code[..., 1::2] << 4)
    return codes, scale, decode(codes, scale)


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The values that rows of codes [..., 64] and scales [..., 8] stand for: [..., 128] float64."""
    n = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (8, 16))
    value = E2M1[n & 7] * np.where(n >> 3, -1.0, 1.0)
    grid = np.concatenate([E4M3, [np.nan]])
    return (value * grid[scales & 0x7F][..., None]).reshape(codes.shape[:-1] + (128,))


def depths(parent: np.ndarray) -> np.ndarray:
    d = np.zeros(parent.shape, np.int64)
    for b in range(parent.shape[0]):
        for i in range(1, parent.shape[1]):
            d[b, i] = d[b, parent[b, i]] + 1
    return d


def rope(qkv: np.ndarray, hq: int, hkv: int, pos: np.ndarray, theta: float, sections, adjacent: bool):
    """qkv [B][N][(hq + 2 hkv) * 128] bits, pos [B][N][3] -> q [B][N][hq][128], k, v [B][hkv][N][128] (float64), and what the
    roundings of the products are relative to (|x1| + |x2|), laid out as q and k."""
    B, N, _ = qkv.shape
    x = bf16(qkv).reshape(B, N, hq + 2 * hkv, 128)
    axis = np.repeat([0, 1, 2], sections)
    angle = pos[..., axis].astype(np.float64) * theta ** (-np.arange(64) / 64.0)
    c, s = np.cos(angle)[:, :, None], np.sin(angle)[:, :, None]
    y, size = x[:, :, :hq + hkv].copy(), np.empty((B, N, hq + hkv, 128))
    a, b = (np.s_[..., 0::2], np.s_[..., 1::2]) if adjacent else (np.s_[..., :64], np.s_[..., 64:])
    x1, x2 = y[a].copy(), y[b].copy()
    y[a], y[b] = x1 * c - x2 * s, x2 * c + x1 * s
    size[a] = size[b] = np.abs(x1) + np.abs(x2)
    k = np.swapaxes(y[:, :, hq:], 1, 2)
    return y[:, :, :hq], k, np.swapaxes(x[:, :, hq + hkv:], 1, 2), size[:, :, :hq], np.swapaxes(size[:, :, hq:], 1, 2)


def plan(length, add, drop, table, held, free, n_free, max_rows):
    """One plan, step by step.  Returns (fits, row_start, slots, row_seq, row_pos, table, held, free, n_free); the state's arrays are copies."""
    B, bps = table.shape
    t, h, f, n = table.copy(), held.copy(), free.copy(), int(n_free)
    row_start = np.zeros(B + 1, np.int32)
    slots, seq, pos = np.full(max_rows, -1, np.int64), np.full(max_rows, -1, np.int32), np.full(max_rows, -1, np.int32)
    no = (False, row_start.copy(), slots.copy(), seq.copy(), pos.copy(), table, held, free, int(n_free))
    if not 0 <= n <= len(f) or int(np.asarray(add, np.int64).sum()) > max_rows:
        return no
    for b in range(B):
        if length[b] < 0 or add[b] < 0 or not 0 <= held[b] <= bps or int(length[b]) + int(add[b]) > bps * 128:
            return no
    for b in range(B):
        if drop is not None and drop[b]:
            for i in range(h[b]):
                if n == len(f):
                    return no
                f[n] = t[b, i]
                n += 1
            h[b] = 0
    for b in range(B):
        while h[b] * 128 < int(length[b]) + int(add[b]):
            if n == 0:
                return no
            n -= 1
            t[b, h[b]] = f[n]
            h[b] += 1
    r = 0
    for b in range(B):
        for p in range(int(length[b]), int(length[b]) + int(add[b])):
            slots[r], seq[r], pos[r] = int(t[b, p // 128]) * 128 + p % 128, b, p
            r += 1
        row_start[b + 1] = r
    return True, row_start, slots, seq, pos, t, h, f, n


def rows_of(codes, scales, layer, plane, table, h, L):
    """Values of the first L rows of one sequence (its row of the block table) and kv head: [L][128]."""
    blocks = table[:(L + 127) // 128]
    return decode(codes[layer, plane, blocks, h].reshape(-1, 64)[:L], scales[layer, plane, blocks, h].reshape(-1, 8)[:L])


def tree_attn(q, codes, scales, layer, table, tree_k, tree_v, parent, prefix_len, scale=None):
    """Attention over the 4-bit cache: out [B][N][Hq][128] float64, and of every row what its roundings are relative to: sum_j p_j |v_j|
    [B][N][Hq][128], the largest sum of magnitudes of a score [B][N][Hq], and sum_j |v_j| [B][N][Hq][128]."""
    B, N, hq, _ = q.shape
    hkv = tree_k.shape[1]
    scale = 1 / np.sqrt(128.0) if scale is None else scale
    out, mass, all_v, size = np.empty(q.shape), np.empty(q.shape), np.empty(q.shape), np.empty(q.shape[:3])
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
            k = np.concatenate([rows_of(codes, scales, layer, 0, table[b], h, L), bf16(tree_k[b, h])])
            v = np.concatenate([rows_of(codes, scales, layer, 1, table[b], h, L), bf16(tree_v[b, h])])
            x = bf16(q[b, :, u])
            with np.errstate(invalid="ignore"):
                s = np.where(see, x @ k.T * scale, -np.inf)
                size[b, :, u] = np.where(see, np.abs(x) @ np.abs(k).T * scale, 0).max(-1)
                p = np.exp(s - s.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                for i in range(N):                       # (a row that is not seen has no part in it, whatever it holds)
                    out[b, i, u] = p[i, see[i]] @ v[see[i]]
                    mass[b, i, u] = p[i, see[i]] @ np.abs(v[see[i]])
                    all_v[b, i, u] = np.abs(v[see[i]]).sum(0)
    return out, mass, size, all_v
