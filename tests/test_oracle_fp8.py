"""Pins of the 64-bit definitions around the 8-bit cache and its blocks (CPU)."""
import numpy as np
import pytest
import torch

from oracle import fp8, packed
from paper_2408_15562_b200 import synth


def bits(x):
    return synth.f32_to_bf16_bits(np.asarray(x, np.float32))


def test_codes_are_torchs():
    byte = np.arange(256).astype(np.uint8)
    want = torch.from_numpy(byte).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(fp8.decode(byte), want)
    rng = np.random.default_rng(0)
    m = np.concatenate([rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 8, 20000), (np.arange(4096) / 16 + 1 / 32) * 2.0 ** rng.integers(-8, 2, 4096), [0.0, -0.0, 448, 464, 2.0 ** -10]])
    m = np.clip(m, -448, 448)
    want = torch.from_numpy(m).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(fp8.encode(m), want)
    assert fp8.encode(np.array([500.0, -1e9])).tolist() == [0x7E, 0xFE] and fp8.encode(np.array([np.nan, np.inf])).tolist() == [0x7F, 0x7F]


def test_scales_by_hand():
    for most, want in ((448, 1), (448.5, 2), (896, 2), (1.75, 2.0 ** -8), (1.7578125, 2.0 ** -7), (0, 2.0 ** -64), (1e-30, 2.0 ** -64), (3e38, 2.0 ** 64)):
        assert fp8.least_scale(most) == want


def test_a_group_begins_and_goes_on():
    codes, scales = np.full((2, 1, 128, 128), 0x7F, np.uint8), np.full((2, 1, 4), np.nan, np.float32)
    x = np.zeros((3, 1, 128))
    x[0, 0, 0], x[1, 0, 1], x[2, 0, 2] = 448, -3.0, 2.0 ** -9
    v = fp8.put(codes, scales, [1, 1, 1], [32, 33, 34], bits(x))
    assert scales[1, 0].tolist()[1] == 1 and np.isnan(scales[1, 0, [0, 2, 3]]).all() and np.isnan(scales[0]).all()
    np.testing.assert_array_equal(v, x)
    # a larger row: everything by twice the scale; the least code falls to a tie that goes to zero
    y = np.zeros((1, 1, 128))
    y[0, 0, 5] = 500
    v = fp8.put(codes, scales, [1], [35], bits(y))
    assert scales[1, 0, 1] == 2 and v[0, 0, 5] == 512                     # (500 / 2 lies between 240 and 256)
    now = fp8.decode(codes[1, 0, 32:36]) * 2.0
    assert now[0, 0] == 448 and now[1, 1] == -3.0 and now[2, 2] == 0.0
    # a smaller one: the scale stays
    fp8.put(codes, scales, [1], [36], bits(np.full((1, 1, 128), 0.25)))
    assert scales[1, 0, 1] == 2 and (fp8.decode(codes[1, 0, 36]) * 2 == 0.25).all()
    # and the group begun anew forgets it
    fp8.put(codes, scales, [1], [32], bits(np.full((1, 1, 128), 0.25)))
    assert scales[1, 0, 1] == 2.0 ** -10


@pytest.mark.parametrize("own,end", [(0.0, -64), (-1.0, -64), (1e-30, -64), (float("nan"), -64), (1e30, 64), (float("inf"), 64)])
def test_a_scale_outside_the_range_is_the_nearer_end(own, end):
    codes, scales = np.zeros((1, 1, 128, 128), np.uint8), np.full((1, 1, 4), own, np.float32)
    codes[0, 0, 0, :3] = 0x38, 0x7E, 0xB8              # 1, 448 and -1
    before = codes[0, 0, 0].copy()
    x = np.zeros((1, 1, 128))
    x[0, 0, 0] = 2.0 ** -60
    v = fp8.put(codes, scales, [0], [1], bits(x))
    assert scales[0, 0, 0] == 2.0 ** end and v[0, 0, 0] == (2.0 ** -60 if end < 0 else 0)
    np.testing.assert_array_equal(codes[0, 0, 0], before)


def test_rows_one_by_one_end_where_rows_together_do():
    """Normal values: a scale that rises step by step leaves the codes that the last one gives at once (double rounding only below the least normal code)."""
    rng = np.random.default_rng(1)
    x = bits(rng.standard_normal((32, 2, 128)) * 2.0 ** np.arange(-8, 0).repeat(4)[:, None, None])
    a, sa = np.zeros((1, 2, 128, 128), np.uint8), np.ones((1, 2, 4), np.float32)
    b, sb = a.copy(), sa.copy()
    fp8.put(a, sa, [0] * 32, np.arange(32), x)
    for i in range(32):
        fp8.put(b, sb, [0], [i], x[i:i + 1])
    np.testing.assert_array_equal(sa, sb)
    da, db = fp8.decode(a[0, :, :32]), fp8.decode(b[0, :, :32])
    normal = np.abs(da) >= 2.0 ** -6
    assert normal.mean() > 0.3
    np.testing.assert_array_equal(da[normal], db[normal])
    assert (np.abs(da - db) <= 2.0 ** -9).all()


def test_the_kept_values_are_within_a_sixteenth():
    rng = np.random.default_rng(2)
    x = bits(rng.standard_normal((40, 3, 128)))
    codes, scales = np.zeros((1, 3, 128, 128), np.uint8), np.ones((1, 3, 4), np.float32)
    v, y = fp8.put(codes, scales, [0] * 40, np.arange(40), x), packed.bf16(x)
    s = np.repeat(scales[0].T, 32, 0)[:40, :, None]
    assert (np.abs(v - y) <= np.maximum(np.abs(y) / 16, s * 2.0 ** -10)).all()
    got, _ = fp8.rows_of(codes[None, None], scales[None, None], 0, 0, np.array([0]), 1, 40)
    np.testing.assert_array_equal(got, v[:, 1])


def test_how_far_small_elements_are_off():
    """At most 2^-10 scales, which is below 2^-17 of the group's largest but may be above 2^-18 of it; each time the group is rounded again at most as much of the new scale: all in all twice the last."""
    codes, scales = np.zeros((1, 1, 128, 128), np.uint8), np.ones((1, 1, 4), np.float32)
    x = np.zeros((1, 1, 128))
    x[0, 0, :2] = 225, 2.0 ** -10
    v = fp8.put(codes, scales, [0], [0], bits(x))
    assert scales[0, 0, 0] == 1 and v[0, 0, 1] == 0 and 2.0 ** -18 < 2.0 ** -10 / 225 < 2.0 ** -17
    rng = np.random.default_rng(5)
    f = rng.standard_normal((32, 1, 128)) * 2.0 ** np.arange(-16, 16)[:, None, None]
    y = packed.bf16(bits(f))
    for i in range(32):
        fp8.put(codes, scales, [0], [i], bits(f[i:i + 1]))
    got, s = fp8.rows_of(codes[None, None], scales[None, None], 0, 0, np.array([0]), 0, 32)
    assert (s < np.abs(y).max() / 224).all()
    assert (np.abs(got - y[:, 0]) <= np.maximum(np.abs(y[:, 0]) / 16, s[:, None] * 2.0 ** -10) + s[:, None] * 2.0 ** -10).all()


def test_attention_is_the_plain_one_on_the_decoded_rows():
    rng = np.random.default_rng(3)
    B, N, hq, hkv, L = 2, 5, 4, 2, np.array([70, 0])
    codes = fp8.encode(rng.standard_normal((1, 2, 3, hkv, 128, 128)) * 60)
    scales = (2.0 ** rng.integers(-8, -4, (1, 2, 3, hkv, 4))).astype(np.float32)
    table = np.array([[2], [1]], np.int32)
    q, tk, tv = bits(rng.standard_normal((B, N, hq, 128))), bits(rng.standard_normal((B, hkv, N, 128))), bits(rng.standard_normal((B, hkv, N, 128)))
    parent = np.array([[-1, 0, 0, 1, 3], [-1, 0, 1, 2, 3]], np.int32)
    out, of = fp8.tree_attn(q, codes, scales, 0, table, tk, tv, parent, L)
    for b in range(B):
        for i in range(N):
            way, at = [], i
            while at >= 0:
                way.append(at)
                at = parent[b, at]
            for u in range(hq):
                h = u // 2
                rows = [np.concatenate([(fp8.decode(codes[0, p, table[b, 0], h]) * np.repeat(scales[0, p, table[b, 0], h].astype(float), 32)[:, None])[:L[b]],
                                        packed.bf16(t[b, h, way])]) for p, t in ((0, tk), (1, tv))]
                s = rows[0] @ packed.bf16(q[b, i, u]) / np.sqrt(128)
                p = np.exp(s - s.max())
                np.testing.assert_allclose(out[b, i, u], p @ rows[1] / p.sum(), rtol=1e-12, atol=1e-13)
    assert (of["mass"] >= np.abs(out) - 1e-12).all() and (of["far"][1] == 0).all()


def consistent(t, h, s, f, n):
    """Every block is on the stack, or held by shares + 1 sequences (or by none and nobody's)."""
    nb, count = len(f), np.zeros(len(f), int)
    for b in range(len(h)):
        row = t[b, :h[b]].tolist()
        assert len(set(row)) == len(row)
        count[row] += 1
    idle = f[:n].tolist()
    assert len(set(idle)) == n and (count[idle] == 0).all() if n else True
    np.testing.assert_array_equal(s, np.maximum(count - 1, 0))
    assert n + (count > 0).sum() == nb


@pytest.mark.parametrize("seed", range(6))
def test_sequences_keep_their_rows_whatever_happens_to_the_blocks(seed):
    rng = np.random.default_rng(seed)
    B, bps, nb = 9, 5, 30
    pool = np.full((nb, 128), -1)                       # what each row holds: a number of its own
    t, h, s, f, n = np.zeros((B, bps), np.int32), np.zeros(B, np.int32), np.zeros(nb, np.int32), rng.permutation(nb).astype(np.int32), nb
    length, want, number = np.zeros(B, np.int32), [[] for _ in range(B)], 0
    moved = forked = 0
    for step in range(60):
        what = rng.choice(["grow", "fork", "drop", "compact"])
        if what == "grow":
            add = np.where(rng.random(B) < 0.3, rng.integers(0, 200, B), 0)
            add = np.minimum(add, bps * 128 - length).astype(np.int32)
            ok, start, slots, _, _, t, h, f, n = packed.plan(length, add, None, t, h, f, n, 10000)
            if ok:
                for b in range(B):
                    for slot in slots[start[b]:start[b + 1]]:
                        pool.reshape(-1)[slot] = number
                        want[b].append(number)
                        number += 1
                length = (length + add).astype(np.int32)
        if what == "fork":
            busy, idle = np.flatnonzero(h > 0), np.flatnonzero(h == 0)
            if len(busy) and len(idle):
                k = int(rng.integers(1, len(idle) + 1))
                src, dst = rng.choice(busy, k).astype(np.int32), rng.permutation(idle)[:k].astype(np.int32)
                r = fp8.fork(src, dst, length, t, h, s, f, n)
                if r:
                    pairs, length, (t, h, s, f, n) = r
                    for a, b in pairs[pairs[:, 0] >= 0]:
                        pool[b] = pool[a]
                    for a, b in zip(src, dst):
                        want[b] = list(want[a])
                    forked += 1
        if what == "drop":
            which = (rng.random(B) < 0.25).astype(np.int32)
            t, h, s, f, n = fp8.drop(which, t, h, s, f, n)
            for b in np.flatnonzero(which):
                want[b], length[b] = [], 0
        if what == "compact":
            pairs, (t, h, s, f, n) = fp8.compact(t, h, s, f, n)
            pairs = pairs[pairs[:, 0] >= 0]
            assert not set(pairs[:, 0]) & set(pairs[:, 1])
            for a, b in pairs:
                pool[b] = pool[a]
                pool[a] = -7
            moved += len(pairs)
            held = {int(x) for b in range(B) for x in t[b, :h[b]]}
            assert held == set(range(len(held)))
        consistent(t, h, s, f, n)
        for b in range(B):
            got = pool[t[b, :h[b]]].reshape(-1)[:length[b]].tolist()
            assert got == want[b]
    assert moved and forked


def test_what_does_not_fit():
    t, h, s, f = np.zeros((3, 2), np.int32), np.array([1, 0, 0], np.int32), np.zeros(4, np.int32), np.array([1, 2, 3, 0], np.int32)
    L, i32 = np.array([100, 0, 0], np.int32), lambda *x: np.array(x, np.int32)  # noqa: E731
    assert fp8.fork(i32(0), i32(1), L, t, h, s, f, 3) is not None
    for src, dst, n in ((i32(0), i32(0), 3), (i32(0, 0), i32(1, 1), 3), (i32(0, 1), i32(1, 2), 3), (i32(3), i32(1), 3), (i32(0), i32(-1), 3), (i32(0), i32(1), 0), (i32(0), i32(1), 5)):
        assert fp8.fork(src, dst, L, t, h, s, f, n) is None
    assert fp8.drop(i32(1, 0, 0), t, h, s, f, 3)[4] == 4 and fp8.drop(i32(1, 0, 0), t, h, s, f, 4) is None
    both = np.array([1, 1, 0], np.int32)                # two hold block 0, and its count says one
    assert fp8.drop(i32(1, 1, 0), t, both, s, f, 3) is None
    assert fp8.compact(t, h, s, f, 3)[0].max() == -1 and fp8.compact(t, h, s, i32(0, 1, 2, 3), 3) is None and fp8.compact(t, h, s, i32(1, 1, 2, 3), 3) is None
    t2 = np.array([[3, 0], [0, 0], [0, 0]], np.int32)
    assert fp8.compact(t2, h, s, i32(2, 0, 1, 9), 3)[0].tolist() == [[3, 0], [-1, -1]] and fp8.compact(t2, h, s, i32(2, 0, 1, 9), 3, 0) is None
