"""Writes into the 8-bit cache, and forks, drops, compactions and copies of blocks, on the GPU against the definitions: bit for bit."""
import threading

import numpy as np
import pytest
import torch

from oracle import fp8, packed
from paper_2408_15562_b200 import binding, synth
from tests import helpers

pytestmark = pytest.mark.gpu

b16, dev = binding.bf16_tensor, helpers.dev


def _context(hq=4, hkv=2, **kw):
    kw.setdefault("max_nodes", 64)
    return binding.Context(hq, hkv, 16, 512, **kw)


def _rows(rng, shape, spread=6):
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-spread, spread + 1, shape[:-1] + (1,))
    return synth.f32_to_bf16_bits(x.astype(np.float32))


def _garbage(rng, layers, nb, hkv):
    return rng.integers(0, 256, (layers, 2, nb, hkv, 128, 128)).astype(np.uint8), (2.0 ** rng.integers(-9, 3, (layers, 2, nb, hkv, 4))).astype(np.float32)


def _same(got, want):
    """Codes with a NaN compared by what they are, not by its sign."""
    got, want = got.cpu().numpy(), want.copy()
    got = np.where((got & 0x7F) == 0x7F, 0x7F, got)
    np.testing.assert_array_equal(got, np.where((want & 0x7F) == 0x7F, 0x7F, want))


@pytest.mark.parametrize("rows,start", [(1, 0), (1, 31), (1, 32), (1, 77), (2, 31), (31, 1), (32, 0), (33, 0), (64, 5), (127, 1), (128, 0), (300, 45), (4000, 9)])
@pytest.mark.parametrize("hkv", [1, 2, 5])
def test_rows_behind_what_is_there(rows, start, hkv):
    rng = np.random.default_rng(rows * 7 + start)
    layers, nb = 2, (start + rows + 127) // 128 + 2
    order = rng.permutation(nb)
    pos = start + np.arange(rows)
    slots = order[pos // 128].astype(np.int64) * 128 + pos % 128
    codes, scales = _garbage(rng, layers, nb, hkv)
    k, v = (_rows(rng, (hkv, rows, 128)) for _ in range(2))
    d_codes, d_scales = dev(codes), dev(scales)
    ctx = _context(hkv, hkv, n_layers=layers)
    kr, vr = (torch.zeros((hkv, rows, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.kv_write_fp8(b16(k), b16(v), dev(slots), d_codes, d_scales, layer=1, k_rounded=kr, v_rounded=vr)
    ctx.check()
    for plane, x, back in ((0, k, kr), (1, v, vr)):
        value = fp8.put(codes[1, plane], scales[1, plane], slots // 128, slots % 128, np.swapaxes(x, 0, 1))
        np.testing.assert_array_equal(back.float().cpu().numpy(), np.swapaxes(value, 0, 1))
    _same(d_codes, codes)
    np.testing.assert_array_equal(d_scales.cpu().numpy(), scales)


def test_rows_of_many_sequences_some_left_out():
    """Runs of several sequences one behind the other, entries of -1 before, in and between them."""
    rng = np.random.default_rng(3)
    hkv, nb = 3, 60
    order, slots = rng.permutation(nb), []
    for b in range(20):
        start, n = int(rng.integers(0, 200)), int(rng.integers(1, 150))
        pos = start + np.arange(n)
        at = order[3 * b + pos // 128].astype(np.int64) * 128 + pos % 128
        at[rng.random(n) < 0.2] = -1
        slots += at.tolist() + [-1] * int(rng.integers(0, 3))
    slots = np.array(slots)
    rows = len(slots)
    codes, scales = _garbage(rng, 1, nb, hkv)
    k, v = (_rows(rng, (hkv, rows, 128)) for _ in range(2))
    d_codes, d_scales = dev(codes), dev(scales)
    ctx = _context(hkv, hkv)
    kr, vr = b16(k), b16(v)
    ctx.kv_write_fp8(kr, vr, dev(slots), d_codes, d_scales, k_rounded=kr, v_rounded=vr)        # (in place)
    ctx.check()
    there = slots >= 0
    for plane, x, back in ((0, k, kr), (1, v, vr)):
        value = fp8.put(codes[0, plane], scales[0, plane], slots[there] // 128, slots[there] % 128, np.swapaxes(x, 0, 1)[there])
        want = packed.bf16(x)
        want[:, there] = np.swapaxes(value, 0, 1)
        np.testing.assert_array_equal(back.float().cpu().numpy(), want)
    _same(d_codes, codes)
    np.testing.assert_array_equal(d_scales.cpu().numpy(), scales)


def test_a_sequence_written_row_by_row_with_rising_scales():
    rng = np.random.default_rng(4)
    hkv, n = 2, 140
    x = _rows(rng, (2, hkv, n, 128), 0)
    f = packed.bf16(x) * 2.0 ** np.linspace(-20, 20, n)[None, None, :, None].round()
    x = synth.f32_to_bf16_bits(f.astype(np.float32))
    codes, scales = _garbage(rng, 1, 2, hkv)
    d_codes, d_scales = dev(codes), dev(scales)
    ctx = _context(hkv, hkv)
    for i in range(n):
        ctx.kv_write_fp8(b16(x[0, :, i:i + 1]), b16(x[1, :, i:i + 1]), dev(np.array([i], np.int64)), d_codes, d_scales)
        for plane in (0, 1):
            fp8.put(codes[0, plane], scales[0, plane], np.array([i // 128]), np.array([i % 128]), np.swapaxes(x[plane, :, i:i + 1], 0, 1))
    ctx.check()
    _same(d_codes, codes)
    np.testing.assert_array_equal(d_scales.cpu().numpy(), scales)


@pytest.mark.parametrize("what", ["zeros", "largest", "least", "ties", "nan", "inf", "own scale", "no scale", "sign of zero", "all odd"])
def test_values_at_the_ends(what):
    rng = np.random.default_rng(5)
    hkv, rows, start = 2, 40, 3
    codes, scales = _garbage(rng, 1, 1, hkv)
    x = _rows(rng, (2, hkv, rows, 128), 0)
    if what == "zeros": x[:] = 0
    if what == "largest": x[:, :, ::3, ::5] = 0x7F7F
    if what == "least": x = synth.f32_to_bf16_bits((packed.bf16(x) * 2.0 ** -75).astype(np.float32))
    if what == "ties":                             # halves between neighbouring codes, at every power of two
        m = 1 + (2 * rng.integers(0, 8, x.shape) + 1) / 16
        x = synth.f32_to_bf16_bits((m * 2.0 ** rng.integers(-12, 7, x.shape) * rng.choice([-1, 1], x.shape)).astype(np.float32))
    if what == "nan": x[0, 0, 5, 7], x[1, 1, 0, 0] = 0x7FC0, 0xFFC1
    if what == "inf": x[0, 0, 5, 7], x[1, 1, 0, 0], x[1, 1, 0, 1] = 0x7F80, 0xFF80, 0x7F80
    if what == "own scale": scales[:] = rng.uniform(1e-3, 0.3, scales.shape)
    if what == "no scale": scales[:] = rng.choice([0.0, -1.0, np.nan, np.inf, 1e-30, 1e30], scales.shape)
    if what == "sign of zero": x[:, :, :, ::2] = 0x8000
    if what == "all odd": x[:] = 0x7F80
    slots = start + np.arange(rows)
    d_codes, d_scales = dev(codes), dev(scales)
    ctx = _context(hkv, hkv)
    kr, vr = (torch.zeros((hkv, rows, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.kv_write_fp8(b16(x[0]), b16(x[1]), dev(slots), d_codes, d_scales, k_rounded=kr, v_rounded=vr)
    ctx.check()
    for plane, back in ((0, kr), (1, vr)):
        value = fp8.put(codes[0, plane], scales[0, plane], slots // 128, slots % 128, np.swapaxes(x[plane], 0, 1))
        np.testing.assert_array_equal(back.float().cpu().numpy(), np.swapaxes(value, 0, 1))
    _same(d_codes, codes)
    np.testing.assert_array_equal(d_scales.cpu().numpy(), scales)


def test_slots_outside_the_cache_are_reported_and_left_out():
    rng = np.random.default_rng(6)
    codes, scales = _garbage(rng, 1, 3, 2)
    k, v = (_rows(rng, (2, 6, 128)) for _ in range(2))
    slots = np.array([32, 33, 3 * 128, -2, 1 << 40, 34], np.int64)
    d_codes, d_scales = dev(codes), dev(scales)
    ctx = _context()
    ctx.kv_write_fp8(b16(k), b16(v), dev(slots), d_codes, d_scales)
    assert ctx.status() == -5
    at = np.array([0, 1, 5])
    for plane, x in ((0, k), (1, v)):
        fp8.put(codes[0, plane], scales[0, plane], slots[at] // 128, slots[at] % 128, np.swapaxes(x, 0, 1)[at])
    _same(d_codes, codes)
    np.testing.assert_array_equal(d_scales.cpu().numpy(), scales)


@pytest.mark.parametrize("B,N,hkv,layers", [(1, 1, 1, 1), (1, 60, 2, 3), (5, 17, 2, 2), (3, 256, 1, 1), (40, 6, 2, 1)])
def test_append(B, N, hkv, layers):
    rng = np.random.default_rng(N)
    L = rng.integers(0, 300, B).astype(np.int32)
    bps = (300 + N + 127) // 128
    nb = B * bps
    table = rng.permutation(nb).reshape(B, bps).astype(np.int32)
    codes, scales = _garbage(rng, layers, nb, hkv)
    tree = _rows(rng, (layers, 2, B, hkv, N, 128))
    path, n_acc = np.full((B, N), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        n_acc[b] = rng.integers(0 if B > 1 else 1, N + 1)
        path[b, :n_acc[b]] = np.sort(rng.permutation(N)[:n_acc[b]])
    d_codes, d_scales = dev(codes), dev(scales)
    ctx = _context(hkv, hkv, n_layers=layers, max_batch=B, max_nodes=N)
    back = torch.full((layers, 2, B, hkv, N, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    new_len = ctx.kv_append_fp8(d_codes, d_scales, dev(table), b16(tree), dev(path), dev(n_acc), dev(L), rounded=back)
    ctx.check()
    want = fp8.append(codes, scales, table, tree, path, n_acc, L)
    np.testing.assert_array_equal(new_len.cpu().numpy(), L + n_acc)
    np.testing.assert_array_equal(back.float().cpu().numpy(), want)
    _same(d_codes, codes)
    np.testing.assert_array_equal(d_scales.cpu().numpy(), scales)


@pytest.mark.parametrize("what", ["node", "low node", "count", "length", "block"])
def test_appends_out_of_range_are_reported_and_leave_out_their_rows(what):
    rng = np.random.default_rng(8)
    B, N, hkv = 2, 8, 2
    table, L = rng.permutation(4).reshape(2, 2).astype(np.int32), np.array([130, 20], np.int32)
    codes, scales = _garbage(rng, 1, 4, hkv)
    tree = _rows(rng, (1, 2, B, hkv, N, 128))
    path, n_acc = np.tile(np.arange(N, dtype=np.int32), (B, 1)), np.array([3, 4], np.int32)
    if what == "node": path[0, 1] = N
    if what == "low node": path[0, 1] = -1
    if what == "count": n_acc[0] = N + 1
    if what == "length": L[0] = 254
    if what == "block": table[0, 1] = 4
    ctx = _context(hkv, hkv, max_batch=B, max_nodes=N)
    d_codes, d_scales = dev(codes), dev(scales)
    ctx.kv_append_fp8(d_codes, d_scales, dev(table), b16(tree), dev(path), dev(n_acc), dev(L))
    assert ctx.status() == -5
    done = dict(b=[1], path=path)
    for plane in (0, 1):
        if "node" in what:
            fp8.put(codes[0, plane], scales[0, plane], table[0, [1, 1]], np.array([2, 4]), np.swapaxes(tree[0, plane, 0][:, [0, 2]], 0, 1))
        fp8.put(codes[0, plane], scales[0, plane], table[1, [0] * 4], 20 + np.arange(4), np.swapaxes(tree[0, plane, 1][:, :4], 0, 1))
    assert done["b"] == [1]
    _same(d_codes, codes)
    np.testing.assert_array_equal(d_scales.cpu().numpy(), scales)


@pytest.mark.parametrize("what", ["node", "low node", "count", "negative count", "length", "negative length", "block", "low block"])
def test_what_an_append_out_of_range_returns(what):
    """Lengths, and kept values: those of rows that are left out are as they were."""
    rng = np.random.default_rng(10)
    B, N, hkv = 2, 8, 2
    table, L = rng.permutation(4).reshape(2, 2).astype(np.int32), np.array([126, 20], np.int32)
    codes, scales = _garbage(rng, 1, 4, hkv)
    tree = _rows(rng, (1, 2, B, hkv, N, 128))
    path, n_acc = np.tile(np.arange(N, dtype=np.int32), (B, 1)), np.array([5, 4], np.int32)
    kept = np.arange(5)                              # of sequence 0: rows 126 .. 130, from the third on in the second block
    length = 131
    if what == "node": path[0, 3], kept = N, np.array([0, 1, 2, 4])
    if what == "low node": path[0, 1], kept = -1, np.array([0, 2, 3, 4])
    if what == "count": n_acc[0], kept, length = N + 1, kept[:0], 126
    if what == "negative count": n_acc[0], kept, length = -1, kept[:0], 126
    if what == "length": L[0], kept, length = 252, kept[:0], 252
    if what == "negative length": L[0], kept, length = -3, kept[:0], -3
    if what == "block": table[0, 1], kept = 4, kept[:2]
    if what == "low block": table[0, 0], kept = -1, kept[2:]
    d_codes, d_scales = dev(codes), dev(scales)
    ctx = _context(hkv, hkv, max_batch=B, max_nodes=N)
    back = torch.full((1, 2, B, hkv, N, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    for keep in (None, back):                        # (once more changes nothing: the scales have risen, the rows are the same)
        new_len = ctx.kv_append_fp8(d_codes, d_scales, dev(table), b16(tree), dev(path), dev(n_acc), dev(L), rounded=keep)
        assert ctx.status() == -5
        assert new_len.tolist() == [length, 24]
    want = np.full(back.shape, np.nan)
    for plane in (0, 1):
        for b, at in ((0, kept), (1, np.arange(4))):
            pos = L[b] + at
            if len(at):
                v = fp8.put(codes[0, plane], scales[0, plane], table[b, pos // 128], pos % 128, np.swapaxes(tree[0, plane, b][:, path[b, at]], 0, 1))
                want[0, plane, b][:, path[b, at]] = np.swapaxes(v, 0, 1)
    np.testing.assert_array_equal(back.float().cpu().numpy(), want)
    _same(d_codes, codes)
    np.testing.assert_array_equal(d_scales.cpu().numpy(), scales)


@pytest.mark.parametrize("behind,n", [(0, 20), (0, 1), (3, 200), (128, 256)])
def test_append_at_the_end_of_the_longest_table(behind, n):
    """Row numbers next to 2^31: the longest table that is accepted, whose last blocks are the sequence's."""
    rng = np.random.default_rng(9)
    N, hkv, bps, nb = 256, 1, (2 ** 31 - 1) // 128, 4
    L = np.array([bps * 128 - n - behind], np.int32)
    table = np.full((1, bps), -7, np.int32)
    table[0, -nb:] = rng.permutation(nb)
    codes, scales = _garbage(rng, 1, nb, hkv)
    tree = _rows(rng, (1, 2, 1, hkv, N, 128))
    path, n_acc = np.full((1, N), -1, np.int32), np.array([n], np.int32)
    path[0, :n] = np.sort(rng.permutation(N)[:n])
    d_codes, d_scales = dev(codes), dev(scales)
    ctx = _context(hkv, hkv, max_batch=1, max_nodes=N)
    new_len = ctx.kv_append_fp8(d_codes, d_scales, dev(table), b16(tree), dev(path), dev(n_acc), dev(L))
    ctx.check()
    fp8.append(codes, scales, table, tree, path, n_acc, L)
    assert new_len.tolist() == [int(L[0]) + n]
    _same(d_codes, codes)
    np.testing.assert_array_equal(d_scales.cpu().numpy(), scales)


# ---- blocks ------------------------------------------------------------------------------------------------------------------------------


class Pool:
    """The state on the device beside the definition's."""

    def __init__(self, rng, B, bps, nb):
        self.rng, self.B, self.bps, self.nb = rng, B, bps, nb
        self.length = np.zeros(B, np.int32)
        self.state = (rng.integers(-9, -1, (B, bps)).astype(np.int32), np.zeros(B, np.int32), np.zeros(nb, np.int32), rng.permutation(nb).astype(np.int32), nb)
        self.ctx = _context(max_batch=B, n_layers=2)
        self.put()

    def put(self):
        self.d_length = dev(self.length)
        self.d = [dev(np.array([x], np.int32) if i == 4 else x) for i, x in enumerate(self.state)]

    def same(self):
        for x, y in zip(self.d, self.state):
            np.testing.assert_array_equal(x.cpu().numpy().reshape(-1), np.asarray(y).reshape(-1))
        np.testing.assert_array_equal(self.d_length.cpu().numpy(), self.length)

    def plan(self, add):
        got = packed.plan(self.length, add, None, *self.state[:2], *self.state[3:], 100000)
        _, _, _, _, _, t, h, f, n = got
        self.ctx.block_plan(self.d_length, dev(add), self.d[0], self.d[1], self.d[3], self.d[4], 100000)
        assert self.ctx.status() == (0 if got[0] else -5)
        self.state = (t, h, self.state[2], f, n)
        return got[0]

    def fork(self, src, dst):
        src, dst = np.asarray(src, np.int32), np.asarray(dst, np.int32)
        want = fp8.fork(src, dst, self.length, *self.state)
        pairs = self.ctx.block_fork(dev(src), dev(dst), self.d_length, *self.d)
        assert self.ctx.status() == (0 if want else -5)
        if want:
            out, self.length, self.state = want
        np.testing.assert_array_equal(pairs.cpu().numpy(), out if want else np.full((len(src), 2), -1))
        self.same()
        return pairs if want else None

    def drop(self, which):
        which = np.asarray(which, np.int32)
        want = fp8.drop(which, *self.state)
        self.ctx.block_free(dev(which), *self.d)
        assert self.ctx.status() == (0 if want else -5)
        if want:
            self.state = want
        self.same()
        return want is not None

    def compact(self, pairs=None):
        want = fp8.compact(*self.state, max_pairs=None if pairs is None else len(pairs))
        got = self.ctx.block_compact(*self.d, pairs=pairs)
        assert self.ctx.status() == (0 if want else -5)
        if want:
            out, self.state = want
        np.testing.assert_array_equal(got.cpu().numpy(), out if want else -1)
        self.same()
        return got if want else None


@pytest.mark.parametrize("seed,B,bps,nb", [(0, 4, 3, 12), (1, 10, 6, 40), (2, 60, 9, 300), (3, 200, 30, 4000), (4, 1024, 4, 3000), (5, 7, 500, 2000), (6, 3, 2, 1)])
def test_a_servers_life(seed, B, bps, nb):
    """Requests come, grow, are forked and dropped, the pool is compacted: the state is carried from call to call."""
    rng = np.random.default_rng(seed)
    p = Pool(rng, B, bps, nb)
    done = dict(fork=0, drop=0, compact=0)
    for step in range(24):
        held = p.state[1]
        busy, idle = np.flatnonzero(held > 0), np.flatnonzero(held == 0)
        what = rng.choice(["plan", "fork", "drop", "compact", "fork"])
        if what == "plan":
            add = np.where(rng.random(B) < 0.4, rng.integers(0, bps * 128 // 3 + 2, B), 0).astype(np.int32)
            add = np.minimum(add, bps * 128 - p.length).astype(np.int32)
            if p.plan(add):
                p.length = (p.length + rng.integers(0, add + 1)).astype(np.int32)
                p.d_length = dev(p.length)
        if what == "fork" and len(busy) and len(idle):
            n = int(rng.integers(1, min(len(idle), 40) + 1))
            done["fork"] += p.fork(rng.choice(busy, n), rng.permutation(idle)[:n]) is not None
        if what == "drop":
            which = (rng.random(B) < 0.4).astype(np.int32) * int(rng.integers(1, 3))
            done["drop"] += p.drop(which)
            p.length = np.where(which != 0, 0, p.length).astype(np.int32)
            p.d_length = dev(p.length)
        if what == "compact":
            done["compact"] += p.compact() is not None
    assert done["drop"] + done["compact"] > 0
    p.drop(np.ones(B))
    assert p.state[4] == nb and not p.state[2].any()


@pytest.mark.parametrize("what", ["source", "target", "twice", "chain", "held", "blocks", "rows", "table", "stack", "popped"])
def test_a_fork_that_does_not_fit_changes_nothing(what):
    p = Pool(np.random.default_rng(1), 5, 3, 9)
    p.plan(np.array([300, 128, 0, 0, 0], np.int32))
    p.length = np.array([300, 128, 0, 0, 0], np.int32)
    t, h, s, f, n = p.state
    src, dst = [0, 1], [2, 3]
    if what == "source": src = [0, 5]
    if what == "target": dst = [2, -1]
    if what == "twice": dst = [2, 2]
    if what == "chain": src = [0, 2]
    if what == "held": dst = [1, 3]
    if what == "blocks": n = 0
    if what == "rows": p.length[1] = 129
    if what == "table": t[0, 1] = 9
    if what == "stack": n = 10
    if what == "popped": f[n - 1] = -3
    p.state = (t, h, s, f, n)
    p.put()
    assert p.fork(src, dst) is None


@pytest.mark.parametrize("what", ["table", "held", "count", "stack", "n_free"])
def test_a_drop_that_does_not_fit_changes_nothing(what):
    p = Pool(np.random.default_rng(2), 4, 3, 9)
    p.plan(np.array([300, 128, 0, 0], np.int32))
    p.length = np.array([300, 128, 0, 0], np.int32)
    p.put()
    p.fork([0], [2])
    t, h, s, f, n = p.state
    if what == "table": t[0, 1] = -1
    if what == "held": h[1] = 4
    if what == "count": s[t[0, 0]] = 0             # two hold it
    if what == "stack": n = 9
    if what == "n_free": n = -1
    p.state = (t, h, s, f, n)
    p.put()
    assert not p.drop([1, 1, 1, 0])


@pytest.mark.parametrize("what", ["table", "held", "both", "twice", "n_free", "pairs"])
def test_a_compaction_that_does_not_fit_changes_nothing(what):
    p = Pool(np.random.default_rng(3), 3, 4, 12)
    p.state = p.state[:3] + (np.arange(12, dtype=np.int32), 12)          # (the highest ones are taken first)
    p.put()
    p.plan(np.array([300, 128, 200], np.int32))
    t, h, s, f, n = p.state
    if what == "table": t[0, 1] = 12
    if what == "held": h[1] = -1
    if what == "both": f[0] = t[1, 0]
    if what == "twice": f[0] = f[1]
    if what == "n_free": n = 13
    p.state = (t, h, s, f, n)
    p.put()
    assert p.compact(torch.zeros((2, 2), dtype=torch.int32, device="cuda") if what == "pairs" else None) is None


def test_blocks_beside_the_stack_and_the_tables_stay_where_they_are():
    """Numbers that neither a sequence holds nor the stack has are nobody's: a compaction does not touch them."""
    p = Pool(np.random.default_rng(4), 2, 4, 70)
    t, h, s, f, n = p.state
    f[:5] = [3, 64, 40, 10, 69]
    t[0, :3], t[1, :2] = [66, 33, 68], [66, 5]
    h[:] = [3, 2]
    s[66] = 1
    p.state = (t, h, s, f, 5)
    p.put()
    pairs = p.compact().cpu().numpy()
    assert pairs[:3].tolist() == [[66, 3], [68, 10], [-1, -1]]


def _spread(p, n):
    """n blocks of the whole range, the first and the last among them, held by the sequences one behind the other (the first block by the last sequence too), the others
    free in any order."""
    t, h, s, f, _ = p.state
    blocks = np.concatenate([[0, p.nb - 1], 1 + p.rng.choice(p.nb - 2, n - 2, replace=False)]).astype(np.int32)
    for b in range(p.B):
        mine = blocks[b::p.B]
        h[b] = len(mine)
        t[b, :h[b]] = mine
    t[-1, h[-1]], s[blocks[0]] = blocks[0], 1
    h[-1] += 1
    rest = np.setdiff1d(np.arange(p.nb, dtype=np.int32), blocks)
    f[:len(rest)] = p.rng.permutation(rest)
    p.state = (t, h, s, f, len(rest))
    p.put()


@pytest.mark.parametrize("nb", [32768, 32769, 130400, 131072, 391200, 393216, 400000, 2 ** 19])
def test_pools_of_any_size_up_to_the_largest(nb):
    """More words of bits than threads, and shared memory around what a kernel has without asking and far beyond."""
    p = Pool(np.random.default_rng(nb), 9, 60, nb)
    _spread(p, 400)
    assert p.fork([8], [8]) is None                  # (a target that is a source changes nothing)
    assert p.compact() is not None
    assert p.drop([0, 1, 0, 1, 1, 0, 0, 1, 1])
    assert p.compact() is not None
    assert p.drop([1] * 9) and p.state[4] == nb


def test_pools_of_two_sizes_from_two_threads():
    """Calls of two host threads, a context each: neither takes from the other what its pool needs of shared memory."""
    pools, wrong = [Pool(np.random.default_rng(i), 9, 60, nb) for i, nb in enumerate((2 ** 19, 140000))], []
    for p in pools:
        _spread(p, 300)
    torch.cuda.synchronize()

    def work(p, i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                pairs = torch.zeros((p.nb // 2, 2), dtype=torch.int32, device="cuda")
                for _ in range(300):
                    p.ctx.block_compact(*p.d, pairs=pairs)
                    p.ctx.block_free(dev(np.zeros(9, np.int32)), *p.d)
                torch.cuda.current_stream().synchronize()
            p.ctx.check()
        except Exception as e:                       # noqa: BLE001
            wrong.append((i, e))

    threads = [threading.Thread(target=work, args=(p, i)) for i, p in enumerate(pools)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong
    for p in pools:
        _, p.state = fp8.compact(*p.state)
        p.same()


@pytest.mark.parametrize("dtype,tail", [(torch.uint8, (2, 128, 128)), (torch.bfloat16, (2, 128, 128)), (torch.float32, (1, 4)), (torch.uint8, (3, 128, 8)), (torch.int32, (5000,))])
def test_copies(dtype, tail):
    rng = np.random.default_rng(6)
    nb = 300
    pool = torch.randint(0, 255, (2, 2, nb) + tail, dtype=torch.int32, device="cuda").to(dtype)
    second = torch.randn((2, 2, nb, 12), device="cuda")
    order = rng.permutation(nb)
    for n in (0, 1, 7, 130):
        pairs = np.full((n + 3, 2), -1, np.int32)
        pairs[:n] = order[:2 * n].reshape(n, 2)
        pairs[:n, 0] = pairs[rng.integers(0, max(1, n), n), 0]          # (a block may be read several times)
        src, dst = torch.from_numpy(pairs[:n, 0]).long().cuda(), torch.from_numpy(pairs[:n, 1]).long().cuda()
        ctx = _context(n_layers=2)
        for two in (False, True):
            want, want2 = pool.clone(), second.clone()
            want[:, :, dst] = want[:, :, src]
            want2[:, :, dst] = want2[:, :, src]
            x, y = pool.clone(), second.clone()
            ctx.block_copy((x, y) if two else x, dev(pairs))
            ctx.check()
            assert torch.equal(x, want) and torch.equal(y, want2 if two else second)


def test_copies_of_numbers_outside_the_pool_are_reported_and_left_out():
    pool = torch.arange(2 * 2 * 9 * 8, dtype=torch.float32, device="cuda").view(2, 2, 9, 8)
    want = pool.clone()
    want[:, :, 5] = want[:, :, 2]
    ctx = _context(n_layers=2)
    ctx.block_copy(pool, dev(np.array([[9, 1], [2, 5], [0, -2], [-1, 3], [-1, -1], [-1, -1]], np.int32)))
    assert ctx.status() == -5
    assert torch.equal(pool, want)


def test_a_pool_beyond_32_bits_of_bytes():
    nb = 80000
    pool = torch.zeros((1, 2, nb, 2, 128, 128), dtype=torch.uint8, device="cuda")
    pool[:, :, nb - 3] = torch.randint(0, 256, (1, 2, 2, 128, 128), dtype=torch.uint8, device="cuda")
    ctx = _context()
    ctx.block_copy(pool, dev(np.array([[nb - 3, nb - 1], [-1, -1]], np.int32)))
    ctx.check()
    assert torch.equal(pool[:, :, nb - 1], pool[:, :, nb - 3]) and pool[:, :, nb - 1].any()


def test_two_answers_to_one_prompt():
    """A prompt is written, forked, both sequences take a step of their own tree and keep its rows, the pool is compacted, the first is
    dropped: what the second attends to stays what it was at every point."""
    rng = np.random.default_rng(20)
    B, hq, hkv, layers, N, bps, nb = 4, 8, 2, 2, 12, 4, 14
    width = (hq + 2 * hkv) * 128
    ctx = binding.Context(hq, hkv, 16, 512, max_nodes=N, n_layers=layers, max_batch=B)
    codes, scales = ctx.new_fp8_cache(nb)
    zeros = lambda *s: dev(np.zeros(s, np.int32))  # noqa: E731
    table, held, shares = zeros(B, bps), zeros(B), zeros(nb)
    free, n_free = dev(np.arange(nb, dtype=np.int32)), dev(np.array([nb], np.int32))
    length = zeros(B)
    prompt = np.array([0, 173, 40, 0], np.int32)
    row_start, slots, row_seq, row_pos = ctx.block_plan(length, dev(prompt), table, held, free, n_free, 256)
    positions = row_pos.clamp(min=0)[None, :, None].repeat(1, 1, 3).contiguous()
    for layer in range(layers):
        _, k, v = ctx.rope_qkv(b16(synth.normal_bf16(rng, (1, 256, width))), 1e4, positions=positions)
        ctx.kv_write_fp8(k, v, slots, codes, scales, layer=layer, k_rounded=k, v_rounded=v)
    length.copy_(dev(prompt))
    # the kept rows of the last layer stand in the cache where the table says
    got = fp8.rows_of(codes.cpu().numpy(), scales.cpu().numpy(), layers - 1, 0, table.cpu().numpy()[2], 1, 40)[0]
    np.testing.assert_array_equal(got, k[0, 1, 173:213].double().cpu().numpy())
    pairs = ctx.block_fork(dev(np.array([1, 1], np.int32)), dev(np.array([0, 3], np.int32)), length, table, held, shares, free, n_free)
    ctx.block_copy((codes, scales), pairs)
    ctx.check()
    np.testing.assert_array_equal(length.cpu().numpy(), [173, 173, 40, 173])
    parent = np.stack([np.array([-1] + [int(rng.integers(0, i)) for i in range(1, N)], np.int32) for _ in range(B)])
    bits = binding.bf16_bits

    def step():
        ctx.block_plan(length, dev(np.where(prompt + length.cpu().numpy() > 0, N, 0).astype(np.int32)), table, held, free, n_free, B * N)
        tree = torch.empty((layers, 2, B, hkv, N, 128), dtype=torch.bfloat16, device="cuda")
        start = length[:, None].repeat(1, 3).contiguous()
        for layer in range(layers):
            q, _, _ = ctx.rope_qkv(b16(synth.normal_bf16(rng, (B, N, width))), 1e4, (20, 20, 24), parent=dev(parent), start=start, k=tree[layer, 0], v=tree[layer, 1])
            out = ctx.tree_attn_fp8(q, codes, scales, table, tree[layer, 0], tree[layer, 1], dev(parent), length, layer=layer)
            ctx.check()
            want = fp8.tree_attn(bits(q), codes.cpu().numpy(), scales.cpu().numpy(), layer, table.cpu().numpy(), bits(tree[layer, 0]), bits(tree[layer, 1]), parent,
                                 length.cpu().numpy())[0]
            err = np.abs(out.float().cpu().numpy() - want)
            assert np.linalg.norm(err) <= 4e-3 * np.linalg.norm(want)
        return tree, q, out

    def rows(b):
        c, s, t, L = codes.cpu().numpy(), scales.cpu().numpy(), table.cpu().numpy()[b], int(length[b])
        return [fp8.rows_of(c, s, x, plane, t, h, L)[0] for x in range(layers) for plane in (0, 1) for h in range(hkv)]

    np.testing.assert_array_equal(rows(0), rows(1))
    for _ in range(2):
        before = rows(3)
        tree, q, out = step()
        paths, n_acc = np.full((B, N), -1, np.int32), np.zeros(B, np.int32)
        for b in (0, 1, 2):                        # (3 keeps nothing)
            way = synth.random_path(rng, parent[b])
            paths[b, :len(way)], n_acc[b] = way, len(way)
        length = ctx.kv_append_fp8(codes, scales, table, tree, dev(paths), dev(n_acc), length)
        ctx.check()
        np.testing.assert_array_equal(rows(3), before)
    again = lambda: ctx.tree_attn_fp8(q, codes, scales, table, tree[1, 0], tree[1, 1], dev(parent), length, layer=1)  # noqa: E731
    first = again()
    before = [rows(b) for b in range(B)]
    pairs = ctx.block_compact(table, held, shares, free, n_free)
    ctx.block_copy((codes, scales), pairs)
    ctx.check()
    assert pairs[0, 0] >= 0 and int(table.max()) < nb - int(n_free)
    for b in range(B):
        np.testing.assert_array_equal(rows(b), before[b])
    assert torch.equal(again(), first)
    ctx.block_free(dev(np.array([0, 1, 0, 0], np.int32)), table, held, shares, free, n_free)
    ctx.check()
    np.testing.assert_array_equal(rows(3), before[3])
    ctx.block_free(dev(np.array([1, 0, 1, 1], np.int32)), table, held, shares, free, n_free)
    ctx.check()
    assert int(n_free) == nb and sorted(free.cpu().tolist()) == list(range(nb)) and not shares.any()


def test_a_captured_cycle_replayed():
    """Fork, copy, append and drop in one graph: a replay does what the call did."""
    rng = np.random.default_rng(21)
    p = Pool(rng, 4, 3, 12)
    p.plan(np.array([200, 0, 0, 0], np.int32))
    p.length = np.array([200, 0, 0, 0], np.int32)
    p.put()
    first = [x.clone() for x in p.d] + [p.d_length.clone()]
    codes, scales = p.ctx.new_fp8_cache(12)
    codes.random_(0, 0x78)
    codes0, scales0 = codes.clone(), scales.clone()
    src, dst, which = dev(np.array([0, 0], np.int32)), dev(np.array([2, 1], np.int32)), dev(np.array([0, 1, 0, 0], np.int32))
    tree = b16(_rows(rng, (2, 2, 4, 2, 5, 128), 0))
    path, count = dev(np.tile(np.array([0, 2, 4] + [-1] * 61, np.int32), (4, 1))), dev(np.array([1, 3, 2, 0], np.int32))
    pairs, new_len = torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")

    def cycle():
        for x, y in zip(p.d + [p.d_length], first):
            x.copy_(y)
        codes.copy_(codes0)
        scales.copy_(scales0)
        p.ctx.block_fork(src, dst, p.d_length, *p.d, pairs=pairs)
        p.ctx.block_copy((codes, scales), pairs)
        p.ctx.kv_append_fp8(codes, scales, p.d[0], tree, path, count, p.d_length, new_len=new_len)
        p.ctx.block_free(which, *p.d)

    cycle()
    p.ctx.check()
    outs = p.d + [p.d_length, codes, scales, pairs, new_len]
    want = [x.clone() for x in outs]
    assert want[-1].tolist() == [201, 203, 202, 0]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cycle()
    for _ in range(3):
        for x in outs:
            x.zero_()
        g.replay()
        assert all(torch.equal(x, y) for x, y in zip(outs, want))
    p.ctx.check()
