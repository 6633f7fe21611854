"""Rotary rows, the block plan, and the writes into the 4-bit cache on the GPU against the 64-bit definitions: whole numbers and kept
values bit for bit, rotated rows to the rounding of their type."""
import numpy as np
import pytest
import torch

from oracle import packed
from paper_2408_15562_b200 import binding, synth
from tests import helpers

pytestmark = pytest.mark.gpu

b16, dev = binding.bf16_tensor, helpers.dev


def _context(hq=4, hkv=2, **kw):
    kw.setdefault("max_nodes", 64)
    return binding.Context(hq, hkv, 16, 512, **kw)


def _near(got, want, size):
    """One rounding to bf16, half a step of it (2^-8) at most, behind products and sums of 32 bits: each of the two products, the sum, and
    the sines (taken to 2^-22, of an angle to 2^-24 of a turn, 2 pi 2^-24 < 2^-21) give less than 2^-20 of |x1| + |x2|."""
    err = np.abs(got.float().cpu().numpy().astype(np.float64) - want)
    bound = np.abs(want) * 2.0 ** -8 * (1 + 2.0 ** -8) + size * 2.0 ** -20
    assert (err <= bound).all(), float((err - bound).max())


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("batch,nodes,sections,heads,pad", [(1, 1, (64, 0, 0), (1, 1), 0), (2, 60, (16, 24, 24), (8, 2), 64), (3, 17, (0, 0, 64), (5, 5), 8),
                                                            (2, 256, (1, 62, 1), (12, 1), 0), (1, 33, (0, 64, 0), (7, 7), 136)])
def test_rope_of_trees(batch, nodes, sections, heads, pad, adjacent):
    rng = np.random.default_rng(nodes)
    hq, hkv = heads
    width = (hq + 2 * hkv) * 128
    wide = synth.normal_bf16(rng, (batch, nodes, width + pad))
    parents = [synth.chain_tree(nodes), synth.star_tree(nodes)] + [np.array([-1] + [int(rng.integers(0, i)) for i in range(1, nodes)], np.int32)]
    parent = np.stack([parents[b % 3] for b in range(batch)]).astype(np.int32)
    start = rng.integers(-1000, 2 ** 31 - 300, (batch, 3)).astype(np.int32)
    ctx = _context(hq, hkv, max_nodes=nodes, max_batch=batch)
    q, k, v = ctx.rope_qkv(b16(wide)[..., :width], 500000.0, sections, parent=dev(parent), start=dev(start), adjacent=adjacent)
    ctx.check()
    pos = start[:, None].astype(np.int64) + packed.depths(parent)[..., None]
    rq, rk, rv, sq, sk = packed.rope(np.ascontiguousarray(wide[..., :width]), hq, hkv, pos, 500000.0, sections, adjacent)
    _near(q, rq, sq)
    _near(k, rk, sk)
    np.testing.assert_array_equal(v.float().cpu().numpy(), rv)


@pytest.mark.parametrize("batch,rows", [(1, 1), (1, 300), (2, 129), (1, 2000)])
def test_rope_of_rows_with_given_positions(batch, rows):
    rng = np.random.default_rng(rows)
    qkv = synth.normal_bf16(rng, (batch, rows, 8 * 128))
    pos = rng.integers(0, [100, 10 ** 5, 4 * 10 ** 6], (batch, rows, 3)).astype(np.int32)
    ctx = _context(max_batch=2)
    for adjacent in (False, True):
        q, k, v = ctx.rope_qkv(b16(qkv), 10000.0, (20, 20, 24), positions=dev(pos), adjacent=adjacent)
        ctx.check()
        rq, rk, rv, sq, sk = packed.rope(qkv, 4, 2, pos, 10000.0, (20, 20, 24), adjacent)
        _near(q, rq, sq)
        _near(k, rk, sk)
        np.testing.assert_array_equal(v.float().cpu().numpy(), rv)


def test_rope_reports_a_tree_that_is_none():
    ctx = _context()
    qkv = b16(synth.normal_bf16(np.random.default_rng(0), (1, 4, 8 * 128)))
    for parent in ([[0, 0, 1, 2]], [[-1, 1, 0, 0]], [[-1, 0, 5, 0]], [[-1, 0, -1, 0]]):
        ctx.rope_qkv(qkv, 1e4, parent=dev(np.array(parent, np.int32)), start=dev(np.zeros((1, 3), np.int32)))
        assert ctx.status() == -8


def _state(rng, B, bps, spare, held):
    order = rng.permutation(int(held.sum()) + spare).astype(np.int32)
    table, at = rng.integers(-9, -1, (B, bps)).astype(np.int32), 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    free = np.full(len(order), -7, np.int32)
    free[:spare] = order[at:]
    return table, free


@pytest.mark.parametrize("seed,B,bps,most,rows", [(0, 1, 3, 100, 500), (1, 5, 7, 300, 1500), (2, 16, 40, 11, 200), (3, 33, 4, 130, 9000), (4, 1024, 3, 30, 40000), (5, 200, 24, 700, 150000)])
def test_plans_one_after_the_other(seed, B, bps, most, rows):
    """Steps of a server: rows are added, some sequences finish and give their blocks back; the state is carried from plan to plan."""
    rng = np.random.default_rng(seed)
    ctx = _context(max_batch=B)
    held = np.zeros(B, np.int32)
    table, free = _state(rng, B, bps, B * bps, held)
    n = B * bps
    length = np.zeros(B, np.int32)
    d_table, d_held, d_free, d_n = dev(table), dev(held), dev(free), dev(np.array([n], np.int32))
    refused = 0
    for step in range(8):
        drop = (rng.random(B) < 0.3).astype(np.int32) if step % 3 else None
        if drop is not None:
            length = np.where(drop != 0, 0, length).astype(np.int32)
        add = rng.integers(0, most + 1, B).astype(np.int32)
        if step != 5:                                                    # (once it may not fit)
            add = np.minimum(add, bps * 128 - length).astype(np.int32)
        want = packed.plan(length, add, drop, table, held, free, n, rows)
        got = ctx.block_plan(dev(length), dev(add), d_table, d_held, d_free, d_n, rows, drop=None if drop is None else dev(drop))
        assert ctx.status() == (0 if want[0] else -5)
        for x, y in zip(got, want[1:5]):
            np.testing.assert_array_equal(x.cpu().numpy(), y)
        fits, _, _, _, _, table, held, free, n = want
        for x, y in ((d_table, table), (d_held, held), (d_free, free), (d_n, [n])):
            np.testing.assert_array_equal(x.cpu().numpy(), y)
        refused += not fits
        if fits:                                                         # (not every row that there is room for is kept)
            length = (length + rng.integers(0, add + 1)).astype(np.int32)
    assert refused < 6


@pytest.mark.parametrize("what", ["length", "add", "held", "n_free", "rows", "blocks", "table", "stack"])
def test_a_plan_that_does_not_fit_changes_nothing(what):
    length, add, held, n = np.array([130, 5], np.int32), np.array([200, 6], np.int32), np.array([2, 1], np.int32), 4
    drop, rows, bps = None, 300, 3
    table, free = _state(np.random.default_rng(0), 2, bps, n, held)
    if what == "length": length[1] = -1
    if what == "add": add[0] = -2
    if what == "held": held[1] = 4
    if what == "n_free": n = 8
    if what == "rows": rows = 205
    if what == "blocks": n = 0
    if what == "table": add[0] = 255
    if what == "stack": drop, n = np.array([1, 1], np.int32), 5
    ctx = _context(max_batch=2)
    d = [dev(table), dev(held), dev(free), dev(np.array([n], np.int32))]
    got = ctx.block_plan(dev(length), dev(add), *d, rows, drop=None if drop is None else dev(drop))
    assert ctx.status() == -5
    assert not packed.plan(length, add, drop, table, held, free, n, rows)[0]
    assert not got[0].any() and all((x == -1).all() for x in got[1:])
    for x, y in zip(d, (table, held, free, [n])):
        np.testing.assert_array_equal(x.cpu().numpy(), y)


def _rows(rng, *shape):
    """Rows with everything that the types can go wrong at: several magnitudes, zeros, ties, infinities and NaN."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-12, 14, shape[:-1] + (8,)).repeat(16, -1).astype(float))
    kind = rng.integers(0, 12, shape[:-1] + (8,)).repeat(16, -1)
    x = np.where(kind == 0, 0.0, x)
    ties = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -6.0, -0.25, -0.0], shape)
    x = np.where(kind == 1, ties * np.exp2(rng.integers(-3, 3, shape[:-1] + (1,)).astype(float)), x)
    x = np.where(kind == 2, x * 1e-30, x)
    x = np.where(kind == 3, x * 1e30, x)
    bits = synth.f32_to_bf16_bits(x.astype(np.float32))
    odd = rng.random(shape) < 0.002
    return np.where(odd, rng.choice(np.array([0x7F80, 0xFF80, 0x7FC0, 0xFFFF], np.uint16), shape), bits).astype(np.uint16)


def _cache(rng, layers, nb, hkv):
    return (rng.integers(0, 256, (layers, 2, nb, hkv, 128, 64), np.uint8), rng.integers(0, 256, (layers, 2, nb, hkv, 128, 8), np.uint8))


def _same_values(got, want):
    got = got.float().cpu().numpy().astype(np.float64)
    np.testing.assert_array_equal(got, want)
    ok = ~np.isnan(want)
    np.testing.assert_array_equal(np.signbit(got[ok]), np.signbit(want[ok]))


@pytest.mark.parametrize("rows,hkv,layers,skip", [(1, 1, 1, False), (7, 2, 2, False), (130, 8, 1, True), (1001, 3, 3, True)])
@pytest.mark.parametrize("rounded", ["none", "own", "in place"])
def test_write_by_slots(rows, hkv, layers, skip, rounded):
    rng = np.random.default_rng(rows)
    nb = rows // 128 + 3
    k, v = _rows(rng, hkv, rows, 128), _rows(rng, hkv, rows, 128)
    slots = rng.permutation(nb * 128)[:rows].astype(np.int64)
    if skip:
        slots[rng.random(rows) < 0.3] = -1
    codes, scales = _cache(rng, layers, nb, hkv)
    ctx = _context(hkv, hkv, n_layers=layers)
    dk, dv, dc, ds = b16(k), b16(v), dev(codes), dev(scales)
    rk, rv = {"none": (None, None), "own": (torch.full_like(dk, 7.0), torch.full_like(dv, 7.0)), "in place": (dk, dv)}[rounded]
    layer = layers - 1
    ctx.kv_write_packed(dk, dv, dev(slots), dc, ds, layer=layer, k_rounded=rk, v_rounded=rv)
    ctx.check()
    keep = slots >= 0
    blk, off = slots[keep] // 128, slots[keep] % 128
    for plane, x, r in ((0, k, rk), (1, v, rv)):
        c, s, value = packed.quantise(x)
        codes[layer, plane][blk, :, off] = c[:, keep].swapaxes(0, 1)
        scales[layer, plane][blk, :, off] = s[:, keep].swapaxes(0, 1)
        if r is not None:
            old = packed.bf16(x) if rounded == "in place" else np.full(x.shape, 7.0)
            _same_values(r, np.where(keep[None, :, None], value, old))
    np.testing.assert_array_equal(ds.cpu().numpy(), scales)
    np.testing.assert_array_equal(dc.cpu().numpy(), codes)


def test_every_bf16_value_beside_a_given_largest_one():
    """All 65536 elements, each in blocks whose scale another element sets: every tie of every scale's mantissa."""
    every = np.arange(65536, dtype=np.uint32).astype(np.uint16).reshape(-1, 8)
    for top in (6.0, 6.75, 7.5, 8.25, 9.0, 9.75, 10.5, 11.25, 0.03, 2688.0):
        x = np.zeros((8192, 8, 16), np.uint16)
        x[:, :, 0] = synth.f32_to_bf16_bits(np.array([top], np.float32))[0]
        x[:, :, 1] = every
        x = x.reshape(1, 8192, 128)
        ctx = _context(1, 1)
        codes, scales = ctx.new_packed_cache(64)
        r = torch.empty((1, 8192, 128), dtype=torch.bfloat16, device="cuda")
        ctx.kv_write_packed(b16(x), b16(x), torch.arange(8192, device="cuda"), codes, scales, k_rounded=r, v_rounded=torch.empty_like(r))
        ctx.check()
        c, s, value = packed.quantise(x)
        np.testing.assert_array_equal(scales[0, 1].cpu().numpy().reshape(1, 8192, 8), s)
        np.testing.assert_array_equal(codes[0, 0].cpu().numpy().reshape(1, 8192, 64), c)
        _same_values(r, value)


def test_write_leaves_out_slots_outside_the_cache():
    rng = np.random.default_rng(0)
    codes, scales = _cache(rng, 1, 2, 2)
    ctx = _context(2, 2)
    x = _rows(rng, 2, 4, 128)
    for bad in (256, -2, 2 ** 40, -2 ** 62):
        dc, ds = dev(codes), dev(scales)
        ctx.kv_write_packed(b16(x), b16(x), dev(np.array([5, bad, 130, -1], np.int64)), dc, ds)
        assert ctx.status() == -5
        changed = (dc.cpu().numpy() != codes).any(-1)[0]                 # [2][blocks][Hkv][128]
        assert {tuple(i) for i in np.argwhere(changed.any((0, 2)))} <= {(0, 5), (1, 2)}


@pytest.mark.parametrize("layers,batch,nodes,hkv", [(1, 1, 1, 1), (3, 4, 60, 2), (2, 3, 200, 3), (32, 1, 40, 8)])
@pytest.mark.parametrize("rounded", ["none", "own", "in place"])
def test_append_of_the_accepted_path(layers, batch, nodes, hkv, rounded):
    rng = np.random.default_rng(nodes)
    max_nodes = max(nodes, 9)
    paths, n_acc = np.full((batch, max_nodes), -1, np.int32), np.zeros(batch, np.int32)
    for b in range(batch):
        p = synth.random_path(rng, synth.pruned_tree(rng, nodes, min(nodes, 12), 5)) if nodes > 1 else np.array([0])
        p = np.arange(nodes) if b == 1 else p                            # (a chain, accepted as a whole: crosses a block)
        paths[b, :len(p)], n_acc[b] = p, len(p)
    if batch > 2:
        n_acc[2] = 0
    L = rng.integers(0, 400, batch).astype(np.int32)
    L[0] = 127
    bps = (400 + nodes) // 128 + 2
    nb = batch * bps + 2
    table = rng.permutation(nb)[:batch * bps].reshape(batch, bps).astype(np.int32)
    tree = _rows(rng, layers, 2, batch, hkv, nodes, 128)
    codes, scales = _cache(rng, layers, nb, hkv)
    ctx = _context(hkv, hkv, n_layers=layers, max_batch=batch, max_nodes=max_nodes)
    dt, dc, ds = b16(tree), dev(codes), dev(scales)
    r = {"none": None, "own": torch.full_like(dt, 7.0), "in place": dt}[rounded]
    new_len = ctx.kv_append_packed(dc, ds, dev(table), dt, dev(paths), dev(n_acc), dev(L), rounded=r)
    ctx.check()
    c, s, value = packed.quantise(tree)
    want = packed.bf16(tree) if rounded == "in place" else np.full(tree.shape, 7.0)
    for b in range(batch):
        for j in range(n_acc[b]):
            row, node = L[b] + j, paths[b, j]
            codes[:, :, table[b, row // 128], :, row % 128] = c[:, :, b, :, node]
            scales[:, :, table[b, row // 128], :, row % 128] = s[:, :, b, :, node]
            want[:, :, b, :, node] = value[:, :, b, :, node]
    np.testing.assert_array_equal(ds.cpu().numpy(), scales)
    np.testing.assert_array_equal(dc.cpu().numpy(), codes)
    np.testing.assert_array_equal(new_len.cpu().numpy(), L + n_acc)
    if r is not None:
        _same_values(r, want)


@pytest.mark.parametrize("what", ["node", "count", "prefix", "negative", "table"])
def test_append_leaves_out_what_does_not_fit(what):
    rng = np.random.default_rng(3)
    codes, scales = _cache(rng, 1, 4, 2)
    ctx = _context(2, 2, max_batch=2, max_nodes=8)
    paths = np.array([[0, 1, 2, -1, -1, -1, -1, -1]] * 2, np.int32)
    n, L, table = np.array([3, 3], np.int32), np.array([100, 127], np.int32), np.array([[0, 1], [2, 3]], np.int32)
    if what == "node": paths[1, 1] = 8
    if what == "count": n[1] = 9
    if what == "prefix": L[1] = 254
    if what == "negative": L[1] = -1
    if what == "table": table[1] = [7, -3]
    dc, ds = dev(codes), dev(scales)
    ctx.kv_append_packed(dc, ds, dev(table), b16(_rows(rng, 1, 2, 2, 2, 8, 128)), dev(paths), dev(n), dev(L))
    assert ctx.status() == -5
    changed = (dc.cpu().numpy() != codes).any((0, 1, 3, 5))              # [blocks][128]
    assert changed[0, 100:103].any() and not changed[0, :100].any() and not changed[1].any()
    left = {tuple(i) for i in np.argwhere(changed[2:])}
    assert left <= ({(0, 127), (1, 1)} if what == "node" else set())


def test_calls_with_nothing_to_do():
    ctx = binding.Context(8, 2, 16, 512, n_layers=2, max_batch=4)
    codes, scales = ctx.new_packed_cache(3)
    i32, bf = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.bfloat16, device="cuda")
    none = torch.empty((0, 5, 3), **i32)
    q, k, v = ctx.rope_qkv(torch.empty((0, 5, 12 * 128), **bf), 1e4, positions=none)
    assert q.shape == (0, 5, 8, 128) and k.shape == v.shape == (0, 2, 5, 128)
    ctx.kv_write_packed(torch.empty((2, 0, 128), **bf), torch.empty((2, 0, 128), **bf), torch.empty((0,), dtype=torch.int64, device="cuda"), codes, scales)
    new = ctx.kv_append_packed(codes, scales, torch.empty((0, 2), **i32), torch.empty((2, 2, 0, 2, 4, 128), **bf), torch.empty((0, 64), **i32),
                               torch.empty((0,), **i32), torch.empty((0,), **i32))
    assert new.shape == (0,)
    out = ctx.tree_attn_packed(torch.empty((0, 4, 8, 128), **bf), codes, scales, torch.empty((0, 2), **i32), torch.empty((0, 2, 4, 128), **bf),
                               torch.empty((0, 2, 4, 128), **bf), torch.empty((0, 4), **i32), torch.empty((0,), **i32))
    assert out.shape == (0, 4, 8, 128)
    free, n_free = torch.arange(3, **i32), torch.tensor([3], **i32)
    row_start, slots, seq, pos = ctx.block_plan(torch.empty((0,), **i32), torch.empty((0,), **i32), torch.empty((0, 2), **i32), torch.empty((0,), **i32), free, n_free, 5)
    assert row_start.tolist() == [0] and slots.tolist() == seq.tolist() == pos.tolist() == [-1] * 5 and n_free.item() == 3
    table, held = torch.zeros((2, 2), **i32), torch.zeros((2,), **i32)
    row_start, slots, seq, pos = ctx.block_plan(torch.tensor([128, 0], **i32), torch.zeros((2,), **i32), table, held, free, n_free, 0)
    assert row_start.tolist() == [0, 0, 0] and slots.numel() == 0 and held.tolist() == [1, 0] and table.tolist() == [[2, 0], [0, 0]] and n_free.item() == 2
    ctx.check()
    assert not codes.any() and not scales.any()


def test_refused_arguments_leave_the_context_usable():
    ctx = binding.Context(8, 2, 16, 512, n_layers=2, max_batch=4)
    codes, scales = ctx.new_packed_cache(3)
    i32, bf = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.bfloat16, device="cuda")
    qkv, start, parent = torch.zeros((1, 4, 12 * 128), **bf), torch.zeros((1, 3), **i32), torch.arange(-1, 3, **i32)[None].contiguous()
    k, slots = torch.zeros((2, 5, 128), **bf), torch.arange(5, device="cuda")
    for kind, call in [
            (binding.FspadError, lambda: ctx.rope_qkv(qkv, 0.0, start=start, parent=parent)),
            (binding.FspadError, lambda: ctx.rope_qkv(qkv, 1e4, (64, 1, 0), start=start, parent=parent)),
            (binding.FspadError, lambda: ctx.rope_qkv(qkv, 1e4, start=start)),
            (ValueError, lambda: ctx.rope_qkv(qkv[:, :, :-128], 1e4, start=start, parent=parent)),
            (ValueError, lambda: ctx.rope_qkv(qkv, 1e4, start=start.cpu(), parent=parent)),
            (TypeError, lambda: ctx.rope_qkv(qkv, 1e4, start=start.long(), parent=parent)),
            (ValueError, lambda: ctx.rope_qkv(qkv, 1e4, start=start, parent=parent, q=torch.zeros((1, 4, 8, 64), **bf))),
            (binding.FspadError, lambda: ctx.kv_write_packed(k, k, slots, codes, scales, layer=2)),
            (binding.FspadError, lambda: ctx.kv_write_packed(k, k, slots, codes, scales, k_rounded=k)),
            (ValueError, lambda: ctx.kv_write_packed(k, k[:, :4], slots, codes, scales)),
            (ValueError, lambda: ctx.kv_write_packed(k, k, slots, codes, scales[:, :, :2])),
            (ValueError, lambda: ctx.kv_write_packed(k.transpose(0, 1), k, slots, codes, scales))]:
        with pytest.raises(kind):
            call()
    assert not codes.any() and not scales.any()
    ctx.kv_write_packed(k, k, slots, codes, scales, layer=1)
    ctx.check()
