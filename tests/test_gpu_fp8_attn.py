"""Attention over the 8-bit cache on the GPU against the 64-bit definition."""
import numpy as np
import pytest
import torch

from oracle import fp8, packed
from paper_2408_15562_b200 import binding, synth
from tests import helpers

pytestmark = pytest.mark.gpu

b16, dev = binding.bf16_tensor, helpers.dev


def fill(codes, scales, table, L, x, plane, layer=0, head=0):
    """Rows x [L][128] (float) of one head to where the table says."""
    pos = np.arange(L)
    bits = synth.f32_to_bf16_bits(np.asarray(x, np.float32))[:, None]
    c, s = codes[layer, plane][:, head:head + 1], scales[layer, plane][:, head:head + 1]
    fp8.put(c, s, table[pos // 128], pos % 128, bits)


class Case:
    def __init__(self, seed, batch, nodes, hq, hkv, lens, tree="random", layers=1, q_size=1.5, spare_blocks=1, bps=None):
        rng = self.rng = np.random.default_rng(seed)
        self.B, self.N, self.hq, self.hkv, self.layers = batch, nodes, hq, hkv, layers
        self.L = np.asarray(lens, np.int32)
        need = (self.L.astype(np.int64) + 127) // 128
        self.bps = bps or max(1, int(need.max()))
        self.nb = int(need.sum()) + spare_blocks
        order, at = rng.permutation(self.nb), 0
        self.table = np.full((batch, self.bps), -5, np.int32)           # entries behind a sequence's end are not looked at
        # e4m3 codes of normal values, scales that differ from group to group
        self.codes = fp8.encode(rng.standard_normal((layers, 2, self.nb, hkv, 128, 128)) * 70)
        self.scales = (2.0 ** rng.integers(-8, -4, (layers, 2, self.nb, hkv, 4))).astype(np.float32)
        live = np.zeros((self.nb, 128), bool)
        for b in range(batch):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
            for i in range(need[b]):
                live[self.table[b, i], :min(128, int(self.L[b]) - 128 * i)] = True
        for x in range(self.nb):                                        # what lies behind the ends may be anything
            self.codes[:, :, x, :, ~live[x]] = 0x7F
            self.scales[:, :, x, :, ~live[x].reshape(4, 32).any(-1)] = np.nan
        self.q = synth.f32_to_bf16_bits((rng.standard_normal((batch, nodes, hq, 128)) * q_size).astype(np.float32))
        self.tk, self.tv = (synth.normal_bf16(rng, (batch, hkv, nodes, 128)) for _ in range(2))
        kinds = dict(chain=lambda: synth.chain_tree(nodes), star=lambda: synth.star_tree(nodes),
                     random=lambda: np.array([-1] + [int(rng.integers(max(0, i - 20), i)) for i in range(1, nodes)], np.int32))
        self.parent = np.stack([kinds[tree]() for _ in range(batch)]).astype(np.int32)

    def context(self, **kw):
        kw.setdefault("max_nodes", self.N)
        return binding.Context(self.hq, self.hkv, 16, 512, n_layers=self.layers, max_batch=self.B, **kw)

    def arguments(self):
        return [b16(self.q), dev(self.codes), dev(self.scales), dev(self.table), b16(self.tk), b16(self.tv), dev(self.parent), dev(self.L)]

    def check(self, out, layer=0, scale=None):
        """Weights are rounded once (bf16, 2^-8 of each, at the coarsest) under sums of 32 bits; scores are sums of 256 products in 32 bits, each off by at
        most 256 * 2^-24 of the sum of their magnitudes, twice that with the reference's own, and the weight by as much: 2^-15.  A query element is
        off by at most 2^-18 of its row's largest, and a score by that much of `far`, twice with the reference's own.  Small weights are whole multiples of
        2^-16 where 2^11 stands for the largest (score and scale of V together): each may be off by 2^-28 of that.  The result is rounded once to bf16."""
        want, of = fp8.tree_attn(self.q, self.codes, self.scales, layer, self.table, self.tk, self.tv, self.parent, self.L, scale)
        got = out.float().cpu().numpy().astype(np.float64)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        ok = np.isfinite(want)
        with np.errstate(invalid="ignore"):
            before = of["mass"] * (2.0 ** -8 + 2.0 ** -12 + 2.0 ** -15 * of["size"][..., None] + np.expm1(2.0 ** -17 * of["far"])[..., None]) + 2.0 ** -28 * of["small"]
            bound = np.abs(want) * 2.0 ** -8 + before * (1 + 2.0 ** -8)
            err = np.abs(got - want)
        assert (err[ok] <= bound[ok]).all(), (float((err - bound)[ok].max()), float(err[ok].max()))
        if ok.all() and want.size >= 4096:         # (and all together, far nearer than the worst of each)
            assert np.linalg.norm(err) <= 4e-3 * np.linalg.norm(want), float(np.linalg.norm(err) / np.linalg.norm(want))


def _run(case, layer=0, **kw):
    ctx = case.context(**kw)
    out = ctx.tree_attn_fp8(*case.arguments(), layer=layer)
    ctx.check()
    return out


@pytest.mark.parametrize("L", [0, 1, 31, 32, 33, 127, 128, 129, 500, 1024])
@pytest.mark.parametrize("heads", [(1, 1), (8, 2), (7, 1), (16, 1)])
def test_single_token(L, heads):
    case = Case(L, 1, 1, *heads, [L])
    case.check(_run(case))


@pytest.mark.parametrize("nodes", [1, 2, 3, 5, 8, 9, 16, 17, 33, 60, 64, 65, 100, 129, 255, 256])
@pytest.mark.parametrize("tree", ["random", "chain", "star"])
def test_trees(nodes, tree):
    case = Case(nodes, 2, nodes, 8, 2, [300, 77], tree)
    case.check(_run(case))


@pytest.mark.parametrize("heads", [(1, 1), (3, 3), (28, 4), (12, 1), (40, 2), (130, 1)])
@pytest.mark.parametrize("nodes", [1, 7, 26, 40])
def test_head_layouts(heads, nodes):
    case = Case(nodes, 3, nodes, *heads, [0, 129, 260])
    case.check(_run(case))


@pytest.mark.parametrize("nodes", [1, 4, 7, 60])
def test_ragged_batch(nodes):
    lens = [0, 1, 2000, 128, 127, 900, 31, 333, 64, 1500, 5, 700, 0, 96, 260, 1111]
    case = Case(7, len(lens), nodes, 8, 2, lens)
    case.check(_run(case))


@pytest.mark.parametrize("nodes", [1, 30])
def test_many_sequences(nodes):
    rng = np.random.default_rng(5)
    case = Case(8, 300, nodes, 2, 1, rng.integers(0, 200, 300))
    case.check(_run(case))


@pytest.mark.parametrize("nodes,heads,batch", [(40, (8, 2), 40), (60, (8, 2), 20), (70, (6, 2), 33), (100, (2, 2), 70), (33, (8, 1), 90), (256, (2, 1), 9), (1, (16, 4), 70), (6, (8, 2), 50)])
def test_lists_that_are_cut_wherever_it_falls(nodes, heads, batch):
    """Ragged runs, many shorter than a part and what a beginning counts, with one row tile, two, and one and two of them in turn."""
    rng = np.random.default_rng(nodes)
    lens = np.where(rng.random(batch) < 0.3, rng.integers(0, 3, batch), rng.integers(0, 700, batch))
    case = Case(nodes, batch, nodes, *heads, lens)
    case.check(_run(case))


@pytest.mark.parametrize("nodes,heads", [(1, (4, 1)), (8, (4, 1)), (60, (4, 1)), (256, (1, 1))])
def test_one_long_sequence_over_all_sms(nodes, heads):
    case = Case(9, 1, nodes, *heads, [30000])
    case.check(_run(case))


def test_layers_and_scale():
    case = Case(10, 2, 6, 8, 2, [200, 64], layers=3)
    args, ctx = case.arguments(), case.context(softmax_scale=0.03)
    for layer in range(3):
        case.check(ctx.tree_attn_fp8(*args, layer=layer), layer, np.float32(0.03).astype(np.float64))
    ctx.check()


@pytest.mark.parametrize("nodes", [1, 60])
def test_queries_of_any_magnitude(nodes):
    """Rows of zeros, of tiny and of huge elements, and rows whose elements lie far apart."""
    case = Case(11, 1, nodes, 8, 2, [400])
    x = packed.bf16(case.q)
    x[:, :, 0] = 0
    x[:, :, 1] *= 2.0 ** -120
    x[:, :, 2] *= 8
    x[:, :, 3, ::2] *= 2.0 ** -30
    x[:, :, 4] *= 2.0 ** 3
    x[:, :, 5, 1:] *= 2.0 ** -9
    case.q = synth.f32_to_bf16_bits(x.astype(np.float32))
    case.check(_run(case))


@pytest.mark.parametrize("nodes", [1, 60, 200])
def test_scores_that_rise_along_the_cache(nodes):
    """The running maximum moves at every unit, the last key outweighs all before it."""
    case = Case(12, 1, nodes, 4, 1, [700])
    fill(case.codes, case.scales, case.table[0], 700, np.linspace(0.01, 3.0, 700)[:, None] * np.ones(128), 0)
    case.q = synth.f32_to_bf16_bits(np.abs(packed.bf16(case.q)).astype(np.float32))
    case.check(_run(case))


@pytest.mark.parametrize("nodes,last", [(1, 13), (4, 13), (5, 9), (60, 9)])
def test_how_exact_small_elements_of_a_query_are(nodes, last):
    """Of each row one element next to 2^-e beside the largest, 1, against a key whose two elements cancel but for the small one's last bit (2^-7 of it, or -2^-8): the scores are 2 and
    -1 from sums of 2 * 2^8, the other cached key's is 0, the values 1 and -1, the result tanh(score / 2).  An element is exact from 2^-9 of the largest on, up to 16 rows a kv head 2^-13 (`last`); a smaller one (at e = last
    the ones below a power of two are) may be off by 2^-17, or 2^-21, of the largest: by 2^-(last + 8), the score by that times 256 * 2^(e + 4) / 2^4, 2^(e - last), and the result by
    half of that.  Otherwise: the score's sum to 2^-15 of the magnitudes, 2^-6, half of that in the result; the weights to 2^-9 and the result to 2^-9."""
    for e in range(4, last + 2):
        case = Case(e, 1, nodes, 8, 2, [2])
        rng, blk = case.rng, int(case.table[0, 0])
        kv = np.zeros((2, 2, 128))
        kv[0, 0] = 256.0
        kv[0, 0, 0] = -2.0 ** (8 - e)
        kv[1] = [[1.0], [-1.0]]
        case.codes[0, :, blk, :, :2] = fp8.encode(kv)[:, None]
        case.scales[0, 0, blk, :, 0], case.scales[0, 1, blk, :, 0] = 2.0 ** (e + 4), 1.0
        below = rng.random((1, nodes, 8)) < 0.5
        x = np.zeros(case.q.shape)
        np.put_along_axis(x, rng.integers(1, 128, below.shape)[..., None], np.where(below, 1 - 2.0 ** -8, 1 + 2.0 ** -7)[..., None] * 2.0 ** -e, -1)
        x[..., 0] = 1.0
        case.q = synth.f32_to_bf16_bits(x.astype(np.float32))
        np.testing.assert_array_equal(packed.bf16(case.q), x)
        t = np.zeros(case.tk.shape, np.float32)
        t[..., 0] = -2.0 ** 12                         # (the tree's keys have no weight)
        case.tk = synth.f32_to_bf16_bits(t)
        want = np.tanh(np.where(below, -0.5, 1.0))[..., None]
        err = np.abs(_run(case, softmax_scale=2.0 ** -4).float().cpu().numpy() - want).max(-1)
        small = np.where(below, 1 - 2.0 ** -8, 1.0) * 2.0 ** -e < 2.0 ** -last
        assert (err <= 2.0 ** -7 + 2.0 ** -8 + np.where(small, 2.0 ** (e - last) / 2, 0.0)).all(), (e, err.max())


@pytest.mark.parametrize("nodes", [1, 60])
@pytest.mark.parametrize("what", ["k", "v", "own", "v falls"])
def test_scales_far_apart_and_a_callers_own(nodes, what):
    """Groups whose scales differ by up to 2^128 (the keys' such that the scores stay moderate), and scales that are no powers of two."""
    case = Case(21, 2, nodes, 8, 2, [700, 130])
    rng = case.rng
    live = np.isfinite(case.scales)
    if what == "own":
        s = rng.uniform(0.002, 0.05, case.scales.shape)
    elif what == "v falls":                        # the first keys' values are the largest ones by far
        s = case.scales.copy()
        for b, L in enumerate(case.L):
            for i in range((int(L) + 127) // 128):
                s[:, 1, case.table[b, i]] = 2.0 ** (40 - 20 * i - 4 * np.arange(4)).astype(np.float64)
    else:
        s = case.scales.copy()
        s[:, "kv".index(what)] = 2.0 ** (rng.integers(-64, -3, s[:, 0].shape) if what == "k" else rng.integers(-64, 65, s[:, 0].shape)).astype(np.float64)
    case.scales = np.where(live, s, np.nan).astype(np.float32)
    case.check(_run(case))


@pytest.mark.parametrize("nodes", [1, 5, 20, 60])
def test_scores_of_nothing_beside_scores_beyond_the_range(nodes):
    """Keys of zeros score 0 whatever the queries' and scales' sizes; the others' scores are -infinity here."""
    case = Case(26, 1, nodes, 4, 1, [300])
    rng, x = case.rng, np.zeros(case.q.shape, np.float32)
    x[..., 0], x[..., 5] = 2.0 ** 100, -2.0 ** 90
    case.q = synth.f32_to_bf16_bits(x)
    zero = rng.permutation(300)[:7]
    k = np.zeros((300, 128))
    k[:, 0] = -1.0 - rng.random(300)
    k[zero] = 0
    pos = np.arange(300)
    case.codes[0, 0, case.table[0, pos // 128], 0, pos % 128] = fp8.encode(k)
    case.scales[0, 0] = np.where(np.isnan(case.scales[0, 0]), np.nan, np.float32(2.0 ** 60))
    case.tk[:] = 0
    want = fp8.tree_attn(case.q, case.codes, case.scales, 0, case.table, case.tk, case.tv, case.parent, case.L)[0]
    got = _run(case).float().cpu().numpy()
    assert np.isfinite(want).all() and np.abs(got - want).max() <= 2.0 ** -7 * np.abs(want).max()


@pytest.mark.parametrize("nodes,heads", [(1, (4, 1)), (5, (8, 2)), (20, (4, 1)), (60, (8, 2)), (1, (16, 16))])
@pytest.mark.parametrize("L", [64, 256, 700, 5000])
@pytest.mark.parametrize("what", ["up", "down", "mixed", "in turn"])
def test_values_scales_at_both_ends_of_the_range(nodes, heads, L, what):
    """V's scales of 2^-64 and 2^64, where all keys weigh alike: those with tiny values have their share of the sum of the weights, whichever come first and whichever part takes them."""
    case = Case(25, 2, nodes, *heads, [L, 0])
    groups = (L + 31) // 32
    exp = dict(up=np.where(np.arange(groups) < groups // 2, -64, 64), down=np.where(np.arange(groups) < groups // 2, 64, -64),
               mixed=case.rng.choice([-64, 64], groups), **{"in turn": np.where(np.arange(groups) // 4 % 2, 64, -64)})[what]
    for g in range(groups):
        case.scales[0, 1, case.table[0, g // 4], :, g % 4] = 2.0 ** float(exp[g])
    case.codes[:, 0, case.table[0, :(L + 127) // 128]] = 0
    case.tk[:] = 0
    case.check(_run(case))
    # the tiny values' keys weigh e^-2 of the others: times their scale 2^-131 of the largest
    case.q[:] = 0
    case.q[..., 0] = 0x3F80
    for g in np.flatnonzero(exp < 0):
        case.codes[0, 0, case.table[0, g // 4], :, 32 * (g % 4):32 * (g % 4) + 32, 0] = fp8.encode(np.array(-2.0))
        case.scales[0, 0, case.table[0, g // 4], :, g % 4] = 1.0
    case.check(_run(case, softmax_scale=1.0), scale=1.0)


@pytest.mark.parametrize("own", [0.0, -1.0, 1e-30, float("nan"), 1e30, float("inf")])
@pytest.mark.parametrize("nodes", [1, 20])
def test_a_write_leaves_what_a_scale_outside_the_range_stands_for(nodes, own):
    """A begun group with a scale of no use: the attention takes the nearer end, and so does a write of further rows (here of tiny ones)."""
    case = Case(24, 1, nodes, 4, 2, [37])
    blk = int(case.table[0, 0])
    case.scales[0, 1, blk, :, 1] = own
    args, ctx = case.arguments(), case.context()
    first = ctx.tree_attn_fp8(*args)
    x = b16(synth.f32_to_bf16_bits((case.rng.standard_normal((2, 2, 3, 128)) * 2.0 ** -70).astype(np.float32)))
    ctx.kv_write_fp8(x[0], x[1], dev(blk * 128 + 37 + np.arange(3)), args[1], args[2])
    again = ctx.tree_attn_fp8(*args)
    ctx.check()
    assert torch.equal(again, first)
    assert (args[2][0, 1, blk, :, 1] == 2.0 ** (64 if own > 1 else -64)).all()


@pytest.mark.parametrize("nodes", [1, 60])
def test_one_heavy_key_and_many_light_ones(nodes):
    """One key with half of the weight, 20000 others with the rest: weights of 2^-15 of the largest, all alike, whose roundings add up."""
    L = 20000
    case = Case(22, 1, nodes, 1, 1, [L])
    k = np.zeros((L, 128))
    k[:, 0] = -1.0
    k[17, 0] = np.log(L)
    fill(case.codes, case.scales, case.table[0], L, k, 0)
    x = np.zeros(case.q.shape, np.float32)
    x[..., 0] = 11.25
    case.q = synth.f32_to_bf16_bits(x)
    case.tk[:] = synth.f32_to_bf16_bits(np.full(case.tk.shape, -0.5, np.float32))
    case.check(_run(case))


@pytest.mark.parametrize("what", ["tree v nan", "tree v inf", "tree k nan", "tree k inf", "cache k", "cache v", "q"])
@pytest.mark.parametrize("nodes,group", [(1, 4), (7, 2), (7, 4), (60, 4), (130, 1)])
def test_values_that_are_no_numbers_reach_only_those_who_see_them(what, nodes, group):
    case = Case(13, 2, nodes, 2 * group, 2, [150, 40])
    if what == "tree v nan": case.tv[0, 1, nodes // 2, 5] = 0x7FC0
    if what == "tree v inf": case.tv[0, 1, nodes // 2, 77] = 0xFF80; case.tv[1, 0, nodes - 1, 0] = 0x7F80
    if what == "tree k nan": case.tk[0, 1, nodes // 2, 5] = 0x7FC0
    if what == "tree k inf": case.tk[0, 1, nodes // 2, :] = 0x7F80
    if what == "cache k": case.codes[0, 0, case.table[0, 1], 1, 3, 20] = 0xFF
    if what == "cache v": case.codes[0, 1, case.table[0, 1], 1, 3, 20] = 0x7F
    if what == "q": case.q[1, nodes // 3, 1, 9] = 0x7FC0; case.q[1, nodes // 3, 0, 9] = 0x7F80
    out = _run(case)
    want = fp8.tree_attn(case.q, case.codes, case.scales, 0, case.table, case.tk, case.tv, case.parent, case.L)[0]
    # a row with an infinity or a NaN in V makes all of the outputs of those who see it NaN, and so does one in K or Q
    bad = ~np.isfinite(want).all(-1)
    got = out.float().cpu().numpy()
    if what == "cache v":                          # (an element of the cache: only its column)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    else:
        np.testing.assert_array_equal(np.isnan(got).all(-1), bad)
        np.testing.assert_array_equal(np.isnan(got).any(-1), bad)
    good = np.isfinite(want) if what == "cache v" else np.broadcast_to(~bad[..., None], want.shape)
    assert np.abs(got - want)[good].max() <= 3e-2


@pytest.mark.parametrize("nodes,heads,batch", [(40, (8, 2), 700), (17, (1, 1), 1500), (128, (2, 2), 500), (150, (2, 1), 400), (200, (2, 2), 400), (40, (56, 28), 30), (130, (4, 2), 300), (160, (4, 2), 200)])
def test_trees_without_a_cache_one_behind_the_other(nodes, heads, batch):
    """Nothing but trees, many to a part, with infinities and NaN in V of every third: the flags of V's rows are in one of two places in turn, and each
    tree's nodes have those of their own tree, in every one of several calls."""
    case = Case(31, batch, nodes, *heads, np.zeros(batch, np.int32), bps=1)
    rng = case.rng
    odd = np.zeros((batch, nodes), bool)
    for b in range(0, batch, 3):
        for i in rng.integers(0, nodes, 2):
            case.tv[b, :, i, rng.integers(0, 128)] = rng.choice([0x7F80, 0xFF80, 0x7FC0])
            odd[b, i] = True
    sees = odd.copy()                                # a node that is odd, or has an ancestor that is (parents come first)
    for i in range(1, nodes):
        sees[:, i] |= sees[np.arange(batch), case.parent[:, i]]
    assert sees.any() and not sees.all()
    ctx, args = case.context(), case.arguments()
    want = np.broadcast_to(sees[:, :, None, None], (batch, nodes, case.hq, 128))
    for _ in range(5):
        out = ctx.tree_attn_fp8(*args)
        ctx.check()
        np.testing.assert_array_equal(torch.isnan(out).cpu().numpy(), want)


@pytest.mark.parametrize("nodes", [1, 4, 60])
def test_tree_rows_of_the_largest_values(nodes):
    case = Case(23, 2, nodes, 8, 2, [150, 0])
    case.tv[:, :, :, ::2] = 0x7F7F                 # bf16's largest
    want = fp8.tree_attn(case.q, case.codes, case.scales, 0, case.table, case.tk, case.tv, case.parent, case.L)[0]
    got = _run(case).float().cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= np.abs(want) * 2.0 ** -6 + 3e-2).all()       # (weights to 2^-8 twice, their sum, the result)


def test_what_is_out_of_range_is_reported_and_stays_in_bounds():
    for nodes in (1, 5, 60):
        case = Case(14, 2, nodes, 4, 2, [300, 200])
        ctx = case.context()
        for bad in ("long", "negative", "block", "low block"):
            args = case.arguments()
            if bad == "long": args[7] = dev(np.array([300, case.bps * 128 + 1], np.int32))
            if bad == "negative": args[7] = dev(np.array([-1, 200], np.int32))
            if bad == "block": args[3] = dev(np.where(np.arange(case.bps) == 1, case.nb, np.maximum(case.table, 0)).astype(np.int32))
            if bad == "low block": args[3] = dev(np.where(np.arange(case.bps) == 0, -1, np.maximum(case.table, 0)).astype(np.int32))
            if bad == "long": args[3] = dev(np.maximum(case.table, 0))
            ctx.tree_attn_fp8(*args)
            assert ctx.status() == -5, bad
        if nodes > 1:
            for parent in (0, 1, 3):
                args = case.arguments()
                args[6][0, 1 if parent else 0] = parent
                ctx.tree_attn_fp8(*args)
                assert ctx.status() == -8
        ctx.tree_attn_fp8(*case.arguments())
        ctx.check()


@pytest.mark.parametrize("nodes", [1, 60])
def test_captured_replayed_and_on_another_stream(nodes):
    case = Case(15, 3, nodes, 8, 2, [900, 64, 333])
    args, ctx = case.arguments(), case.context()
    want = ctx.tree_attn_fp8(*args)
    graphs = []
    for _ in range(2):
        g, out = torch.cuda.CUDAGraph(), torch.empty_like(want)
        with torch.cuda.graph(g):
            ctx.tree_attn_fp8(*args, out=out)
        graphs.append((g, out))
    for _ in range(3):
        for g, out in graphs:
            out.fill_(9)
            g.replay()
        assert all(torch.equal(out, want) for _, out in graphs)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    out, ws = torch.full_like(want, 9), torch.empty(ctx.tree_attn_fp8_workspace_bytes(), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    ctx.tree_attn_fp8(*args, out=out, workspace=ws, stream=st)
    st.synchronize()
    assert torch.equal(out, want)
    # other lengths in the same buffers, as a replayed step meets them
    args[7].copy_(dev(np.array([100, 0, 300], np.int32)))
    graphs[0][0].replay()
    case.L = np.array([100, 0, 300], np.int32)
    case.check(graphs[0][1])
    ctx.check()


@pytest.mark.parametrize("nodes", [1, 60])
def test_two_calls_at_once_with_a_workspace_each(nodes):
    cases = [Case(18, 4, nodes, 8, 2, [3001, 64, 333, 1500]), Case(19, 4, nodes, 8, 2, [0, 2500, 700, 129])]
    ctx = cases[0].context()
    args = [c.arguments() for c in cases]
    want = [ctx.tree_attn_fp8(*a) for a in args]
    size = ctx.tree_attn_fp8_workspace_bytes()
    own = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in cases]
    out = [[torch.full_like(w, 9) for _ in range(8)] for w in want]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for i in range(8):
        for a, o, ws, st in zip(args, out, own, streams):
            ctx.tree_attn_fp8(*a, out=o[i], workspace=ws, stream=st)
    torch.cuda.synchronize()
    ctx.check()
    assert all(torch.equal(x, w) for o, w in zip(out, want) for x in o)


@pytest.mark.parametrize("nodes", [1, 5, 60])
def test_results_do_not_depend_on_the_run(nodes):
    case = Case(16, 5, nodes, 8, 2, [900, 64, 333, 0, 1700])
    args, ctx = case.arguments(), case.context()
    first = ctx.tree_attn_fp8(*args)
    for _ in range(20):
        assert torch.equal(ctx.tree_attn_fp8(*args), first)


@pytest.mark.parametrize("nodes", [3, 40])
def test_a_cache_beyond_32_bits_of_bytes(nodes):
    """Blocks whose codes lie more than 2^32 bytes into the array: 4.9 GB a plane, of which the call reads the ends."""
    nb, hkv = 150000, 2
    codes = torch.zeros((1, 2, nb, hkv, 128, 128), dtype=torch.uint8, device="cuda")
    scales = torch.ones((1, 2, nb, hkv, 4), dtype=torch.float32, device="cuda")
    case = Case(17, 2, nodes, 4, 2, [256, 140], spare_blocks=0)
    where = np.array([nb - 1, 3, nb - 7, 131072], np.int32)
    at = torch.from_numpy(where).long().cuda()
    codes[:, :, at] = dev(case.codes)
    scales[:, :, at] = dev(case.scales)
    args = case.arguments()
    args[1], args[2], args[3] = codes, scales, dev(where[case.table])
    ctx = case.context()
    out = ctx.tree_attn_fp8(*args)
    ctx.check()
    case.check(out)
