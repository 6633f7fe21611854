"""Attention over the 4-bit cache on the GPU against the 64-bit definition."""
import numpy as np
import pytest
import torch

from oracle import packed
from paper_2408_15562_b200 import binding, synth
from tests import helpers

pytestmark = pytest.mark.gpu

b16, dev = binding.bf16_tensor, helpers.dev


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
        self.scales = np.full((layers, 2, self.nb, hkv, 128, 8), 0x7F, np.uint8)      # and rows there may be anything
        self.codes = rng.integers(0, 256, (layers, 2, self.nb, hkv, 128, 64), np.uint8)
        for b in range(batch):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
            for i in range(need[b]):
                rows = min(128, int(self.L[b]) - 128 * i)
                x = synth.normal_bf16(rng, (layers, 2, hkv, rows, 128))
                c, s, _ = packed.quantise(x)
                self.codes[:, :, self.table[b, i], :, :rows], self.scales[:, :, self.table[b, i], :, :rows] = c, s
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
        """Weights are rounded once (bf16, 2^-8 of each) under sums of 32 bits; scores are sums of 128 products in 32 bits, each off by at
        most 128 * 2^-24 of the sum of their magnitudes, and the weight by as much (and twice that with the reference's own);
        the result, which is that far from the right one, is rounded once to bf16.  Weights as fp16 are whole multiples of 2^-24 where
        they are small, and 2^7 stands for the weight of the largest score but the lag, so that each may be off by 2^-32 of the sum besides."""
        want, mass, size, all_v = packed.tree_attn(self.q, self.codes, self.scales, layer, self.table, self.tk, self.tv, self.parent, self.L, scale)
        got = out.float().cpu().numpy().astype(np.float64)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        ok = np.isfinite(want)
        before = mass * (2.0 ** -8 + 2.0 ** -12 + 2.0 ** -15 * size[..., None]) + 2.0 ** -32 * all_v
        bound = np.abs(want) * 2.0 ** -8 + before * (1 + 2.0 ** -8)
        err = np.abs(got - want)
        assert (err[ok] <= bound[ok]).all(), (float((err - bound)[ok].max()), float(err[ok].max()))
        if ok.all() and want.size >= 4096:         # (and all together, far nearer than the worst of each)
            assert np.linalg.norm(err) <= 4e-3 * np.linalg.norm(want), float(np.linalg.norm(err) / np.linalg.norm(want))


def _run(case, layer=0, **kw):
    ctx = case.context(**kw)
    out = ctx.tree_attn_packed(*case.arguments(), layer=layer)
    ctx.check()
    return out


@pytest.mark.parametrize("L", [0, 1, 31, 32, 33, 127, 128, 129, 500, 1024])
@pytest.mark.parametrize("heads", [(1, 1), (8, 2), (7, 1), (16, 1)])
def test_single_token(L, heads):
    case = Case(L, 1, 1, *heads, [L])
    case.check(_run(case))


@pytest.mark.parametrize("nodes", [1, 2, 3, 5, 16, 17, 33, 60, 64, 65, 100, 129, 255, 256])
@pytest.mark.parametrize("tree", ["random", "chain", "star"])
def test_trees(nodes, tree):
    case = Case(nodes, 2, nodes, 8, 2, [300, 77], tree)
    case.check(_run(case))


@pytest.mark.parametrize("heads", [(1, 1), (3, 3), (28, 4), (12, 1), (40, 2), (130, 1)])
@pytest.mark.parametrize("nodes", [1, 7, 40])
def test_head_layouts(heads, nodes):
    case = Case(nodes, 3, nodes, *heads, [0, 129, 260])
    case.check(_run(case))


@pytest.mark.parametrize("nodes", [1, 4, 60])
def test_ragged_batch(nodes):
    lens = [0, 1, 2000, 128, 127, 900, 31, 333, 64, 1500, 5, 700, 0, 96, 260, 1111]
    case = Case(7, len(lens), nodes, 8, 2, lens)
    case.check(_run(case))


@pytest.mark.parametrize("nodes", [1, 30])
def test_many_sequences(nodes):
    rng = np.random.default_rng(5)
    case = Case(8, 300, nodes, 2, 1, rng.integers(0, 200, 300))
    case.check(_run(case))


@pytest.mark.parametrize("nodes,heads", [(1, (4, 1)), (60, (4, 1)), (256, (1, 1))])
def test_one_long_sequence_over_all_sms(nodes, heads):
    case = Case(9, 1, nodes, *heads, [6000])
    case.check(_run(case))


def test_layers_and_scale():
    case = Case(10, 2, 6, 8, 2, [200, 64], layers=3)
    args, ctx = case.arguments(), case.context(softmax_scale=0.03)
    for layer in range(3):
        case.check(ctx.tree_attn_packed(*args, layer=layer), layer, np.float32(0.03).astype(np.float64))
    ctx.check()


@pytest.mark.parametrize("nodes", [1, 60])
def test_queries_of_any_magnitude(nodes):
    """Rows of zeros, of tiny and of huge elements, and rows whose elements lie far apart; one key far ahead of the others."""
    case = Case(11, 1, nodes, 8, 2, [400])
    x = packed.bf16(case.q)
    x[:, :, 0] = 0
    x[:, :, 1] *= 2.0 ** -120
    x[:, :, 2] *= 8
    x[:, :, 3, ::2] *= 2.0 ** -30
    x[:, :, 4] *= 2.0 ** 3
    case.q = synth.f32_to_bf16_bits(x.astype(np.float32))
    case.check(_run(case))


@pytest.mark.parametrize("nodes", [1, 60, 200])
def test_scores_that_rise_along_the_cache(nodes):
    """The running maximum moves at every unit, the last key outweighs all before it."""
    case = Case(12, 1, nodes, 4, 1, [700])
    k = np.linspace(0.01, 3.0, 700)[:, None] * np.ones(128)
    for i in range(6):
        rows = min(128, 700 - 128 * i)
        c, s, _ = packed.quantise(synth.f32_to_bf16_bits(k[128 * i:128 * i + rows].astype(np.float32)))
        case.codes[0, 0, case.table[0, i], 0, :rows], case.scales[0, 0, case.table[0, i], 0, :rows] = c, s
    case.q = synth.f32_to_bf16_bits(np.abs(packed.bf16(case.q)).astype(np.float32))
    case.check(_run(case))


@pytest.mark.parametrize("what", ["tree v nan", "tree v inf", "tree k nan", "tree k inf", "cache", "q"])
@pytest.mark.parametrize("nodes,group", [(7, 2), (60, 4), (130, 1)])
def test_values_that_are_no_numbers_reach_only_those_who_see_them(what, nodes, group):
    case = Case(13, 2, nodes, 2 * group, 2, [150, 40])
    if what == "tree v nan": case.tv[0, 1, nodes // 2, 5] = 0x7FC0
    if what == "tree v inf": case.tv[0, 1, nodes // 2, 77] = 0xFF80; case.tv[1, 0, nodes - 1, 0] = 0x7F80
    if what == "tree k nan": case.tk[0, 1, nodes // 2, 5] = 0x7FC0
    if what == "tree k inf": case.tk[0, 1, nodes // 2, :] = 0x7F80
    if what == "cache": case.scales[0, 1, case.table[0, 1], 1, 3, 2] = 0x7F
    if what == "q": case.q[1, nodes // 3, 1, 9] = 0x7FC0; case.q[1, nodes // 3, 0, 9] = 0x7F80
    out = _run(case)
    want = packed.tree_attn(case.q, case.codes, case.scales, 0, case.table, case.tk, case.tv, case.parent, case.L)[0]
    # a row with an infinity or a NaN in V makes all of the outputs of those who see it NaN, and so does one in K or Q
    bad = ~np.isfinite(want).all(-1)
    got = out.float().cpu().numpy()
    if what == "cache":                            # (an element of the cache: only the columns of its block)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    else:
        np.testing.assert_array_equal(np.isnan(got).all(-1), bad)
        np.testing.assert_array_equal(np.isnan(got).any(-1), bad)
    good = np.isfinite(want) if what == "cache" else np.broadcast_to(~bad[..., None], want.shape)
    assert np.abs(got - want)[good].max() <= 3e-2


def test_what_is_out_of_range_is_reported_and_stays_in_bounds():
    for nodes in (1, 60):
        case = Case(14, 2, nodes, 4, 2, [300, 200])
        ctx = case.context()
        for bad in ("long", "negative", "block", "low block"):
            args = case.arguments()
            if bad == "long": args[7] = dev(np.array([300, case.bps * 128 + 1], np.int32))
            if bad == "negative": args[7] = dev(np.array([-1, 200], np.int32))
            if bad == "block": args[3] = dev(np.where(np.arange(case.bps) == 1, case.nb, np.maximum(case.table, 0)).astype(np.int32))
            if bad == "low block": args[3] = dev(np.where(np.arange(case.bps) == 0, -1, np.maximum(case.table, 0)).astype(np.int32))
            if bad == "long": args[3] = dev(np.maximum(case.table, 0))
            ctx.tree_attn_packed(*args)
            assert ctx.status() == -5, bad
        if nodes > 1:
            for parent in (0, 1, 3):
                args = case.arguments()
                args[6][0, 1 if parent else 0] = parent
                ctx.tree_attn_packed(*args)
                assert ctx.status() == (-8 if parent != 0 else -8)
        ctx.tree_attn_packed(*case.arguments())
        ctx.check()


@pytest.mark.parametrize("nodes", [1, 60])
def test_captured_replayed_and_on_another_stream(nodes):
    case = Case(15, 3, nodes, 8, 2, [900, 64, 333])
    args, ctx = case.arguments(), case.context()
    want = ctx.tree_attn_packed(*args)
    graphs = []
    for _ in range(2):
        g, out = torch.cuda.CUDAGraph(), torch.empty_like(want)
        with torch.cuda.graph(g):
            ctx.tree_attn_packed(*args, out=out)
        graphs.append((g, out))
    for _ in range(3):
        for g, out in graphs:
            out.fill_(9)
            g.replay()
        assert all(torch.equal(out, want) for _, out in graphs)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    out, ws = torch.full_like(want, 9), torch.empty(ctx.tree_attn_packed_workspace_bytes(nodes, 3), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    ctx.tree_attn_packed(*args, out=out, workspace=ws, stream=st)
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
    cases = [Case(18, 4, nodes, 8, 2, [3000, 64, 333, 1500]), Case(19, 4, nodes, 8, 2, [0, 2500, 700, 129])]
    ctx = cases[0].context()
    args = [c.arguments() for c in cases]
    want = [ctx.tree_attn_packed(*a) for a in args]
    size = ctx.tree_attn_packed_workspace_bytes(nodes, 4)
    own = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in cases]
    out = [[torch.full_like(w, 9) for _ in range(8)] for w in want]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for i in range(8):
        for a, o, ws, st in zip(args, out, own, streams):
            ctx.tree_attn_packed(*a, out=o[i], workspace=ws, stream=st)
    torch.cuda.synchronize()
    ctx.check()
    assert all(torch.equal(x, w) for o, w in zip(out, want) for x in o)


@pytest.mark.parametrize("nodes", [1, 60])
def test_results_do_not_depend_on_the_run(nodes):
    case = Case(16, 5, nodes, 8, 2, [900, 64, 333, 0, 1700])
    args, ctx = case.arguments(), case.context()
    first = ctx.tree_attn_packed(*args)
    for _ in range(20):
        assert torch.equal(ctx.tree_attn_packed(*args), first)


def test_a_cache_beyond_32_bits_of_bytes():
    """Blocks whose codes lie more than 2^32 bytes into the array: 3.3 GB a plane, of which the call reads the ends."""
    nb, hkv = 200000, 2
    codes = torch.zeros((1, 2, nb, hkv, 128, 64), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((1, 2, nb, hkv, 128, 8), dtype=torch.uint8, device="cuda")
    case = Case(17, 2, 3, 4, 2, [256, 140], spare_blocks=0)
    where = np.array([nb - 1, 3, nb - 7, 131072], np.int32)
    at = torch.from_numpy(where).long().cuda()
    codes[:, :, at] = dev(case.codes)
    scales[:, :, at] = dev(case.scales)
    args = case.arguments()
    args[1], args[2], args[3] = codes, scales, dev(where[case.table])
    ctx = case.context()
    out = ctx.tree_attn_packed(*args)
    ctx.check()
    case.check(out)


def test_from_the_product_to_the_cache_and_back():
    """Two requests as a server takes them: blocks for the prompts, rotary positions, the prompts' rows into the 4-bit cache, then steps of a
    tree each: rotary positions by depth, attention over the cache, the accepted rows of every layer behind the prefix."""
    rng = np.random.default_rng(20)
    B, hq, hkv, layers, N, bps = 2, 8, 2, 2, 12, 4
    width = (hq + 2 * hkv) * 128
    ctx = binding.Context(hq, hkv, 16, 512, max_nodes=N, n_layers=layers, max_batch=B)
    nb = B * bps
    codes, scales = ctx.new_packed_cache(nb)
    table, held = dev(np.zeros((B, bps), np.int32)), dev(np.zeros(B, np.int32))
    free, n_free = dev(rng.permutation(nb).astype(np.int32)), dev(np.array([nb], np.int32))
    length = dev(np.zeros(B, np.int32))
    prompt = np.array([130, 77], np.int32)
    row_start, slots, row_seq, row_pos = ctx.block_plan(length, dev(prompt), table, held, free, n_free, 256)
    qkv = b16(synth.normal_bf16(rng, (1, 256, width)))
    positions = row_pos.clamp(min=0)[None, :, None].repeat(1, 1, 3).contiguous()
    kept = []
    for layer in range(layers):
        _, k, v = ctx.rope_qkv(qkv, 1e4, positions=positions)
        ctx.kv_write_packed(k, v, slots, codes, scales, layer=layer, k_rounded=k, v_rounded=v)
        kept.append((k, v))
    length = dev(prompt)
    ctx.check()
    # the kept rows of sequence 1 stand in the cache where the table says
    got = packed.rows_of(codes.cpu().numpy(), scales.cpu().numpy(), 1, 0, table.cpu().numpy()[1], 1, 77)
    np.testing.assert_array_equal(got, kept[1][0][0, 1, 130:207].double().cpu().numpy())
    for step in range(3):
        parent = np.stack([np.array([-1] + [int(rng.integers(0, i)) for i in range(1, N)], np.int32) for _ in range(B)])
        ctx.block_plan(length, dev(np.full(B, N, np.int32)), table, held, free, n_free, B * N)
        tree = torch.empty((layers, 2, B, hkv, N, 128), dtype=torch.bfloat16, device="cuda")
        start = length[:, None].repeat(1, 3).contiguous()
        for layer in range(layers):
            product = synth.normal_bf16(rng, (B, N, width))
            q, _, _ = ctx.rope_qkv(b16(product), 1e4, (20, 20, 24), parent=dev(parent), start=start, k=tree[layer, 0], v=tree[layer, 1])
            out = ctx.tree_attn_packed(q, codes, scales, table, tree[layer, 0], tree[layer, 1], dev(parent), length, layer=layer)
            ctx.check()
            bits = binding.bf16_bits
            want = packed.tree_attn(bits(q), codes.cpu().numpy(), scales.cpu().numpy(), layer, table.cpu().numpy(), bits(tree[layer, 0]),
                                          bits(tree[layer, 1]), parent, length.cpu().numpy())[0]
            err = np.abs(out.float().cpu().numpy() - want)
            assert np.linalg.norm(err) <= 4e-3 * np.linalg.norm(want)
        paths, n_acc = np.full((B, N), -1, np.int32), np.zeros(B, np.int32)
        for b in range(B):
            p = synth.random_path(rng, parent[b])
            paths[b, :len(p)], n_acc[b] = p, len(p)
        length = ctx.kv_append_packed(codes, scales, table, tree, dev(paths), dev(n_acc), length)
        ctx.check()


def test_a_captured_step_replayed_is_the_step_called():
    """Blocks, rotary positions, attention and append of a step in one graph, replayed over growing lengths."""
    rng = np.random.default_rng(21)
    B, hq, hkv, N, bps = 3, 8, 2, 9, 6
    width, nb = (hq + 2 * hkv) * 128, 3 * 6
    parent = dev(np.stack([np.array([-1] + [int(rng.integers(0, i)) for i in range(1, N)], np.int32) for _ in range(B)]))
    path = np.full((B, N), -1, np.int32)
    count = np.array([2, 1, 0], np.int32)
    p = parent.cpu().numpy()
    for b in range(B):
        path[b, 0] = 0
        path[b, 1] = int(np.flatnonzero(p[b] == 0)[0])
    path, count, free = dev(path), dev(count), rng.permutation(nb).astype(np.int32)
    qkv = b16(synth.normal_bf16(rng, (B, N, width)))

    class State:
        def __init__(self):
            self.ctx = binding.Context(hq, hkv, 16, 512, max_nodes=N, max_batch=B)
            self.codes, self.scales = self.ctx.new_packed_cache(nb)
            self.table, self.held = dev(np.zeros((B, bps), np.int32)), dev(np.zeros(B, np.int32))
            self.free, self.n_free, self.length = dev(free), dev(np.array([nb], np.int32)), dev(np.array([0, 126, 255], np.int32))
            self.add, self.tree = dev(np.full(B, N, np.int32)), torch.empty((1, 2, B, hkv, N, 128), dtype=torch.bfloat16, device="cuda")

        def step(self):
            plan = self.ctx.block_plan(self.length, self.add, self.table, self.held, self.free, self.n_free, B * N)
            start = self.length[:, None].repeat(1, 3)
            q, _, _ = self.ctx.rope_qkv(qkv, 1e4, (20, 20, 24), parent=parent, start=start, k=self.tree[0, 0], v=self.tree[0, 1])
            out = self.ctx.tree_attn_packed(q, self.codes, self.scales, self.table, self.tree[0, 0], self.tree[0, 1], parent, self.length)
            self.length.copy_(self.ctx.kv_append_packed(self.codes, self.scales, self.table, self.tree, path, count, self.length))
            return (out,) + plan

    called, replayed = State(), State()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = replayed.step()
    for _ in range(5):
        want = called.step()
        graph.replay()
        for name in ("codes", "scales", "table", "held", "free", "n_free", "length"):
            assert torch.equal(getattr(called, name), getattr(replayed, name)), name
        assert all(torch.equal(x, y) for x, y in zip(want, out))
    called.ctx.check()
    replayed.ctx.check()
    assert replayed.length.tolist() == [10, 131, 255]


@pytest.mark.parametrize("nodes", [8, 15, 16, 17, 24, 25, 32, 33])
@pytest.mark.parametrize("tree", ["random", "chain"])
@pytest.mark.parametrize("batch", [2, 170])
def test_around_the_line_between_the_kernels(nodes, tree, batch):
    """Up to 32 rows a kv head, and from 25 nodes on by the number of runs: on both sides of it."""
    case = Case(22, batch, nodes, 2, 2, [(37 * b) % 140 for b in range(batch)], tree=tree)
    case.check(_run(case))
