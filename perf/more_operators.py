"""What is measured of the operators around a cache held in 8 bits, and their plain forms.

  write    K/V rows of prompts, or the next row of every sequence of a batch, into the 8-bit cache, by slots
  append   the accepted path's K/V rows of every layer into the 8-bit cache
  attn     tree-masked attention over the 8-bit cache (one node: the single-token step)
  fork     sequences that go on from another one's rows: whole blocks are shared, the last one is copied; some are then dropped again
  compact  the blocks in use moved to the lowest numbers, for sequences that share some of them

The cache: one e4m3 code an element and one scale for 32 rows of a head, in blocks of 128 rows: codes [layers][2][blocks][Hkv][128][128],
scales [layers][2][blocks][Hkv][4].  A written group of 32 rows gets the least power of two with which its largest magnitude is at most 448;
rows that come into a begun group leave its scale as it is or raise it, and its codes are then rounded again.
"""
import math

import numpy as np
import torch

own = False

D = 128
BLOCK = 128
GROUP = 32
E4M3 = torch.float8_e4m3fn
LEAST, MOST = 2.0 ** -64, 2.0 ** 64


def listed():
    return [
        # The next token of 256 sequences: a row each, into begun groups.
        dict(name="write_step_256", kind="write", seqs=256, lo=1, hi=1, hkv=8, layers=1),
        # Prompts of four requests that go on behind what is cached of them, 16 K rows in all.
        dict(name="write_4_prompts", kind="write", seqs=4, lo=2051, hi=6155, hkv=8, layers=1),
        # The accepted path of one sequence in 32 layers.
        dict(name="append_1x32_layers", kind="append", batch=1, nodes=60, width=10, hkv=8, layers=32, lo=2048, hi=2048, acc=5),
        # Accepted paths of a batch of 64 in 16 layers, long ones.
        dict(name="append_64x16_layers", kind="append", batch=64, nodes=60, width=4, hkv=8, layers=16, lo=100, hi=500, acc=24),
        # Single-token step of one sequence: latency.
        dict(name="attn_token_2k", kind="attn", batch=1, nodes=1, width=1, hq=32, hkv=8, lo=2048, hi=2048, layers=1),
        # Single-token step of a ragged batch with long contexts: the cache is streamed.
        dict(name="attn_token_batch32_long", kind="attn", batch=32, nodes=1, width=1, hq=64, hkv=8, lo=4000, hi=32000, layers=1),
        # Verify step of a server's batch: 16 trees of 60 nodes.
        dict(name="attn_tree_batch16", kind="attn", batch=16, nodes=60, width=10, hq=32, hkv=8, lo=512, hi=4096, layers=1),
        # One tree over a long context with eight query heads per KV head: a contraction.
        dict(name="attn_tree_gqa8_32k", kind="attn", batch=1, nodes=60, width=10, hq=64, hkv=8, lo=32700, hi=32700, layers=1),
        # Two answers to one short prompt, in a small target.
        dict(name="fork_2_of_300", kind="fork", prompts=1, fan=2, rows=300, hkv=8, layers=2, bits=8),
        # Sixty-four answers to four prompts of 5000 rows, 32 layers.
        dict(name="fork_64_of_5000", kind="fork", prompts=4, fan=16, rows=5001, hkv=8, layers=32, bits=8),
        # A small pool with a few holes.
        dict(name="compact_48", kind="compact", seqs=5, live=31, free=17, moves=7, shared=3, hkv=8, layers=2, bits=8),
        # A server's pool after many requests have gone, in bf16.
        dict(name="compact_400_bf16", kind="compact", seqs=90, live=260, free=140, moves=88, shared=40, hkv=8, layers=4, bits=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 8), (64, 8), (32, 32), (8, 2), (28, 4), (52, 52), (12, 1), (40, 8), (5, 5), (24, 8)]


def draw(rng):
    kind = rng.choice(["write", "write", "append", "attn", "attn", "attn", "attn", "attn", "attn", "fork", "compact"])
    hq, hkv = rng.choice(HEADS)
    layers = rng.choice([1, 2])
    if kind == "write":
        seqs = _log(rng, 1, 300)
        hi = _log(rng, 1, max(2, 16000 * 8 // max(8, hkv) // seqs))
        return dict(kind=kind, seqs=seqs, lo=rng.randint(1, hi), hi=hi, hkv=hkv, layers=layers)
    if kind == "append":
        hkv = min(hkv, 8)
        batch, nodes = _log(rng, 1, 32), _log(rng, 1, 120)
        return dict(kind=kind, batch=batch, nodes=nodes, width=rng.choice([1, 3, 10]), hkv=hkv, layers=rng.randint(1, max(1, 256 // batch // 4)),
                    lo=0, hi=_log(rng, 2, 500), acc=rng.randint(1, min(nodes, 24)))
    if kind == "fork":
        hkv, layers = min(hkv, 8), _log(rng, 1, 16)
        return dict(kind=kind, prompts=rng.randint(1, 4), fan=_log(rng, 1, 24), rows=_log(rng, 1, 5000), hkv=hkv, layers=layers, bits=rng.choice([8, 16]))
    if kind == "compact":
        hkv, live = min(hkv, 8), _log(rng, 8, 300)
        free = _log(rng, 4, 200)
        return dict(kind=kind, seqs=rng.randint(1, live // 4), live=live, free=free, moves=rng.randint(0, min(free, live)), shared=rng.randint(0, live // 4),
                    hkv=hkv, layers=rng.randint(1, 4), bits=rng.choice([8, 16]))
    nodes = 1 if rng.random() < 0.35 else _log(rng, 2, 256)
    batch = _log(rng, 1, 32)
    rows_flop, row_bytes = 512 * hq * nodes, 2 * 128 * hkv
    most = min(60000000000 // rows_flop, 1100000000 // row_bytes) // batch
    hi = _log(rng, 8, max(16, min(40000, most)))
    return dict(kind=kind, batch=batch, nodes=nodes, width=rng.choice([1, 3, 10, 30]), hq=hq, hkv=hkv, lo=rng.choice([0, hi // 8, hi]), hi=hi, layers=layers)


# ---- inputs ------------------------------------------------------------------------------------------------------------------------------


def _lens(n, lo, hi):
    """n lengths from lo to hi, evenly spread and in no order; both ends occur."""
    at = [lo + int((hi - lo + 1) * math.fmod(0.5 + 0.6180339887498949 * k, 1.0)) for k in range(n)]
    at[0] = hi
    if n > 1:
        at[-1] = lo
    return np.minimum(np.array(at, np.int64), hi)


def _trees(batch, nodes, width, seed):
    """parent[batch][nodes] of trees whose nodes hang on one of the `width` nodes before them."""
    rng = np.random.RandomState(seed % (1 << 31))
    i = np.arange(1, nodes)
    back = 1 + (rng.random_sample((batch, nodes - 1)) * np.minimum(i, width)).astype(np.int64)
    return np.concatenate([np.full((batch, 1), -1, np.int64), i - back], axis=1).astype(np.int32)


def _paths(parent, want):
    """Of every tree the way from the root to a deep node, cut to at most `want` nodes, and how many they are."""
    batch, nodes = parent.shape
    path, n = np.full((batch, nodes), -1, np.int32), np.zeros(batch, np.int32)
    for b in range(batch):
        way, at = [], nodes - 1
        while at >= 0:
            way.append(at)
            at = int(parent[b, at])
        way = way[::-1][:want]
        path[b, :len(way)], n[b] = way, len(way)
    return path, n


def _table(rng, batch, lens, bps, spare):
    """Blocks of `batch` sequences in scrambled order: a table [batch][bps] and the number of blocks."""
    need = (np.asarray(lens) + BLOCK - 1) // BLOCK
    n_blocks = int(need.sum()) + spare
    order = rng.permutation(n_blocks)
    table, at = np.zeros((batch, bps), np.int32), 0
    for b in range(batch):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    return table, n_blocks


def _live(table, lens, n_blocks):
    """Truth values [n_blocks][128]: rows that a sequence holds."""
    live = np.zeros((n_blocks, BLOCK), bool)
    for b, L in enumerate(lens):
        for i in range((int(L) + BLOCK - 1) // BLOCK):
            live[table[b, i], :min(BLOCK, int(L) - i * BLOCK)] = True
    return live


def _cache(g, layers, n_blocks, hkv, live):
    """Codes and scales as normally distributed rows leave them.  Elsewhere is what was there before: codes and scales that are no numbers."""
    lut = (torch.special.ndtri((torch.arange(4096, dtype=torch.float64) + 0.5) / 4096) * 70).to(E4M3).view(torch.uint8).cuda()
    shape = (layers, 2, n_blocks, hkv, BLOCK)
    codes = lut[torch.randint(0, 4096, shape + (D,), generator=g, device="cuda", dtype=torch.int32)]
    scales = torch.exp2(torch.randint(-7, -4, shape[:-1] + (BLOCK // GROUP,), generator=g, device="cuda").float())
    if live is not None:
        live = torch.from_numpy(live).cuda()
        codes.masked_fill_(~live[None, None, :, None, :, None], 0x7F)
        scales.masked_fill_(~live.view(-1, BLOCK // GROUP, GROUP).any(-1)[None, None, :, None], math.nan)
    return codes, scales


def _rows(g, *shape):
    """bf16 K/V rows: normal values, a few channels far larger than the others, some rows too."""
    x = torch.randn(shape, generator=g, device="cuda")
    boost = torch.ones(D, device="cuda")
    boost[3::41] = 6.0
    return (x * boost * torch.exp2(torch.randint(-1, 2, shape[:-1] + (1,), generator=g, device="cuda").float())).to(torch.bfloat16)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        s["ctx"] = _context(case)
    return s


def _inputs(case, seed):
    g, rng, kind = _gen(seed), np.random.RandomState(seed % (1 << 31)), case["kind"]
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    s, hkv, layers = dict(case=case), case["hkv"], case["layers"]
    if kind == "write":
        S = case["seqs"]
        add, lens = _lens(S, case["lo"], case["hi"]), rng.randint(0, 300, S)
        bps = int((lens + add).max() + BLOCK - 1) // BLOCK
        table, nb = _table(rng, S, lens + add, bps, 2)
        nb = int(((add + 300 + BLOCK - 1) // BLOCK).sum()) + 2             # (as many for every seed)
        slots = np.concatenate([table[b, p // BLOCK] * np.int64(BLOCK) + p % BLOCK for b in range(S) for p in [np.arange(lens[b], lens[b] + add[b])]])
        T = len(slots)
        s["k"], s["v"] = _rows(g, hkv, T, D), _rows(g, hkv, T, D)
        s["slots"] = torch.from_numpy(slots).cuda()
        s["codes"], s["scales"] = _cache(g, layers, nb, hkv, None)
        s["layer"] = layers - 1
        s["k_rounded"], s["v_rounded"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        return s
    if kind in ("fork", "compact"):
        return _pages(s, case, g, rng, i32)
    B, N = case["batch"], case["nodes"]
    parent, lens = _trees(B, N, case["width"], seed), _lens(B, case["lo"], case["hi"])
    s["prefix_len"] = i32(lens)
    if kind == "append":
        path, n_acc = _paths(parent, case["acc"])
        bps = (case["hi"] + N + BLOCK - 1) // BLOCK
        table, nb = _table(rng, B, lens + N, bps, 2)
        s.update(path=i32(path), n_acc=i32(n_acc), table=i32(table), tree_kv=_rows(g, layers, 2, B, hkv, N, D))
        s["codes"], s["scales"] = _cache(g, layers, nb, hkv, None)
        s["rounded"] = torch.zeros_like(s["tree_kv"])
        return s
    hq = case["hq"]
    bps = max(1, (case["hi"] + BLOCK - 1) // BLOCK)
    table, nb = _table(rng, B, lens, bps, 1)
    s["codes"], s["scales"] = _cache(g, layers, nb, hkv, _live(table, lens, nb))
    s.update(table=i32(table), parent=i32(parent), layer=layers - 1)
    s["q"] = (1.5 * torch.randn((B, N, hq, D), generator=g, device="cuda")).to(torch.bfloat16)
    s["tree_k"], s["tree_v"] = _rows(g, B, hkv, N, D), _rows(g, B, hkv, N, D)
    return s


def _pages(s, case, g, rng, i32):
    """The state of a pool: tables, blocks held, how many more sequences hold a block, free blocks; and the pool itself."""
    if case["kind"] == "fork":
        P, fan, rows = case["prompts"], case["fan"], case["rows"]
        B, bps, full = P * (1 + fan), (rows + BLOCK - 1) // BLOCK + 1, (rows + BLOCK - 1) // BLOCK
        nb = P * (full + fan) + 5
        order = rng.permutation(nb)
        seq = rng.permutation(B)
        table, held, length = np.zeros((B, bps), np.int32), np.zeros(B, np.int32), np.zeros(B, np.int32)
        for p in range(P):
            table[seq[p], :full], held[seq[p]], length[seq[p]] = order[p * full:(p + 1) * full], full, rows
        s["src"], s["dst"] = i32(np.repeat(seq[:P], fan)), i32(seq[P:])
        drop = np.zeros(B, np.int32)
        drop[seq[P::2]] = 1
        s["drop"] = i32(drop)
        shares, n_free = np.zeros(nb, np.int32), nb - P * full
        free = np.concatenate([order[P * full:], np.zeros(P * full, np.int64)])
    else:
        n_live, n_free = case["live"], case["free"]
        nb = n_live + n_free
        low, high = rng.permutation(n_live), n_live + rng.permutation(n_free)
        m = case["moves"]
        live = rng.permutation(np.concatenate([low[m:], high[:m]]))
        free = np.concatenate([rng.permutation(np.concatenate([low[:m], high[m:]])), np.zeros(n_live, np.int64)])
        B, shared = case["seqs"], case["shared"]
        # every block in use has a first holder; the `shared` first ones begin the tables of further sequences too
        cut = np.sort(rng.randint(0, n_live - shared + 1, B - 1)) if B > 1 else np.zeros(0, np.int64)
        own_blocks = np.split(live[shared:], cut)
        begins = [live[:shared] if b == 0 else live[:rng.randint(0, shared + 1)] for b in range(B)]
        bps = n_live + 1
        table, held, shares = np.zeros((B, bps), np.int32), np.zeros(B, np.int32), np.full(nb, -1, np.int32)
        for b in range(B):
            row = np.concatenate([begins[b], own_blocks[b]])
            table[b, :len(row)], held[b] = row, len(row)
            shares[row] += 1
        shares = np.maximum(shares, 0)
        length = held * BLOCK
    # (one buffer, so that a pass can begin from the same state again)
    parts = [("table", table), ("held", held), ("length", length), ("shares", shares), ("free", free), ("n_free", [n_free])]
    s["first"] = i32(np.concatenate([np.asarray(x, np.int64).reshape(-1) for _, x in parts]))
    s["ints"] = s["first"].clone()
    at = 0
    for name, x in parts:
        x = np.asarray(x)
        s[name] = s["ints"][at:at + x.size].view(x.shape)
        at += x.size
    layers, hkv = case["layers"], case["hkv"]
    if case["bits"] == 8:
        s["pool"] = _cache(g, layers, nb, hkv, None)
    else:
        s["pool"] = (torch.randn((layers, 2, nb, hkv, BLOCK, D), generator=g, device="cuda", dtype=torch.bfloat16),)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------------------------


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own(s, kind)
    return {"write": _write, "append": _append, "attn": _attn, "fork": _fork, "compact": _compact}[kind](s)


def _context(c):
    """The handle that a program makes once and keeps."""
    from paper_2408_15562_b200 import binding
    hkv = c["hkv"]
    return binding.Context(c.get("hq", hkv), hkv, 16, 256, max_nodes=min(256, c.get("nodes", 1)), max_batch=c.get("batch", 512),
                           n_layers=c["layers"])


def _pool_out(s):
    return dict(codes=s["pool"][0].view(E4M3), scales=s["pool"][1]) if len(s["pool"]) == 2 else dict(rows=s["pool"][0])


def _own(s, kind):
    ctx = s["ctx"]
    if kind == "write":
        ctx.kv_write_fp8(s["k"], s["v"], s["slots"], s["codes"], s["scales"], layer=s["layer"], k_rounded=s["k_rounded"], v_rounded=s["v_rounded"])
        return dict(k=s["k_rounded"], v=s["v_rounded"], scales=s["scales"], codes=s["codes"].view(E4M3))
    if kind == "append":
        new_len = ctx.kv_append_fp8(s["codes"], s["scales"], s["table"], s["tree_kv"], s["path"], s["n_acc"], s["prefix_len"], rounded=s["rounded"])
        return dict(rounded=s["rounded"], scales=s["scales"], codes=s["codes"].view(E4M3), new_len=new_len)
    if kind == "attn":
        return dict(out=ctx.tree_attn_fp8(s["q"], s["codes"], s["scales"], s["table"], s["tree_k"], s["tree_v"], s["parent"], s["prefix_len"],
                                          layer=s["layer"]))
    s["ints"].copy_(s["first"])
    if kind == "fork":
        pairs = ctx.block_fork(s["src"], s["dst"], s["length"], s["table"], s["held"], s["shares"], s["free"], s["n_free"])
        ctx.block_copy(s["pool"], pairs)
        ctx.block_free(s["drop"], s["table"], s["held"], s["shares"], s["free"], s["n_free"])
    else:
        pairs = ctx.block_compact(s["table"], s["held"], s["shares"], s["free"], s["n_free"])
        ctx.block_copy(s["pool"], pairs)
    return dict(pairs=pairs, state=s["ints"], **_pool_out(s))


# ---- plain forms -------------------------------------------------------------------------------------------------------------------------


def _least_scale(most):
    """The least power of two, in the allowed range, with which magnitudes up to `most` are at most 448."""
    m, e = torch.frexp(most / 448.0)
    return torch.where(most > 0, torch.ldexp(torch.ones_like(most), e - (m == 0.5).to(e.dtype)), torch.full_like(most, LEAST)).clamp(LEAST, MOST)


def _put(codes, scales, blk, off, x):
    """Rows x [planes][Hkv][rows][128] into planes of codes [planes][blocks][Hkv][128][128] and scales [planes][blocks][Hkv][4]; the kept values."""
    P, nb, H = scales.shape[:3]
    group, at = torch.unique(blk * (BLOCK // GROUP) + off // GROUP, return_inverse=True)
    most = torch.zeros((P, H, len(group)), device=x.device)
    most.scatter_reduce_(2, at.expand(P, H, -1), x.float().abs().amax(-1), "amax")
    begun = torch.ones(len(group), dtype=torch.bool, device=x.device)
    begun[at[off % GROUP == 0]] = False
    need = _least_scale(most)
    gb, go = group // (BLOCK // GROUP), group % (BLOCK // GROUP)
    old = scales[:, gb, :, go].permute(1, 2, 0)                                     # [planes][Hkv][groups]
    new = torch.where(begun, torch.maximum(old, need), need)
    # rows of the groups begun before, by the new scale
    which = torch.nonzero(begun).flatten()
    rows = codes.view(P, nb, H, BLOCK // GROUP, GROUP, D)
    kept = rows[:, gb[which], :, go[which]].view(E4M3).float()                      # [groups][planes][Hkv][32][128]
    ratio = (old / new)[:, :, which].permute(2, 0, 1)[..., None, None]
    rows[:, gb[which], :, go[which]] = (kept * ratio).to(E4M3).view(torch.uint8)
    scales[:, gb, :, go] = new.permute(2, 0, 1)
    s = new[:, :, at][..., None]
    c = (x.float() / s).clamp(-448, 448).to(E4M3)
    codes[:, blk, :, off] = c.view(torch.uint8).permute(2, 0, 1, 3)
    return (c.float() * s).to(torch.bfloat16)


def _write(s):
    at = s["slots"]
    value = _put(s["codes"][s["layer"]], s["scales"][s["layer"]], at // BLOCK, at % BLOCK, torch.stack([s["k"], s["v"]]))
    s["k_rounded"].copy_(value[0])
    s["v_rounded"].copy_(value[1])
    return dict(k=s["k_rounded"], v=s["v_rounded"], scales=s["scales"], codes=s["codes"].view(E4M3))


def _append(s):
    path, n_acc, L = s["path"].long(), s["n_acc"], s["prefix_len"].long()
    B, N = path.shape
    b, j = torch.nonzero(torch.arange(N, device=path.device)[None] < n_acc[:, None], as_tuple=True)
    node, pos = path[b, j], L[b] + j
    x = s["tree_kv"].flatten(0, 1)[:, b, :, node].permute(1, 2, 0, 3)               # [planes][Hkv][rows][128]
    value = _put(s["codes"].flatten(0, 1), s["scales"].flatten(0, 1), s["table"][b, pos // BLOCK].long(), pos % BLOCK, x)
    s["rounded"].flatten(0, 1)[:, b, :, node] = value.permute(2, 0, 1, 3)
    return dict(rounded=s["rounded"], scales=s["scales"], codes=s["codes"].view(E4M3), new_len=(L + n_acc).to(torch.int32))


def _ancestors(parent):
    """[B][N][N] truth values: node j is node i or one of its ancestors."""
    B, N = parent.shape
    step = torch.eye(N, dtype=torch.float64, device=parent.device).repeat(B, 1, 1)
    step[:, 1:] += torch.nn.functional.one_hot(parent[:, 1:].long(), N).double()
    return torch.linalg.matrix_power(step, N) > 0.5


def _values(s, plane):
    """K (0) or V (1) rows of every sequence: [B][Hkv][rows][128]."""
    table = s["table"].long()
    codes, scales = s["codes"][s["layer"], plane][table].transpose(1, 2), s["scales"][s["layer"], plane][table].transpose(1, 2)
    return (codes.view(E4M3).float().unflatten(-2, (BLOCK // GROUP, GROUP)) * scales[..., None, None]).flatten(3, 4).flatten(2, 3)


def _attn(s):
    B, N, hq, _ = s["q"].shape
    hkv = s["tree_k"].shape[1]
    q = s["q"].float().view(B, N, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, D) / math.sqrt(D)
    k, v = _values(s, 0), _values(s, 1)
    there = torch.arange(k.shape[2], device=k.device)[None] < s["prefix_len"][:, None]
    v = torch.where(there[:, None, :, None], v, 0.0)
    x = torch.where(there[:, None, None], q @ k.transpose(-1, -2), -math.inf)
    seen = _ancestors(s["parent"])[:, None].repeat(1, 1, hq // hkv, 1)
    t = torch.where(seen, q @ s["tree_k"].float().transpose(-1, -2), -math.inf)
    most = torch.maximum(x.amax(-1, keepdim=True), t.amax(-1, keepdim=True))
    x, t = torch.exp(x - most), torch.exp(t - most)
    o = (x @ v + t @ s["tree_v"].float()) / (x.sum(-1, keepdim=True) + t.sum(-1, keepdim=True))
    return dict(out=o.view(B, hkv, hq // hkv, N, D).permute(0, 3, 1, 2, 4).reshape(B, N, hq, D).to(torch.bfloat16))


def _copy(s, src, dst):
    for x in s["pool"]:
        x[:, :, dst] = x[:, :, src]


def _pairs(src, dst, n):
    out = torch.full((n, 2), -1, dtype=torch.int32, device=src.device)
    out[:len(src), 0], out[:len(src), 1] = src, dst
    return out


def _push(s, freed):
    """Blocks onto the stack, the highest number first."""
    n = s["n_free"].long()
    s["free"][n + torch.arange(len(freed), device=freed.device)] = freed.flip(0).to(torch.int32)
    s["n_free"] += len(freed)


def _fork(s):
    s["ints"].copy_(s["first"])
    table, src, dst = s["table"], s["src"].long(), s["dst"].long()
    rows = s["length"][src]
    full, part = rows // BLOCK, rows % BLOCK != 0
    i = torch.arange(table.shape[1], device=table.device)[None]
    table[dst] = torch.where(i < full[:, None], table[src], table[dst])
    s["shares"].index_add_(0, table[src][i < full[:, None]].long(), torch.ones_like(full)[:, None].expand(-1, i.shape[1])[i < full[:, None]])
    which = torch.nonzero(part).flatten()
    old = table[src[which], full[which].long()]
    new = s["free"][s["n_free"].long() - 1 - torch.arange(len(which), device=which.device)]
    table[dst[which], full[which].long()] = new
    s["n_free"] -= len(which)
    s["held"][dst] = full + part.to(torch.int32)
    s["length"][dst] = rows
    _copy(s, old.long(), new.long())
    # some of them are dropped again
    gone = (i < s["held"][:, None]) & (s["drop"] != 0)[:, None]
    count = torch.zeros_like(s["shares"]).index_add_(0, table[gone].long(), torch.ones_like(table[gone]))
    left = s["shares"] - count
    s["shares"].copy_(left.clamp(min=0))
    s["held"].masked_fill_(s["drop"] != 0, 0)
    _push(s, torch.nonzero((count > 0) & (left < 0)).flatten())
    return dict(pairs=_pairs(old, new, len(src)), state=s["ints"], **_pool_out(s))


def _compact(s):
    s["ints"].copy_(s["first"])
    table, shares, nb = s["table"], s["shares"], s["shares"].numel()
    i = torch.arange(table.shape[1], device=table.device)[None]
    mine = i < s["held"][:, None]
    live, free = torch.zeros(nb, dtype=torch.bool, device=table.device), torch.zeros(nb, dtype=torch.bool, device=table.device)
    live[table[mine].long()] = True
    free[s["free"][:int(s["n_free"])].long()] = True
    low = (live | free).cumsum(0) <= live.sum()
    src, dst = torch.nonzero(live & ~low).flatten(), torch.nonzero(free & low).flatten()
    to = torch.arange(nb, device=table.device, dtype=torch.int32)
    to[src] = dst.to(torch.int32)
    table.copy_(torch.where(mine, to[table.long()], table))
    shares[dst] = shares[src]
    shares[src] = 0
    free[dst], free[src] = False, True
    s["free"][:int(s["n_free"])] = torch.nonzero(free).flatten().flip(0).to(torch.int32)
    _copy(s, src, dst)
    return dict(pairs=_pairs(src, dst, max(1, nb // 2)), state=s["ints"], **_pool_out(s))


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------------------------


def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None                                  # (copies and whole numbers)
    s = _inputs(case, seed)
    if case["kind"] == "attn":
        return _exact_attn(s)
    scales = s["scales"].double()
    if case["kind"] == "write":
        slots = s["slots"].cpu().numpy()
        k, v = (_exact_put(scales[s["layer"], plane], slots // BLOCK, slots % BLOCK, x.transpose(0, 1)).transpose(0, 1) for plane, x in ((0, s["k"]), (1, s["v"])))
        return dict(k=k, v=v, scales=scales, codes=None)
    out = torch.zeros_like(s["tree_kv"], dtype=torch.float64)
    path, n, L, table = (s[k].cpu().numpy() for k in ("path", "n_acc", "prefix_len", "table"))
    for b in range(path.shape[0]):
        rows = L[b] + np.arange(n[b])
        node = torch.from_numpy(path[b, :n[b]].astype(np.int64)).cuda()
        for layer in range(out.shape[0]):
            for plane in (0, 1):
                x = s["tree_kv"][layer, plane, b][:, node].transpose(0, 1)
                out[layer, plane, b][:, node] = _exact_put(scales[layer, plane], table[b, rows // BLOCK], rows % BLOCK, x).transpose(0, 1)
    return dict(rounded=out, scales=scales, codes=None, new_len=None)


def _exact_put(scales, blk, off, x):
    """Rows x [rows][Hkv][128] of one plane to their places: scales [blocks][Hkv][4] (64 bits) are brought up to date, the kept values come back."""
    bits = torch.arange(127, device="cuda")
    e, m = bits >> 3, (bits & 7).double()
    grid = torch.where(e > 0, torch.ldexp(1 + m / 8, e - 7), m / 512)
    out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    starts = np.flatnonzero(np.diff(blk * 4 + off // GROUP, prepend=-1))
    ends = np.append(starts[1:], len(blk))
    powers = torch.exp2(torch.arange(-64, 65, dtype=torch.float64, device="cuda"))
    most = x.double().abs().amax(-1)                                                # [rows][Hkv]
    number = torch.from_numpy(np.repeat(np.arange(len(starts)), ends - starts)).cuda()
    top = torch.zeros((len(starts), x.shape[1]), dtype=torch.float64, device="cuda")
    top.index_reduce_(0, number, most, "amax")
    scale = powers[torch.searchsorted(powers, top / 448).clamp(max=128)]
    at = torch.from_numpy(blk[starts].astype(np.int64)).cuda(), torch.from_numpy((off[starts] // GROUP).astype(np.int64)).cuda()
    before = scales[at[0], :, at[1]]
    goes_on = torch.from_numpy(off[starts] % GROUP != 0).cuda()[:, None]
    scale = torch.where(goes_on, torch.fmax(before, scale), scale)
    scales[at[0], :, at[1]] = scale
    y = x.double() / scale[number][..., None]
    hi = torch.bucketize(y.abs(), grid).clamp(1, 126)
    below, above = y.abs() - grid[hi - 1], grid[hi] - y.abs()
    near = torch.where((below < above) | ((below == above) & (hi % 2 == 1)), grid[hi - 1], grid[hi])
    out.copy_(torch.copysign(near, y) * scale[number][..., None])
    return out


def _exact_attn(s):
    B, N, hq, _ = s["q"].shape
    hkv = s["tree_k"].shape[1]
    lens, table, parent = (s[k].cpu().numpy() for k in ("prefix_len", "table", "parent"))
    out = torch.empty((B, N, hq, D), dtype=torch.float64, device="cuda")
    byte = torch.arange(256, device="cuda")
    e, m = (byte >> 3) & 15, (byte & 7).double()
    value = torch.where(e > 0, torch.ldexp(1 + m / 8, e - 7), m / 512) * (1 - 2 * (byte >> 7))
    for b in range(B):
        L = int(lens[b])
        blocks = torch.from_numpy(table[b, :(L + BLOCK - 1) // BLOCK].astype(np.int64)).cuda()
        see = torch.zeros((N, L + N), dtype=torch.bool)
        see[:, :L] = True
        for i in range(N):
            at = i
            while at >= 0:
                see[i, L + at] = True
                at = int(parent[b, at])
        see = see.cuda()
        for h in range(hkv):
            rows = []
            for plane, tree in ((0, s["tree_k"]), (1, s["tree_v"])):
                c = s["codes"][s["layer"], plane, blocks, h].reshape(-1, D)[:L].int()
                sc = s["scales"][s["layer"], plane, blocks, h].reshape(-1).double().repeat_interleave(GROUP)[:L]
                rows.append(torch.cat([value[c] * sc[:, None], tree[b, h].double()]))
            for u in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                w = (s["q"][b, :, u].double() @ rows[0].T) / math.sqrt(D)
                w = torch.softmax(w.masked_fill(~see, -math.inf), dim=-1)
                out[b, :, u] = w @ rows[1]
    return dict(out=out)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------------------


def work(case):
    kind, hkv, layers = case["kind"], case["hkv"], case["layers"]
    if kind == "write":
        T = int(_lens(case["seqs"], case["lo"], case["hi"]).sum())
        rows = 2 * T * hkv
        return dict(bytes=rows * (2 * D * 2 + D) + T * 8, flops=rows * D * 4)
    if kind == "append":
        rows = layers * 2 * case["batch"] * hkv * min(case["acc"], case["nodes"])
        return dict(bytes=rows * (2 * D * 2 + D), flops=rows * D * 4)
    if kind in ("fork", "compact"):
        block = layers * 2 * hkv * BLOCK * D * case["bits"] // 8
        if kind == "compact":
            return dict(bytes=2 * case["moves"] * block + 8 * case["live"], flops=case["live"])
        part = 1 if case["rows"] % BLOCK else 0
        rows = case["prompts"] * (1 + case["fan"]) * (case["rows"] // BLOCK + part)
        return dict(bytes=part * case["prompts"] * (1 + case["fan"]) * block + 8 * rows, flops=rows)
    B, N, hq = case["batch"], case["nodes"], case["hq"]
    keys = int(_lens(B, case["lo"], case["hi"]).sum())
    return dict(bytes=keys * hkv * 2 * (D + 4 / GROUP) + B * N * (hq + hkv) * D * 2 * 2, flops=4 * D * hq * N * (keys + B))
