"""What is measured of the operators around a cache held in 4 bits, and their plain forms.

  rope     rotary positions of several axes (time, height, width) on the rows of the QKV product, which leave in the layouts that the
           attention and the cache calls take; positions of tree nodes follow from the tree, those of prompt rows are given
  plan     block tables and the slots of new rows from the lengths of the requests
  write    K/V rows of a prompt into the 4-bit cache, by slots
  append   the accepted path's K/V rows of every layer into the 4-bit cache
  attn     tree-masked attention over the 4-bit cache (one node: the single-token step)

The cache: e2m1 codes, element 2i in the low and 2i + 1 in the high half of byte i, and one e4m3 scale for 16 elements, in blocks of 128
rows: codes [layers][2][blocks][Hkv][128][64], scales [layers][2][blocks][Hkv][128][8].
"""
import math

import numpy as np
import torch

own = False

D = 128
BLOCK = 128
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # One tree behind the QKV product of a layer: 60 rows, latency.
        dict(name="rope_tree_60", kind="rope", tree=1, batch=1, nodes=60, width=10, hq=32, hkv=8, far=2048, adjacent=0, sec_t=64, sec_h=0, sec_w=0, pad=0),
        # A prompt with video frames: three axes, far positions, rows of a wider buffer.
        dict(name="rope_video_8k", kind="rope", tree=0, batch=1, nodes=8201, width=1, hq=32, hkv=8, far=1000000, adjacent=0, sec_t=16, sec_h=24, sec_w=24, pad=64),
        # A step of a batch: every sequence gets room for one accepted path.
        dict(name="plan_step_batch16", kind="plan", batch=16, lo=512, hi=4096, add_lo=11, add_hi=11, drop=0, bps=40, extra_rows=0),
        # A server's admission: 200 slots, all of them given to new requests of up to 600 rows.
        dict(name="plan_admit_200", kind="plan", batch=200, lo=0, hi=0, add_lo=1, add_hi=600, drop=1, bps=24, extra_rows=777),
        # A short prompt of one request.
        dict(name="write_77_rows", kind="write", rows=77, hkv=8, layers=2, blocks=16, skip=0),
        # A long prompt, or several, with padding rows between them.
        dict(name="write_16k_rows", kind="write", rows=16411, hkv=8, layers=1, blocks=144, skip=1),
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
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 8), (64, 8), (32, 32), (8, 2), (28, 4), (52, 52), (12, 1), (40, 8), (5, 5), (24, 8)]


def draw(rng):
    kind = rng.choice(["rope", "rope", "plan", "write", "append", "attn", "attn", "attn", "attn", "attn"])
    hq, hkv = rng.choice(HEADS)
    if kind == "rope":
        tree = rng.randint(0, 1)
        sec_t = rng.randint(0, 64)
        sec_h = rng.randint(0, 64 - sec_t)
        batch, nodes = (_log(rng, 1, 32), _log(rng, 1, 256)) if tree else (rng.choice([1, 1, 2, 3]), _log(rng, 1, 2600))
        return dict(kind=kind, tree=tree, batch=batch, nodes=nodes, width=rng.choice([1, 3, 10, 30]), hq=hq, hkv=hkv, far=_log(rng, 10, 4000000),
                    adjacent=rng.randint(0, 1), sec_t=sec_t, sec_h=sec_h, sec_w=64 - sec_t - sec_h, pad=rng.choice([0, 8, 200]))
    if kind == "plan":
        batch, drop = _log(rng, 1, 500), rng.randint(0, 1)
        hi = 0 if drop else _log(rng, 1, 4000)
        add = _log(rng, 1, max(2, 100000 // batch)) if drop else _log(rng, 1, 64)
        return dict(kind=kind, batch=batch, lo=0, hi=hi, add_lo=0, add_hi=add, drop=drop, bps=(hi + add) // BLOCK + 1 + rng.randint(0, 9),
                    extra_rows=rng.choice([0, 1, 1000]))
    if kind == "write":
        rows = _log(rng, 1, 16000 * 8 // max(8, hkv))
        return dict(kind=kind, rows=rows, hkv=hkv, layers=rng.randint(1, 2), blocks=rows // BLOCK + rng.randint(1, 20), skip=rng.randint(0, 1))
    if kind == "append":
        hkv = min(hkv, 8)
        batch = _log(rng, 1, 32)
        nodes = _log(rng, 1, 120)
        return dict(kind=kind, batch=batch, nodes=nodes, width=rng.choice([1, 3, 10]), hkv=hkv, layers=rng.randint(1, max(1, 256 // batch // 4)),
                    lo=0, hi=_log(rng, 2, 500), acc=rng.randint(1, min(nodes, 24)))
    nodes = 1 if rng.random() < 0.35 else _log(rng, 2, 256)
    batch = _log(rng, 1, 32)
    rows_flop, row_bytes = 512 * hq * nodes, 2 * 72 * hkv
    most = min(60000000000 // rows_flop, 600000000 // row_bytes) // batch
    hi = _log(rng, 8, max(16, min(40000, most)))
    return dict(kind=kind, batch=batch, nodes=nodes, width=rng.choice([1, 3, 10, 30]), hq=hq, hkv=hkv, lo=rng.choice([0, hi // 8, hi]), hi=hi,
                layers=rng.choice([1, 2]))


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


def _cache(g, layers, n_blocks, hkv, dead):
    """Codes and scales as normally distributed rows leave them; `dead` rows [n_blocks][128] hold what was there before: scales that are no numbers."""
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    x = torch.special.ndtri((torch.arange(4096, dtype=torch.float64) + 0.5) / 4096) * 3.1
    lut = (torch.bucketize(x.abs(), edges) + 8 * (x < 0)).to(torch.uint8).cuda()
    shape = (layers, 2, n_blocks, hkv, BLOCK)
    r = torch.randint(0, 1 << 24, shape + (64,), generator=g, device="cuda", dtype=torch.int32)
    codes = lut[r & 4095] | (lut[r >> 12] << 4)
    del r
    s = 0.32 * torch.exp(0.3 * torch.randn(shape + (8,), generator=g, device="cuda"))
    scales = s.to(torch.float8_e4m3fn).view(torch.uint8)
    if dead is not None:
        scales.masked_fill_(torch.from_numpy(dead).cuda()[None, None, :, None, :, None], 0x7F)
    return codes, scales


def _rows(g, *shape):
    """bf16 K/V rows: normal values, a few channels far larger than the others."""
    x = torch.randn(shape, generator=g, device="cuda")
    boost = torch.ones(D, device="cuda")
    boost[3::41] = 6.0
    return (x * boost).to(torch.bfloat16)


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
    s = dict(case=case)
    if kind == "rope":
        B, N, hq, hkv = (case[k] for k in ("batch", "nodes", "hq", "hkv"))
        width = (hq + 2 * hkv) * D
        s["qkv"] = torch.randn((B, N, width + case["pad"]), generator=g, device="cuda").to(torch.bfloat16)[..., :width]
        s["theta"], s["sections"] = 500000.0, (case["sec_t"], case["sec_h"], case["sec_w"])
        if case["tree"]:
            s["parent"], s["start"], s["positions"] = i32(_trees(B, N, case["width"], seed)), i32(rng.randint(0, case["far"], (B, 3))), None
        else:
            s["parent"], s["start"], s["positions"] = None, None, i32(rng.randint(0, case["far"], (B, N, 3)))
        return s
    if kind == "plan":
        B, bps = case["batch"], case["bps"]
        lens, add = _lens(B, case["lo"], case["hi"]), rng.permutation(_lens(B, case["add_lo"], case["add_hi"]))
        held_rows = rng.permutation(_lens(B, 1, bps * BLOCK)) if case["drop"] else lens
        table, n_blocks = _table(rng, B, held_rows, bps, 0)
        held = (held_rows + BLOCK - 1) // BLOCK
        spare = int(np.maximum((lens + add + BLOCK - 1) // BLOCK, 1).sum()) + 5
        free = np.zeros(n_blocks + spare, np.int64)
        free[:spare] = n_blocks + rng.permutation(spare)
        s.update(len=i32(lens), add=i32(add), drop=i32(np.ones(B)) if case["drop"] else None, table=i32(table), held=i32(held), free=i32(free),
                 n_free=i32([spare]), max_rows=int(_lens(B, case["add_lo"], case["add_hi"]).sum()) + case["extra_rows"])
        return s
    if kind == "write":
        T, hkv, nb = case["rows"], case["hkv"], case["blocks"]
        s["k"], s["v"] = _rows(g, hkv, T, D), _rows(g, hkv, T, D)
        slots = (rng.permutation(nb)[:, None] * BLOCK + np.arange(BLOCK)[None]).reshape(-1)[:T].astype(np.int64)
        if case["skip"]:
            slots[rng.permutation(T)[:T // 7]] = -1
        s["slots"] = torch.from_numpy(slots).cuda()
        s["codes"], s["scales"] = _cache(g, case["layers"], nb, hkv, None)
        s["layer"] = case["layers"] - 1
        s["k_rounded"], s["v_rounded"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        return s
    B, N, hkv, layers = (case[k] for k in ("batch", "nodes", "hkv", "layers"))
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
    dead = np.ones((nb, BLOCK), bool)
    for b in range(B):
        for i in range((int(lens[b]) + BLOCK - 1) // BLOCK):
            dead[table[b, i], :min(BLOCK, int(lens[b]) - i * BLOCK)] = False
    s["codes"], s["scales"] = _cache(g, layers, nb, hkv, dead)
    s.update(table=i32(table), parent=i32(parent), layer=layers - 1)
    s["q"] = (1.5 * torch.randn((B, N, hq, D), generator=g, device="cuda")).to(torch.bfloat16)
    s["tree_k"], s["tree_v"] = _rows(g, B, hkv, N, D), _rows(g, B, hkv, N, D)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------------------------


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own(s, kind)
    return {"rope": _rope, "plan": _plan, "write": _write, "append": _append, "attn": _attn}[kind](s)


def _context(c):
    """The handle that a program makes once and keeps."""
    from paper_2408_15562_b200 import binding
    hkv = c.get("hkv", 1)
    return binding.Context(c.get("hq", hkv), hkv, 16, 256, max_nodes=min(256, c.get("nodes", 1)), max_batch=c.get("batch", 1),
                           n_layers=c.get("layers", 1))


def _own(s, kind):
    ctx = s["ctx"]
    if kind == "rope":
        q, k, v = ctx.rope_qkv(s["qkv"], s["theta"], s["sections"], parent=s["parent"], start=s["start"], positions=s["positions"],
                               adjacent=bool(s["case"]["adjacent"]))
        return dict(q=q, k=k, v=v)
    if kind == "plan":
        row_start, slots, row_seq, row_pos = ctx.block_plan(s["len"], s["add"], s["table"], s["held"], s["free"], s["n_free"], s["max_rows"],
                                                            drop=s["drop"])
        return dict(row_start=row_start, slots=slots, row_seq=row_seq, row_pos=row_pos, table=s["table"], held=s["held"], free=s["free"],
                    n_free=s["n_free"])
    if kind == "write":
        ctx.kv_write_packed(s["k"], s["v"], s["slots"], s["codes"], s["scales"], layer=s["layer"], k_rounded=s["k_rounded"], v_rounded=s["v_rounded"])
        return dict(k=s["k_rounded"], v=s["v_rounded"], scales=s["scales"].view(torch.float8_e4m3fn), codes=s["codes"])
    if kind == "append":
        new_len = ctx.kv_append_packed(s["codes"], s["scales"], s["table"], s["tree_kv"], s["path"], s["n_acc"], s["prefix_len"],
                                       rounded=s["rounded"])
        return dict(rounded=s["rounded"], scales=s["scales"].view(torch.float8_e4m3fn), codes=s["codes"], new_len=new_len)
    return dict(out=ctx.tree_attn_packed(s["q"], s["codes"], s["scales"], s["table"], s["tree_k"], s["tree_v"], s["parent"], s["prefix_len"],
                                         layer=s["layer"]))


# ---- plain forms -------------------------------------------------------------------------------------------------------------------------


def _ancestors(parent):
    """[B][N][N] truth values: node j is node i or one of its ancestors."""
    B, N = parent.shape
    step = torch.eye(N, dtype=torch.float64, device=parent.device).repeat(B, 1, 1)
    step[:, 1:] += torch.nn.functional.one_hot(parent[:, 1:].long(), N).double()
    return torch.linalg.matrix_power(step, N) > 0.5


def _rope(s):
    qkv, (st, sh, sw) = s["qkv"], s["sections"]
    B, N, _ = qkv.shape
    hq, hkv = s["case"]["hq"], s["case"]["hkv"]
    pos = s["positions"]
    if pos is None:
        depth = _ancestors(s["parent"]).sum(-1) - 1
        pos = s["start"][:, None, :] + depth[..., None]
    axis = torch.tensor([0] * st + [1] * sh + [2] * sw, device=qkv.device)
    inv = s["theta"] ** (-torch.arange(0, D, 2, dtype=torch.float64, device=qkv.device) / D)
    a = pos[..., axis].double() * inv
    c, n = torch.cos(a).float()[:, :, None], torch.sin(a).float()[:, :, None]
    x = qkv.reshape(B, N, hq + 2 * hkv, D)
    y = x[:, :, :hq + hkv].float()
    if s["case"]["adjacent"]:
        y1, y2 = y[..., 0::2], y[..., 1::2]
        y = torch.stack([y1 * c - y2 * n, y2 * c + y1 * n], dim=-1).flatten(-2)
    else:
        y1, y2 = y[..., :64], y[..., 64:]
        y = torch.cat([y1 * c - y2 * n, y2 * c + y1 * n], dim=-1)
    y = y.to(torch.bfloat16)
    return dict(q=y[:, :, :hq].contiguous(), k=y[:, :, hq:].transpose(1, 2).contiguous(), v=x[:, :, hq + hkv:].transpose(1, 2).contiguous())


def _plan(s):
    length, add, table, held, free = s["len"].long(), s["add"].long(), s["table"], s["held"].long(), s["free"]
    B, bps = table.shape
    dev, n_blocks, n_free = table.device, free.numel(), s["n_free"].long()
    gone = s["drop"].long() != 0 if s["drop"] is not None else torch.zeros(B, dtype=torch.bool, device=dev)
    i = torch.arange(bps, device=dev)[None]
    back = torch.where(gone, held, 0)
    at = n_free + (back.cumsum(0) - back)[:, None] + i
    stack = torch.cat([free, free[:1]]).scatter(0, torch.where(i < back[:, None], at, n_blocks).flatten(), table.flatten())
    n_free = n_free + back.sum()
    have = torch.where(gone, 0, held)
    take = ((length + add + BLOCK - 1) // BLOCK - have).clamp(min=0)
    at = n_free - 1 - (take.cumsum(0) - take)[:, None] - (i - have[:, None])
    new = (i >= have[:, None]) & (i < (have + take)[:, None])
    fresh = torch.where(new, stack[at.clamp(0, n_blocks)], table)
    end = add.cumsum(0)
    r = torch.arange(s["max_rows"], device=dev)
    q = torch.searchsorted(end, r, right=True)
    there = q < B
    q = q.clamp(max=B - 1)
    p = length[q] + r - (end - add)[q]
    slots = fresh[q, (p // BLOCK).clamp(max=bps - 1)].long() * BLOCK + p % BLOCK
    s["table"].copy_(fresh)
    s["held"].copy_(have + take)
    s["free"].copy_(stack[:n_blocks])
    s["n_free"].copy_(n_free - take.sum())
    i32 = torch.int32
    return dict(row_start=torch.cat([end[:1] * 0, end]).to(i32), slots=torch.where(there, slots, -1), row_seq=torch.where(there, q, -1).to(i32),
                row_pos=torch.where(there, p, -1).to(i32), table=s["table"], held=s["held"], free=s["free"], n_free=s["n_free"])


def _quantise(x):
    """[..., 128] bf16 -> codes [..., 64], scales [..., 8] (bytes), and the values they stand for."""
    y = x.float().unflatten(-1, (8, 16))
    most = y.abs().amax(-1, keepdim=True)
    scale = (most / torch.full_like(most, 6.0)).clamp(max=448.0).to(torch.float8_e4m3fn)      # (by a number: a product with 1/6)
    v = scale.float()
    m = (y / torch.where(v > 0, v, 1.0)).abs() * (v > 0)
    code = (m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)
    neg = torch.signbit(y)
    value = torch.tensor(E2M1, device=x.device)[code] * v
    value = torch.where(neg, -value, value).flatten(-2).to(torch.bfloat16)
    code = (code + 8 * neg).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale.view(torch.uint8).squeeze(-1), value


def _write(s):
    keep = torch.nonzero(s["slots"] >= 0).flatten()
    at = s["slots"][keep]
    kv = torch.stack([s["k"], s["v"]])[:, :, keep]
    codes, scales, value = _quantise(kv)
    blk, off = at // BLOCK, at % BLOCK
    s["codes"][s["layer"]][:, blk, :, off] = codes.permute(2, 0, 1, 3)
    s["scales"][s["layer"]][:, blk, :, off] = scales.permute(2, 0, 1, 3)
    s["k_rounded"][:, keep] = value[0]
    s["v_rounded"][:, keep] = value[1]
    return dict(k=s["k_rounded"], v=s["v_rounded"], scales=s["scales"].view(torch.float8_e4m3fn), codes=s["codes"])


def _append(s):
    path, n_acc, L = s["path"].long(), s["n_acc"], s["prefix_len"].long()
    B, N = path.shape
    b, j = torch.nonzero(torch.arange(N, device=path.device)[None] < n_acc[:, None], as_tuple=True)
    node, pos = path[b, j], L[b] + j
    codes, scales, value = _quantise(s["tree_kv"][:, :, b, :, node])
    blk, off = s["table"][b, pos // BLOCK].long(), pos % BLOCK
    s["codes"][:, :, blk, :, off] = codes
    s["scales"][:, :, blk, :, off] = scales
    s["rounded"][:, :, b, :, node] = value
    return dict(rounded=s["rounded"], scales=s["scales"].view(torch.float8_e4m3fn), codes=s["codes"], new_len=(L + n_acc).to(torch.int32))


def _values(s, plane):
    """K (0) or V (1) rows of every sequence: [B][Hkv][rows][128]."""
    table = s["table"].long()
    codes, scales = s["codes"][s["layer"], plane][table].transpose(1, 2), s["scales"][s["layer"], plane][table].transpose(1, 2)
    pair = torch.tensor([[v * w for v in E2M1] for w in (1.0, -1.0)], device=codes.device).flatten()
    byte = torch.arange(256, device=codes.device)
    x = torch.stack([pair[byte & 15], pair[byte >> 4]], dim=-1)[codes.int()]
    x = x.flatten(-2).unflatten(-1, (8, 16)) * scales.view(torch.float8_e4m3fn).float()[..., None]
    return x.flatten(-2).flatten(2, 3)


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


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------------------------


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "plan":
        return None
    if kind == "rope":
        return _exact_rope(s)
    if kind == "write":
        k, v = torch.zeros_like(s["k"], dtype=torch.float64), torch.zeros_like(s["v"], dtype=torch.float64)
        scales = s["scales"].view(torch.float8_e4m3fn).double()
        at = s["slots"].cpu().numpy()
        rows = torch.from_numpy(np.flatnonzero(at >= 0)).cuda()
        for plane, x, y in ((0, s["k"], k), (1, s["v"], v)):
            value, scale = _exact_values(x[:, rows])
            y[:, rows] = value
            scales[s["layer"], plane, s["slots"][rows] // BLOCK, :, s["slots"][rows] % BLOCK] = scale.transpose(0, 1)
        return dict(k=k, v=v, scales=scales, codes=None)
    if kind == "append":
        out = torch.zeros_like(s["tree_kv"], dtype=torch.float64)
        scales = s["scales"].view(torch.float8_e4m3fn).double()
        path, n, L, table = (s[k].cpu().numpy() for k in ("path", "n_acc", "prefix_len", "table"))
        for b in range(path.shape[0]):
            for j in range(n[b]):
                value, scale = _exact_values(s["tree_kv"][:, :, b, :, path[b, j]])
                out[:, :, b, :, path[b, j]] = value
                row = int(L[b]) + j
                scales[:, :, int(table[b, row // BLOCK]), :, row % BLOCK] = scale
        return dict(rounded=out, scales=scales, codes=None, new_len=None)
    return _exact_attn(s)


def _exact_rope(s):
    qkv = s["qkv"].double()
    B, N, _ = qkv.shape
    hq, hkv = s["case"]["hq"], s["case"]["hkv"]
    if s["positions"] is None:
        parent, start = s["parent"].cpu().numpy(), s["start"].cpu().numpy()
        depth = np.zeros((B, N), np.int64)
        for i in range(1, N):
            depth[:, i] = depth[np.arange(B), parent[:, i]] + 1
        pos = start[:, None].astype(np.int64) + depth[..., None]
    else:
        pos = s["positions"].cpu().numpy().astype(np.int64)
    z = torch.empty((B, N, 64), dtype=torch.complex128, device="cuda")
    first = 0
    for axis, count in enumerate(s["sections"]):
        for i in range(first, first + count):
            angle = torch.from_numpy(pos[..., axis].astype(np.float64) * math.exp(-2 * i / D * math.log(s["theta"]))).cuda()
            z[..., i] = torch.polar(torch.ones_like(angle), angle)
        first += count
    x = qkv.view(B, N, hq + 2 * hkv, D)
    w = x[:, :, :hq + hkv].unflatten(-1, (64, 2) if s["case"]["adjacent"] else (2, 64))
    w = w if s["case"]["adjacent"] else w.transpose(-1, -2)
    w = torch.view_as_real(torch.view_as_complex(w.contiguous()) * z[:, :, None])
    w = (w if s["case"]["adjacent"] else w.transpose(-1, -2)).flatten(-2)
    return dict(q=w[:, :, :hq], k=w[:, :, hq:].transpose(1, 2), v=x[:, :, hq + hkv:].transpose(1, 2))


def _exact_values(x):
    """The values that rows [..., 128] are kept as and their scales, each the nearest one of its type (a tie: the one with the even code)."""
    y = x.double().unflatten(-1, (8, 16))
    bits = torch.arange(127, device="cuda")
    e, m = bits >> 3, (bits & 7).double()
    e4m3 = torch.where(e > 0, torch.ldexp(1 + m / 8, e - 7), m / 512)
    most = y.abs().amax(-1)
    scale = _nearest(most / torch.full_like(most, 6.0), e4m3)
    e2m1 = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    m = _nearest(torch.where(scale[..., None] > 0, y.abs() / scale[..., None], 0.0), e2m1) * scale[..., None]
    return torch.where(y < 0, -m, m).flatten(-2), scale


def _nearest(x, grid):
    hi = torch.bucketize(x, grid).clamp(1, len(grid) - 1)
    below, above = x - grid[hi - 1], grid[hi] - x
    return torch.where((below < above) | ((below == above) & (hi % 2 == 1)), grid[hi - 1], grid[hi])


def _exact_attn(s):
    B, N, hq, _ = s["q"].shape
    hkv = s["tree_k"].shape[1]
    lens, table, parent = (s[k].cpu().numpy() for k in ("prefix_len", "table", "parent"))
    out = torch.empty((B, N, hq, D), dtype=torch.float64, device="cuda")
    magnitude = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
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
                c = s["codes"][s["layer"], plane, blocks, h].reshape(-1, 64)[:L].int()
                sc = s["scales"][s["layer"], plane, blocks, h].reshape(-1, 8)[:L].view(torch.float8_e4m3fn).double()
                x = torch.empty((L, D), dtype=torch.float64, device="cuda")
                for half in (0, 1):
                    n = (c >> (4 * half)) & 15
                    x[:, half::2] = magnitude[n & 7] * (1 - 2 * (n >> 3)) * sc.repeat_interleave(8, dim=1)
                rows.append(torch.cat([x, tree[b, h].double()]))
            for u in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                w = (s["q"][b, :, u].double() @ rows[0].T) / math.sqrt(D)
                w = torch.softmax(w.masked_fill(~see, -math.inf), dim=-1)
                out[b, :, u] = w @ rows[1]
    return dict(out=out)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind == "rope":
        rows = case["batch"] * case["nodes"]
        heads = case["hq"] + 2 * case["hkv"]
        return dict(bytes=rows * (heads * D * 2 * 2 + (4 if case["tree"] else 12)), flops=rows * (case["hq"] + case["hkv"]) * D * 3)
    if kind == "plan":
        B = case["batch"]
        rows = int(_lens(B, case["add_lo"], case["add_hi"]).sum()) + case["extra_rows"]
        return dict(bytes=rows * 16 + B * 24, flops=rows)
    if kind == "write":
        rows = 2 * case["rows"] * case["hkv"]
        return dict(bytes=rows * (2 * D * 2 + 72) + case["rows"] * 8, flops=rows * D * 4)
    if kind == "append":
        rows = case["layers"] * 2 * case["batch"] * case["hkv"] * min(case["acc"], case["nodes"])
        return dict(bytes=rows * (2 * D * 2 + 72), flops=rows * D * 4)
    B, N, hq, hkv = (case[k] for k in ("batch", "nodes", "hq", "hkv"))
    keys = int(_lens(B, case["lo"], case["hi"]).sum())
    return dict(bytes=keys * hkv * 2 * 72 + B * N * (hq + hkv) * D * 2 * 2, flops=4 * D * hq * N * (keys + B))
