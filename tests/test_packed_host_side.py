"""What the operators around the 4-bit cache refuse, and in which order: api_cache.cu compiled for the CPU against stand-ins for the device and the
launchers (`packed_fake.cpp`).  What is refused launches nothing.  The binding's own refusals run in processes of their own, as no device is needed."""
import ctypes
import math
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2408_15562_b200", "csrc")
NULL, CUDA, TREE, SHAPE, ALIGN, RANGE, LARGE, DEVICE = "NULL", "CUDA", "TREE_TOO_LARGE", "SHAPE", "ALIGN", "RANGE", "TOO_LARGE", "DEVICE"
P, ODD = 0x10000, 0x10008                  # a 16-byte aligned address that nothing reads, and one that is not
P1, P2, P3 = 0x20000, 0x30000, 0x40000     # further ones
HQ, HKV, NODES, LAYERS, BATCH = 8, 2, 64, 3, 2000


def codes():
    import re
    text = open(os.path.join(ROOT, "include", "fspad.h")).read()
    return {m[0]: int(m[1]) for m in re.findall(r"#define\s+FSPAD_ERR_(\w+)\s+\(?(-?\d+)\)?", text)} or \
           {m[0]: int(m[1]) for m in re.findall(r"FSPAD_ERR_(\w+)\s*=\s*(-?\d+)", text)}


ERR = codes()


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("packed_host_side") / "libpackedhost.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic",
                           "-DatomicCAS(p,a,b)=((void)(p),(void)(a),(void)(b))",
                           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-I/usr/local/cuda/include",
                           "-x", "c++", os.path.join(CSRC, "api_cache.cu"), os.path.join(HERE, "packed_fake.cpp"), "-o", out])
    lib = ctypes.CDLL(out)
    vp, ci = ctypes.c_void_p, ctypes.c_int
    lib.fake_context.restype = vp
    lib.fake_log.restype = ctypes.c_char_p
    lib.fake_turns.restype = ctypes.c_double
    lib.fake_context_free.argtypes = [vp]
    lib.fspad_device.argtypes = [vp]
    lib.fspad_rope_qkv.argtypes = [vp, vp, ctypes.c_int64, vp, vp, vp, ci, ci, ctypes.c_double, ci, ci, ci, ci, vp, vp, vp, vp]
    lib.fspad_block_plan.argtypes = [vp] * 4 + [ci] * 3 + [vp] * 4 + [ci] + [vp] * 5
    lib.fspad_kv_write_packed.argtypes = [vp] * 4 + [ci, ci, vp, vp, ci, vp, vp, vp]
    lib.fspad_kv_append_packed.argtypes = [vp] * 4 + [ci, ci] + [vp] * 4 + [ci, ci, vp, vp, vp]
    lib.fspad_tree_attn_packed_workspace_bytes.argtypes = [vp, ci, ci]
    lib.fspad_tree_attn_packed_workspace_bytes.restype = ctypes.c_size_t
    lib.fspad_tree_attn_packed.argtypes = [vp] * 4 + [ci, vp, ci, ci] + [vp] * 4 + [ci, ci, vp, vp, ctypes.c_size_t, vp]
    lib.ctx = lib.fake_context(HQ, HKV, NODES, LAYERS, BATCH)
    yield lib
    lib.fake_context_free(lib.ctx)


# the arguments of each call, in order, with values that are accepted
CALLS = {
    "rope_qkv": dict(qkv=P, row_stride=(HQ + 2 * HKV) * 128, positions=None, start=P, parent=P, n_nodes=NODES, batch=2, theta=1e4, sec_t=16, sec_h=24,
                     sec_w=24, adjacent=0, q=P1, k=P2, v=P3, stream=None),
    "block_plan": dict(len=P, add=P, drop=None, batch=5, blocks_per_seq=4, n_blocks=9, block_table=P, held=P, free_blocks=P, n_free=P, max_rows=7,
                       row_start=P, slots=P, row_seq=None, row_pos=None, stream=None),
    "kv_write_packed": dict(k=P, v=P, slots=P, rows=7, layer=2, codes=P, scales=P, n_blocks=9, k_rounded=None, v_rounded=None, stream=None),
    "kv_append_packed": dict(codes=P, scales=P, block_table=P, blocks_per_seq=4, n_blocks=9, tree_kv=P, accepted_path=P, n_accepted=P, prefix_len=P,
                             n_nodes=NODES, batch=2, rounded=None, new_len=None, stream=None),
    "tree_attn_packed": dict(q=P, codes=P, scales=P, layer=1, block_table=P, blocks_per_seq=4, n_blocks=9, tree_k=P, tree_v=P, parent=P, prefix_len=P,
                             n_nodes=NODES, batch=2, out=P1, workspace=P, workspace_bytes=NODES * 2 * 1000, stream=None),
}


def run(lib, name, ctx="own", device=0, fails=0, fits=1, **change):
    args = dict(CALLS[name])
    assert set(change) <= set(args)
    args.update(change)
    lib.fake_set(device, fails, fits)
    rc = getattr(lib, "fspad_" + name)(lib.ctx if ctx == "own" else ctx, *args.values())
    return rc, lib.fake_log().decode().splitlines()


TREE_SIZES = [(dict(n_nodes=NODES + 1), TREE), (dict(n_nodes=0), SHAPE), (dict(n_nodes=-1), SHAPE), (dict(batch=-1), SHAPE), (dict(batch=BATCH + 1), SHAPE)]
BLOCKS = [(dict(blocks_per_seq=0), SHAPE), (dict(n_blocks=0), SHAPE), (dict(n_blocks=-1), SHAPE), (dict(blocks_per_seq=1 << 24), LARGE)]


def _null(*names):
    return [({n: None}, NULL) for n in names]


def _odd(*names):
    return [({n: ODD}, ALIGN) for n in names]


REFUSED = {
    "rope_qkv": _null("qkv", "q", "k", "v", "start", "parent") + _odd("qkv", "q", "k", "v") + TREE_SIZES + [
        (dict(positions=P), NULL), (dict(positions=P, start=None), NULL), (dict(positions=P, parent=None), NULL),
        (dict(positions=P, start=None, parent=None, n_nodes=0), SHAPE), (dict(positions=P, start=None, parent=None, batch=BATCH + 1), SHAPE),
        (dict(positions=P, start=None, parent=None, n_nodes=1 << 30, batch=2), LARGE),
        (dict(sec_t=17), SHAPE), (dict(sec_t=0), SHAPE), (dict(sec_t=65, sec_h=-1, sec_w=0), SHAPE), (dict(sec_t=-8, sec_h=48), SHAPE),
        (dict(row_stride=(HQ + 2 * HKV) * 128 - 8), SHAPE), (dict(row_stride=(HQ + 2 * HKV) * 128 + 4), SHAPE), (dict(row_stride=0), SHAPE),
        (dict(theta=0.0), RANGE), (dict(theta=-1.0), RANGE), (dict(theta=math.nan), RANGE), (dict(theta=math.inf), RANGE), (dict(theta=5e-324), RANGE)] + [(dict([c]), RANGE) for c in [("q", P), ("k", P), ("v", P), ("q", P2), ("k", P3), ("v", P1)]],
    "block_plan": _null("len", "add", "block_table", "held", "free_blocks", "n_free", "row_start", "slots") + BLOCKS + [
        (dict(batch=-1), SHAPE), (dict(batch=BATCH + 1), SHAPE), (dict(max_rows=-1), SHAPE), (dict(batch=1025), LARGE)],
    "kv_write_packed": _null("k", "v", "slots", "codes", "scales") + _odd("k", "v", "codes", "scales") + [
        (dict(k_rounded=P), NULL), (dict(v_rounded=P), NULL), (dict(k_rounded=ODD, v_rounded=P), ALIGN), (dict(k_rounded=P, v_rounded=ODD), ALIGN),
        (dict(rows=-1), SHAPE), (dict(layer=-1), SHAPE), (dict(layer=LAYERS), SHAPE), (dict(n_blocks=0), SHAPE), (dict(rows=1 << 30), LARGE)],
    "kv_append_packed": _null("codes", "scales", "block_table", "tree_kv", "accepted_path", "n_accepted", "prefix_len") +
        _odd("codes", "scales", "tree_kv", "rounded") + TREE_SIZES + BLOCKS + [(dict(new_len=P), RANGE)],
    "tree_attn_packed": _null("q", "codes", "scales", "block_table", "tree_k", "tree_v", "parent", "prefix_len", "out", "workspace") +
        _odd("q", "codes", "scales", "tree_k", "tree_v", "out", "workspace") + TREE_SIZES + BLOCKS + [
        (dict(layer=-1), SHAPE), (dict(layer=LAYERS), SHAPE), (dict(workspace_bytes=NODES * 2 * 1000 - 1), RANGE), (dict(fits=0), LARGE), (dict(out=P), RANGE)],
}


@pytest.mark.parametrize("name,change,want", [(n, c, w) for n, cases in REFUSED.items() for c, w in cases])
def test_what_is_refused(lib, name, change, want):
    rc, log = run(lib, name, **change)
    assert rc == ERR[want] and not log, (rc, log)


@pytest.mark.parametrize("name", CALLS)
def test_contexts_devices_and_failed_launches(lib, name):
    assert run(lib, name, ctx=None) == (ERR[NULL], [])
    assert run(lib, name, device=1) == (ERR[DEVICE], [])
    assert run(lib, name, device=-1) == (ERR[CUDA], [])
    rc, log = run(lib, name, fails=1)
    assert rc == ERR[CUDA] and len(log) == 1
    rc, log = run(lib, name)
    assert rc == 0 and len(log) == 1
    assert lib.fspad_device(lib.ctx) == 0 and lib.fspad_device(None) == -1


def test_nothing_to_do_launches_nothing_but_a_plan_is_written(lib):
    for name in ("rope_qkv", "kv_append_packed", "tree_attn_packed"):
        assert run(lib, name, batch=0) == (0, [])
    assert run(lib, "kv_write_packed", rows=0) == (0, [])
    rc, log = run(lib, "block_plan", batch=0)
    assert rc == 0 and log == ["plan 0 4 9 7"]          # row_start[0] and the slots
    assert run(lib, "block_plan", max_rows=0)[0] == 0


def test_what_the_launchers_get(lib):
    assert run(lib, "rope_qkv")[1] == ["rope 1536 tree 64 2 16 40 halves 0"]
    turns = [lib.fake_turns(i) for i in range(64)]
    assert turns == pytest.approx([1e4 ** (-i / 64) / (2 * math.pi) for i in range(64)], rel=1e-14)
    run(lib, "rope_qkv", theta=5e5)                      # (another theta, and the first once more)
    assert lib.fake_turns(63) == pytest.approx(5e5 ** (-63 / 64) / (2 * math.pi), rel=1e-14)
    run(lib, "rope_qkv")
    assert [lib.fake_turns(i) for i in range(64)] == turns
    assert run(lib, "rope_qkv", positions=P, start=None, parent=None, n_nodes=5000, batch=1, adjacent=3, stream=7)[1] == [
        "rope 1536 given 5000 1 16 40 adjacent 7"]
    rows = 9 * HKV * 128                                 # of a layer's K or V
    k, s = P + 2 * rows * 64, P + 2 * rows * 8
    assert run(lib, "tree_attn_packed")[1] == [f"attention {k} {s} {k + rows * 64} {s + rows * 8} 64 2"]
    nb = 1 << 21                                         # offsets of a layer beyond 32 bits
    rows = nb * HKV * 128
    k, s = P + 4 * rows * 64, P + 4 * rows * 8
    assert run(lib, "tree_attn_packed", n_blocks=nb, layer=2)[1] == [f"attention {k} {s} {k + rows * 64} {s + rows * 8} 64 2"]


def test_workspace_bytes(lib):
    size = lib.fspad_tree_attn_packed_workspace_bytes
    assert size(lib.ctx, 3, 2) == 6000 and size(None, 3, 2) == 0
    assert size(lib.ctx, NODES + 1, 2) == 0 and size(lib.ctx, 0, 2) == 0 and size(lib.ctx, 1, BATCH + 1) == 0


SCRIPT = """
import ctypes, sys, types
import torch
from paper_2408_15562_b200 import binding
what = sys.argv[1]
bf, i32, u8 = torch.bfloat16, torch.int32, torch.uint8
ctx = types.SimpleNamespace(_h=ctypes.c_void_p(), _sizes=(8, 2, 1, 4))
ctx._packed_call = lambda *a: binding.Context._packed_call(ctx, *a)
binding._stream = lambda s: 0
C = binding.Context
def fake(*shape, dtype=bf, at="cuda:0"):
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode(): return torch.empty(shape, dtype=dtype, device=at)
def host(*shape, dtype=bf): return torch.zeros(shape, dtype=dtype)
def attention(q, **kw):
    a = dict(codes=host(1), scales=host(1), block_table=host(1), tree_k=host(1), tree_v=host(1), parent=host(1), prefix_len=host(1), workspace=host(1))
    return C.tree_attn_packed(ctx, q, **{**a, **kw})
try:
    if what == "rope host": C.rope_qkv(ctx, host(1, 4, 1536), 1e4)
    if what == "rope type": C.rope_qkv(ctx, host(1, 4, 1536).float(), 1e4)
    if what == "rope list": C.rope_qkv(ctx, [1.0], 1e4)
    if what == "rope theta": C.rope_qkv(ctx, fake(1, 4, 1536), "x")
    if what == "rope width": C.rope_qkv(ctx, fake(1, 4, 1530), 1e4)
    if what == "rope dims": C.rope_qkv(ctx, fake(4, 1536), 1e4)
    if what == "rope sections": C.rope_qkv(ctx, fake(1, 4, 1536), 1e4, (64, 0))
    if what == "rope section": C.rope_qkv(ctx, fake(1, 4, 1536), 1e4, (64, 0, 1 << 40))
    if what == "rope rows": C.rope_qkv(ctx, fake(2, 5, 1536)[:, :4], 1e4)
    if what == "rope elements": C.rope_qkv(ctx, fake(1, 4, 1536, 2)[..., 0], 1e4)
    if what == "rope parent": C.rope_qkv(ctx, fake(1, 4, 1536), 1e4, parent=fake(1, 5, dtype=i32), start=fake(1, 3, dtype=i32))
    if what == "rope start": C.rope_qkv(ctx, fake(1, 4, 1536), 1e4, start=fake(1, 2, dtype=i32))
    if what == "plan table": C.block_plan(ctx, None, None, fake(3, dtype=i32), None, fake(3, dtype=i32), None, 4)
    if what == "plan rows": C.block_plan(ctx, None, None, fake(3, 2, dtype=i32), None, fake(3, dtype=i32), None, -1)
    if what == "plan type": C.block_plan(ctx, None, None, fake(3, 2), None, fake(3, dtype=i32), None, 4)
    if what == "plan length": C.block_plan(ctx, fake(4, dtype=i32), None, fake(3, 2, dtype=i32), None, fake(3, dtype=i32), None, 4)
    if what == "write slots": C.kv_write_packed(ctx, None, None, fake(3, dtype=i32), None, None)
    if what == "write codes": C.kv_write_packed(ctx, None, None, fake(3, dtype=torch.int64), fake(1, 2, 5, 2, 128, 63, dtype=u8), None)
    if what == "write host": C.kv_write_packed(ctx, None, None, host(3).long(), None, None)
    if what == "append codes": C.kv_append_packed(ctx, fake(2, 2, 5, 2, 128, 64, dtype=u8), *[None] * 6)
    if what == "attention q": attention(fake(1, 4, 8, 128)[:, :, :4])
    if what == "attention type": attention(fake(1, 4, 8, 128, dtype=torch.float16))
    if what == "attention codes": attention(fake(1, 4, 8, 128), codes=fake(1, 2, 5, 2, 64, 64, dtype=u8))
    if what.startswith("good"):
        a = dict(q=fake(1, 4, 8, 128), codes=fake(1, 2, 5, 2, 128, 64, dtype=u8), scales=fake(1, 2, 5, 2, 128, 8, dtype=u8), block_table=fake(1, 6, dtype=i32),
                 tree_k=fake(1, 2, 4, 128), tree_v=fake(1, 2, 4, 128), parent=fake(1, 4, dtype=i32), prefix_len=fake(1, dtype=i32), out=fake(1, 4, 8, 128),
                 workspace=fake(9, dtype=u8))
        bad = dict(scales=fake(1, 2, 5, 2, 128, 4, dtype=u8), block_table=fake(6, dtype=i32), tree_k=fake(1, 4, 2, 128), tree_v=fake(1, 2, 5, 128),
                   parent=fake(4, dtype=i32), prefix_len=fake(2, dtype=i32), out=fake(1, 4, 8, 64), workspace=fake(9, dtype=i32))
        if what[5:]: a[what[5:]] = bad[what[5:]]
        attention(**a)
    print("returned")
except Exception as e:
    print(type(e).__name__, str(e).splitlines()[0] if str(e) else "")
"""


@pytest.mark.parametrize("what,kind,text", [
    ("rope host", "ValueError", "must live on cuda"), ("rope type", "TypeError", "expected BFloat16"), ("rope list", "TypeError", "expected a tensor"),
    ("rope theta", "TypeError", ""), ("rope width", "ValueError", "expected [batch][nodes][1536]"), ("rope dims", "ValueError", "expected"),
    ("rope sections", "TypeError", "arguments"), ("rope section", "OverflowError", "fit"), ("rope rows", "ValueError", "evenly spaced"),
    ("rope elements", "ValueError", "contiguous"), ("rope parent", "ValueError", "parent: expected shape (1, 4), got (1, 5)"),
    ("rope start", "ValueError", "start: expected shape (1, 3)"), ("plan table", "ValueError", "block_table"), ("plan rows", "ValueError", "max_rows"),
    ("plan type", "TypeError", "expected Int"), ("plan length", "ValueError", "length: expected shape (3), got (4)"), ("write slots", "TypeError", "expected Long"),
    ("write codes", "ValueError", "codes: expected shape (1, 2, 5, 2, 128, 64), got (1, 2, 5, 2, 128, 63)"), ("write host", "ValueError", "cuda"),
    ("append codes", "ValueError", "codes: expected shape (1, 2, 5, 2, 128, 64)"), ("attention q", "ValueError", "contiguous"),
    ("attention type", "TypeError", "expected BFloat16, got Half"), ("attention codes", "ValueError", "codes: expected shape"),
    ("good", "FspadError", ""),                          # (the NULL context)
    ("good scales", "ValueError", "scales: expected shape"), ("good block_table", "ValueError", "block_table: expected [batch][blocks]"),
    ("good tree_k", "ValueError", "tree_k: expected shape (1, 2, 4, 128), got (1, 4, 2, 128)"), ("good tree_v", "ValueError", "tree_v"),
    ("good parent", "ValueError", "parent: expected shape (1, 4), got (4)"), ("good prefix_len", "ValueError", "prefix_len"),
    ("good out", "ValueError", "out: expected shape"), ("good workspace", "TypeError", "workspace: expected Byte"),
])
def test_what_the_binding_refuses(what, kind, text):
    r = subprocess.run([sys.executable, "-c", SCRIPT, what], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
    assert r.stdout.startswith(kind) and "Error" in r.stdout and text in r.stdout, r.stdout
