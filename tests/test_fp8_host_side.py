"""What the operators around the 8-bit cache and on blocks refuse, and in which order: api_fp8.cu compiled for the CPU against stand-ins for the device and the
launchers (`fp8_fake.cpp`).  What is refused launches nothing.  The binding's own refusals run in processes of their own, as no device is needed."""
import ctypes
import os
import re
import subprocess
import sys

import pytest

from paper_2408_15562_b200 import binding
from tests.test_packed_host_side import ERR

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2408_15562_b200", "csrc")
NULL, CUDA, TREE, SHAPE, ALIGN, RANGE, LARGE, DEVICE = "NULL", "CUDA", "TREE_TOO_LARGE", "SHAPE", "ALIGN", "RANGE", "TOO_LARGE", "DEVICE"
HQ, HKV, NODES, LAYERS, BATCH = 8, 2, 64, 3, 2000
P = [0x100000 * (i + 1) for i in range(16)]      # 16-byte aligned addresses that nothing reads, far apart
ODD = 0x100008


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fp8_host_side") / "libfp8host.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic",
                           "-DatomicCAS(p,a,b)=((void)(p),(void)(a),(void)(b))",
                           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-I/usr/local/cuda/include",
                           "-x", "c++", os.path.join(CSRC, "api_fp8.cu"), os.path.join(HERE, "fp8_fake.cpp"), "-o", out])
    lib = ctypes.CDLL(out)
    vp, ci, cl = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    lib.fake_context.restype = vp
    lib.fake_log.restype = ctypes.c_char_p
    lib.fake_context_free.argtypes = [vp]
    lib.fspad_kv_write_fp8.argtypes = [vp] * 4 + [ci, ci, vp, vp, ci, vp, vp, vp]
    lib.fspad_kv_append_fp8.argtypes = [vp] * 4 + [ci, ci] + [vp] * 4 + [ci, ci, vp, vp, vp]
    lib.fspad_tree_attn_fp8_workspace_bytes.argtypes = [vp]
    lib.fspad_tree_attn_fp8_workspace_bytes.restype = ctypes.c_size_t
    lib.fspad_tree_attn_fp8.argtypes = [vp] * 4 + [ci, vp, ci, ci] + [vp] * 4 + [ci, ci, vp, vp, ctypes.c_size_t, vp]
    lib.fspad_block_fork.argtypes = [vp] * 3 + [ci, vp, ci, ci, ci] + [vp] * 7
    lib.fspad_block_free.argtypes = [vp] * 2 + [ci] * 3 + [vp] * 6
    lib.fspad_block_compact.argtypes = [vp] + [ci] * 3 + [vp] * 6 + [ci, vp]
    lib.fspad_block_copy.argtypes = [vp, vp, cl, vp, cl, ci, ci, vp, ci, vp]
    lib.ctx = lib.fake_context(HQ, HKV, NODES, LAYERS, BATCH)
    yield lib
    lib.fake_context_free(lib.ctx)


POOL = dict(batch=5, blocks_per_seq=4, n_blocks=9, block_table=P[0], held=P[1], shares=P[2], free_blocks=P[3], n_free=P[4])
# the arguments of each call, in order, with values that are accepted
CALLS = {
    "kv_write_fp8": dict(k=P[0], v=P[1], slots=P[2], rows=7, layer=2, codes=P[3], scales=P[4], n_blocks=9, k_rounded=None, v_rounded=None, stream=None),
    "kv_append_fp8": dict(codes=P[0], scales=P[1], block_table=P[2], blocks_per_seq=4, n_blocks=9, tree_kv=P[3], accepted_path=P[4], n_accepted=P[5], prefix_len=P[6],
                          n_nodes=NODES, batch=2, rounded=None, new_len=None, stream=None),
    "tree_attn_fp8": dict(q=P[0], codes=P[1], scales=P[2], layer=1, block_table=P[3], blocks_per_seq=4, n_blocks=9, tree_k=P[4], tree_v=P[5], parent=P[6],
                          prefix_len=P[7], n_nodes=NODES, batch=2, out=P[8], workspace=P[9], workspace_bytes=128000, stream=None),
    "block_fork": dict(src=P[5], dst=P[6], n=2, len=P[7], **POOL, pairs=P[8], stream=None),
    "block_free": dict(drop=P[5], **POOL, stream=None),
    "block_compact": dict(**POOL, pairs=P[5], max_pairs=4, stream=None),
    "block_copy": dict(pool=P[0], block_bytes=32768, pool2=P[1], block_bytes2=32, planes=6, n_blocks=9, pairs=P[2], n_pairs=3, stream=None),
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
STATE = BLOCKS + [(dict(batch=-1), SHAPE), (dict(batch=BATCH + 1), SHAPE), (dict(batch=1025), LARGE), (dict(n_blocks=(1 << 19) + 1), LARGE)] + \
    [({n: None}, NULL) for n in ("block_table", "held", "shares", "free_blocks", "n_free")] + \
    [({a: P[b]}, RANGE) for a, b in (("held", 0), ("shares", 0), ("free_blocks", 1), ("n_free", 2), ("block_table", 3))] + \
    [(dict(held=P[0] + 4 * 5 * 4 - 4), RANGE), (dict(n_free=P[3] + 32), RANGE)]


def _null(*names):
    return [({n: None}, NULL) for n in names]


def _odd(*names):
    return [({n: ODD}, ALIGN) for n in names]


ROWS = 7 * HKV * 256
TREE_KV = LAYERS * 2 * 2 * HKV * NODES * 256
REFUSED = {
    "kv_write_fp8": _null("k", "v", "slots", "codes", "scales") + _odd("k", "v", "codes", "scales") + [
        (dict(k_rounded=P[5]), NULL), (dict(v_rounded=P[5]), NULL), (dict(k_rounded=ODD, v_rounded=P[5]), ALIGN), (dict(k_rounded=P[5], v_rounded=ODD), ALIGN),
        (dict(rows=-1), SHAPE), (dict(layer=-1), SHAPE), (dict(layer=LAYERS), SHAPE), (dict(n_blocks=0), SHAPE), (dict(rows=1 << 29), LARGE),
        (dict(k_rounded=P[1], v_rounded=P[5]), RANGE), (dict(k_rounded=P[5], v_rounded=P[0]), RANGE), (dict(k_rounded=P[5], v_rounded=P[5]), RANGE),
        (dict(k_rounded=P[0] + 16, v_rounded=P[1]), RANGE), (dict(k_rounded=P[0], v_rounded=P[1] + ROWS - 16), RANGE)],
    "kv_append_fp8": _null("codes", "scales", "block_table", "tree_kv", "accepted_path", "n_accepted", "prefix_len") +
        _odd("codes", "scales", "tree_kv", "rounded") + TREE_SIZES + BLOCKS + [({"new_len": P[i]}, RANGE) for i in (2, 4, 5, 6)] +
        [(dict(new_len=P[4] + 4 * NODES * 2 - 4), RANGE), (dict(new_len=P[2] + 4 * 4 * 2 - 4), RANGE), (dict(rounded=P[3] + 16), RANGE), (dict(rounded=P[3] + TREE_KV - 16), RANGE)],
    "tree_attn_fp8": _null("q", "codes", "scales", "block_table", "tree_k", "tree_v", "parent", "prefix_len", "out", "workspace") +
        _odd("q", "codes", "scales", "tree_k", "tree_v", "out", "workspace") + TREE_SIZES + BLOCKS + [
        (dict(layer=-1), SHAPE), (dict(layer=LAYERS), SHAPE), (dict(workspace_bytes=127999), RANGE), (dict(fits=0), LARGE)] + [(dict(out=P[i]), RANGE) for i in (0, 4, 5)],
    "block_fork": _null("src", "dst", "len", "pairs") + STATE + [(dict(n=-1), SHAPE), (dict(n=6), SHAPE)] +
        [({a: P[b]}, RANGE) for a in ("src", "dst", "len", "pairs") for b in range(5)] +
        [(dict(pairs=P[5]), RANGE), (dict(pairs=P[6]), RANGE), (dict(pairs=P[7]), RANGE), (dict(len=P[5]), RANGE), (dict(len=P[6]), RANGE)],
    "block_free": _null("drop") + STATE + [(dict(drop=P[b]), RANGE) for b in range(5)],
    "block_compact": _null("pairs") + STATE + [(dict(max_pairs=-1), SHAPE), (dict(max_pairs=10), SHAPE)] + [(dict(pairs=P[b]), RANGE) for b in range(5)],
    "block_copy": _null("pool", "pool2", "pairs") + _odd("pool", "pool2") + [(dict(pairs=0x100004), ALIGN), (dict(block_bytes=0), SHAPE), (dict(block_bytes=24), SHAPE),
        (dict(block_bytes=-16), SHAPE), (dict(block_bytes2=24), SHAPE), (dict(block_bytes2=-16), SHAPE), (dict(block_bytes2=0), NULL), (dict(planes=0), SHAPE),
        (dict(n_blocks=0), SHAPE), (dict(n_pairs=-1), SHAPE), (dict(block_bytes=1 << 41), LARGE), (dict(block_bytes2=1 << 41), LARGE),
        (dict(block_bytes=1 << 40, n_blocks=1 << 20), LARGE)],
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


def test_nothing_to_do_launches_nothing_but_pairs_are_written(lib):
    for name in ("kv_append_fp8", "tree_attn_fp8", "block_free"):
        assert run(lib, name, batch=0) == (0, [])
    assert run(lib, "kv_write_fp8", rows=0) == (0, [])
    assert run(lib, "block_fork", n=0) == (0, []) and run(lib, "block_fork", n=0, batch=0) == (0, [])
    assert run(lib, "block_copy", n_pairs=0) == (0, [])
    assert run(lib, "block_compact", batch=0) == (0, ["compact 0 4 9 4 0"])


def test_what_the_launchers_get(lib):
    heads = 9 * HKV                                      # of a layer's K or V
    k, s = P[1] + 2 * heads * 16384, P[2] + 2 * heads * 16
    assert run(lib, "tree_attn_fp8", stream=7)[1] == [f"attention {k} {s} {k + heads * 16384} {s + heads * 16} 64 2 7"]
    nb = 1 << 21                                         # offsets of a layer beyond 32 bits
    heads = nb * HKV
    k, s = P[1] + 4 * heads * 16384, P[2] + 4 * heads * 16
    assert run(lib, "tree_attn_fp8", n_blocks=nb, layer=2)[1] == [f"attention {k} {s} {k + heads * 16384} {s + heads * 16} 64 2 0"]
    assert run(lib, "kv_write_fp8", k_rounded=P[0], v_rounded=P[1], stream=5)[1] == ["write 7 2 9 5"]
    assert run(lib, "kv_append_fp8", rounded=P[3])[1] == ["append 4 9 64 2 0"]
    assert run(lib, "block_copy", pool2=None, block_bytes2=0, block_bytes=1 << 33)[1] == [f"copy {1 << 33} 0 6 9 3 0"]
    assert lib.fspad_tree_attn_fp8_workspace_bytes(lib.ctx) == 128000 and lib.fspad_tree_attn_fp8_workspace_bytes(None) == 0


def test_every_declared_name_with_a_digit_is_bound():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "fspad.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(fspad_[a-z0-9_]+)\s*\(", src)))
    assert names == sorted(binding.EXPORTS + binding.EXPORTS_FP8)
    lib = binding.load()
    for n in names:
        assert hasattr(lib, n), n


SCRIPT = """
import ctypes, sys, types
import torch
from paper_2408_15562_b200 import binding
what = sys.argv[1]
bf, i32, u8, i64, f32 = torch.bfloat16, torch.int32, torch.uint8, torch.int64, torch.float32
ctx = types.SimpleNamespace(_h=ctypes.c_void_p(), _sizes=(8, 2, 1, 4))
ctx._packed_call = lambda *a: binding.Context._packed_call(ctx, *a)
binding._stream = lambda s: 0
C = binding.Context
def fake(*shape, dtype=bf, at="cuda:0"):
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode(): return torch.empty(shape, dtype=dtype, device=at)
def ints(*shape): return fake(*shape, dtype=i32)
codes, scales = lambda: fake(1, 2, 5, 2, 128, 128, dtype=u8), lambda: fake(1, 2, 5, 2, 4, dtype=f32)
def attention(**kw):
    a = dict(q=fake(1, 4, 8, 128), codes=codes(), scales=scales(), block_table=ints(1, 6), tree_k=fake(1, 2, 4, 128), tree_v=fake(1, 2, 4, 128), parent=ints(1, 4),
             prefix_len=ints(1), out=fake(1, 4, 8, 128), workspace=fake(9, dtype=u8))
    a.update(kw)
    return C.tree_attn_fp8(ctx, **a)
def write(**kw):
    a = dict(k=fake(2, 3, 128), v=fake(1, 2, 3, 128), slots=fake(3, dtype=i64), codes=codes(), scales=scales(), k_rounded=fake(2, 3, 128), v_rounded=fake(2, 3, 128))
    a.update(kw)
    return C.kv_write_fp8(ctx, **a)
def append(**kw):
    a = dict(codes=codes(), scales=scales(), block_table=ints(3, 6), tree_kv=fake(1, 2, 3, 2, 4, 128), accepted_path=ints(3, 4), n_accepted=ints(3), prefix_len=ints(3),
             rounded=fake(1, 2, 3, 2, 4, 128), new_len=ints(3))
    a.update(kw)
    return C.kv_append_fp8(ctx, **a)
state = lambda: dict(block_table=ints(3, 6), held=ints(3), shares=ints(9), free_blocks=ints(9), n_free=ints(1))
def fork(**kw): return C.block_fork(ctx, **{**dict(src=ints(2), dst=ints(2), length=ints(3), pairs=ints(2, 2)), **state(), **kw})
def drop(**kw): return C.block_free(ctx, **{**dict(drop=ints(3)), **state(), **kw})
def compact(**kw): return C.block_compact(ctx, **{**dict(pairs=ints(4, 2)), **state(), **kw})
def copy(pool=None, pairs=None): return C.block_copy(ctx, (codes(), scales()) if pool is None else pool, ints(3, 2) if pairs is None else pairs)
host = torch.zeros(3)
try:
    print("returned", eval(what))
except Exception as e:
    print(type(e).__name__, str(e).splitlines()[0] if str(e) else "")
"""


@pytest.mark.parametrize("what,kind,text", [
    ("attention()", "FspadError", ""), ("write()", "FspadError", ""), ("append()", "FspadError", ""), ("fork()", "FspadError", ""), ("drop()", "FspadError", ""),
    ("compact()", "FspadError", ""), ("copy()", "FspadError", ""),                       # (the NULL context)
    ("attention(q=host)", "TypeError", "q: expected BFloat16, got Float"), ("attention(q=fake(1, 4, 8, 128, at='cpu'))", "ValueError", "must live on cuda"),
    ("attention(q=fake(1, 4, 9, 128)[:, :, :8])", "ValueError", "contiguous"), ("attention(q=fake(1, 4, 7, 128))", "ValueError", "q: expected shape (1, 4, 8, 128)"),
    ("attention(codes=fake(1, 2, 5, 2, 128, 64, dtype=u8))", "ValueError", "codes: expected shape (1, 2, 5, 2, 128, 128), got (1, 2, 5, 2, 128, 64)"),
    ("attention(scales=fake(1, 2, 5, 2, 8, dtype=f32))", "ValueError", "scales: expected shape (1, 2, 5, 2, 4)"), ("attention(scales=fake(1, 2, 5, 2, 4))", "TypeError", "scales"),
    ("attention(block_table=ints(6))", "ValueError", "block_table"), ("attention(tree_k=fake(1, 4, 2, 128))", "ValueError", "tree_k"), ("attention(tree_v=fake(1, 2, 5, 128))", "ValueError", "tree_v"),
    ("attention(parent=ints(4))", "ValueError", "parent"), ("attention(prefix_len=ints(2))", "ValueError", "prefix_len"), ("attention(out=fake(1, 4, 8, 64))", "ValueError", "out"),
    ("attention(workspace=ints(9))", "TypeError", "workspace"), ("attention(layer=1 << 40)", "OverflowError", "fit"),
    ("write(slots=ints(3))", "TypeError", "slots: expected Long"), ("write(slots=fake(3, 1, dtype=i64))", "ValueError", "slots"), ("write(k=fake(2, 4, 128))", "ValueError", "k: expected shape (2, 3, 128)"),
    ("write(v_rounded=fake(2, 4, 128))", "ValueError", "v_rounded"), ("write(codes=host)", "TypeError", "codes"),
    ("append(tree_kv=fake(1, 2, 3, 2, 4, 64))", "ValueError", "tree_kv"), ("append(accepted_path=ints(3, 5))", "ValueError", "accepted_path: expected shape (3, 4), got (3, 5)"),
    ("append(n_accepted=ints(2))", "ValueError", "n_accepted"), ("append(rounded=fake(1, 2, 3, 2, 5, 128))", "ValueError", "rounded"), ("append(new_len=ints(2))", "ValueError", "new_len"),
    ("fork(src=fake(2))", "TypeError", "src"), ("fork(dst=ints(3))", "ValueError", "dst: expected shape (2), got (3)"), ("fork(length=ints(2))", "ValueError", "length"),
    ("fork(pairs=ints(3, 2))", "ValueError", "pairs"), ("fork(held=ints(2))", "ValueError", "held"), ("fork(shares=ints(8))", "ValueError", "shares: expected shape (9), got (8)"),
    ("fork(n_free=ints(2))", "ValueError", "n_free"), ("fork(free_blocks=ints(9, 1))", "ValueError", "free_blocks"), ("fork(src=ints(2, 1))", "ValueError", "src"),
    ("drop(drop=ints(2))", "ValueError", "drop"), ("drop(block_table=ints(3))", "ValueError", "block_table"), ("compact(pairs=ints(4, 3))", "ValueError", "pairs"),
    ("copy(pool=codes(), pairs=ints(3, 3))", "ValueError", "pairs"), ("copy(pool=host)", "ValueError", "pool"), ("copy(pool=(codes(), fake(1, 2, 6, 4, dtype=f32)))", "ValueError", "pool"),
    ("copy(pool=fake(2, 2, 5, 4))", "ValueError", "pool"), ("copy(pool=[1])", "TypeError", "pool"),
])
def test_what_the_binding_refuses(what, kind, text):
    r = subprocess.run([sys.executable, "-c", SCRIPT, what], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
    assert r.stdout.startswith(kind) and "Error" in r.stdout and text in r.stdout, r.stdout
