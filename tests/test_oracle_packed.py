"""The 64-bit definitions around the 4-bit cache against torch's own types, brute force and hand-worked cases."""
import numpy as np
import torch

from oracle import packed
from paper_2408_15562_b200 import synth


def test_scales_and_codes_are_the_types_values():
    byte = torch.arange(127, dtype=torch.uint8)
    np.testing.assert_array_equal(packed.E4M3, byte.view(torch.float8_e4m3fn).double().numpy())
    bits = synth.normal_bf16(np.random.default_rng(0), (4000, 128))
    codes, scales, value = packed.quantise(bits)
    x = packed.bf16(bits).reshape(-1, 8, 16)
    most = torch.from_numpy(np.abs(x).max(-1)).float()
    want = (most / torch.full_like(most, 6.0)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(scales, want)
    # no other code of the type is nearer
    s = packed.E4M3[scales][..., None]
    every = np.concatenate([packed.E2M1, -packed.E2M1])
    best = np.abs(x[..., None] - s[..., None] * every).min(-1)
    np.testing.assert_array_equal(np.abs(x - value.reshape(x.shape)), best)


def test_ties_signs_and_ends():
    def bits(*v):
        t = torch.zeros(128)
        t[:len(v)] = torch.tensor(v)
        return t.to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)[None]

    # a scale of exactly one: thresholds go to the even code
    codes, scales, value = packed.quantise(bits(6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, -0.0))
    assert scales[0, 0] == 0x38 and value[0, :10].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -4]
    assert codes[0, :6].tolist() == [0x07, 0x22, 0x44, 0x66, 0xE8, 0x08] and np.signbit(value[0, 8]) and np.signbit(value[0, 10])
    # scales: a tie, the largest, below the smallest; blocks that are not finite
    assert packed.quantise(bits(6 * (1 + 1 / 16)))[1][0, 0] == 0x38 and packed.quantise(bits(6 * (1 + 3 / 16)))[1][0, 0] == 0x3A
    assert packed.quantise(bits(1e30))[1][0, 0] == 0x7E and packed.quantise(bits(1e30))[2][0, 0] == 2688
    codes, scales, value = packed.quantise(bits(6 * 2.0 ** -10))
    assert scales[0, 0] == 0 and not value.any()
    assert packed.quantise(bits(6 * 2.0 ** -9))[1][0, 0] == 1
    codes, scales, value = packed.quantise(bits(1.0, float("inf")))
    assert scales[0].tolist() == [0x7F] + [0] * 7 and np.isnan(value[0, :16]).all() and not codes.any()


def test_rope_turns_pairs_by_their_axis():
    rng = np.random.default_rng(1)
    qkv = synth.normal_bf16(rng, (2, 3, 4 * 128))
    pos = rng.integers(0, 10 ** 6, (2, 3, 3))
    q, k, v, _, _ = packed.rope(qkv, 2, 1, pos, 1e4, (10, 30, 24), False)
    x = packed.bf16(qkv).reshape(2, 3, 4, 128)
    for i, axis in ((0, 0), (9, 0), (10, 1), (39, 1), (40, 2), (63, 2)):
        a = pos[1, 2, axis] * 1e4 ** (-2 * i / 128)
        z = (x[1, 2, 1, i] + 1j * x[1, 2, 1, 64 + i]) * np.exp(1j * a)
        np.testing.assert_allclose([q[1, 2, 1, i], q[1, 2, 1, 64 + i]], [z.real, z.imag], rtol=1e-9, atol=1e-9)
    np.testing.assert_array_equal(v, x[:, :, 3:].swapaxes(1, 2))
    np.testing.assert_allclose(np.linalg.norm(k), np.linalg.norm(x[:, :, 2]), rtol=1e-12)
    adj = packed.rope(qkv.reshape(2, 3, 4, 2, 64).swapaxes(-1, -2).reshape(2, 3, -1), 2, 1, pos, 1e4, (10, 30, 24), True)[0]
    np.testing.assert_array_equal(adj[..., 0::2], q[..., :64])


def test_plan_by_hand():
    table = np.array([[4, 7, 0], [2, 0, 0]], np.int32)
    free = np.array([9, 8, 1, 0, 0], np.int32)
    r = packed.plan([130, 3], [200, 0], [0, 1], table, np.array([2, 1], np.int32), free, 3, 203)
    fits, row_start, slots, seq, pos, t, h, f, n = r
    assert fits and row_start.tolist() == [0, 200, 200]
    # sequence 1 gives block 2 back (9 8 1 2); sequence 0 pops it; sequence 1 takes one for its three rows
    assert t.tolist() == [[4, 7, 2], [1, 0, 0]] and h.tolist() == [3, 1] and n == 2 and f[:4].tolist() == [9, 8, 1, 2]
    assert slots[0] == 7 * 128 + 2 and slots[199] == 2 * 128 + 73 and slots[200:].tolist() == [-1] * 3
    assert seq[199] == 0 and pos[199] == 329 and seq[200] == -1
    assert not packed.plan([130, 3], [300, 0], None, table, h * 0 + [2, 1], free, 3, 300)[0]        # beyond the table
    assert not packed.plan([0, 0], [384, 384], None, table, h * 0, free, 3, 1000)[0]                # six blocks of three
    assert not packed.plan([0, 0], [1, 2], None, table, h * 0, free, 3, 2)[0]


def test_attention_is_a_softmax_over_what_a_node_sees():
    rng = np.random.default_rng(2)
    n_blocks, hkv, N, L = 3, 2, 5, 131
    codes = rng.integers(0, 256, (1, 2, n_blocks, hkv, 128, 64), np.uint8)
    scales = rng.integers(0x20, 0x38, (1, 2, n_blocks, hkv, 128, 8), np.uint8)
    scales[:, :, 0, :, 3:] = 0x7F                                        # behind the end
    table = np.array([[2, 0]], np.int32)
    q, tk, tv = (synth.normal_bf16(rng, s) for s in ((1, N, 4, 128), (1, hkv, N, 128), (1, hkv, N, 128)))
    tv[0, 1, 3] = 0x7FC0                                                 # a NaN that nodes 3 and 4 alone see
    parent = np.array([[-1, 0, 1, 0, 3]], np.int32)
    out, mass, size, _ = packed.tree_attn(q, codes, scales, 0, table, tk, tv, parent, [L])
    assert np.isnan(out[0, 3:, 2:]).all() and np.isfinite(out[0, :3]).all() and np.isfinite(out[0, :, :2]).all()
    for node, seen in ((0, [0]), (2, [0, 1, 2]), (4, [0, 3, 4])):
        k = np.concatenate([packed.rows_of(codes, scales, 0, 0, table[0], 0, L), packed.bf16(tk[0, 0, seen])])
        v = np.concatenate([packed.rows_of(codes, scales, 0, 1, table[0], 0, L), packed.bf16(tv[0, 0, seen])])
        w = np.exp(packed.bf16(q[0, node, 1]) @ k.T / np.sqrt(128))
        np.testing.assert_allclose(out[0, node, 1], w @ v / w.sum(), rtol=1e-10, atol=1e-12)
    assert (mass[0, :3] >= np.abs(out[0, :3])).all() and (size > 0).all()
