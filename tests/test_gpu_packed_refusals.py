"""Refused calls around the 4-bit cache on the GPU: what comes after them works."""
import numpy as np
import pytest
import torch

from paper_2408_15562_b200 import binding
from tests import helpers
from tests.test_gpu_packed_attn import Case

pytestmark = pytest.mark.gpu

dev = helpers.dev


@pytest.mark.parametrize("nodes", [1, 60])
def test_attention_after_a_refused_first_call(nodes):
    case = Case(41, 2, nodes, 8, 2, [300, 77])
    ctx, args = case.context(), case.arguments()
    for i, wrong in ((0, args[0].cpu()), (0, [1.0]), (4, args[4].cpu()), (7, args[7].cpu()), (3, args[3][:1])):
        with pytest.raises((TypeError, ValueError)):
            ctx.tree_attn_packed(*args[:i], wrong, *args[i + 1:])
    with pytest.raises(binding.FspadError):
        ctx.tree_attn_packed(*args, layer=1)
    out = ctx.tree_attn_packed(*args)
    ctx.check()
    case.check(out)
    kept = ctx._workspace.data_ptr()
    assert ctx._workspace.numel() >= ctx.tree_attn_packed_workspace_bytes(nodes, 2)
    assert torch.equal(ctx.tree_attn_packed(*args), out) and ctx._workspace.data_ptr() == kept


@pytest.mark.parametrize("nodes", [1, 60])
def test_a_first_call_that_is_captured(nodes):
    """Its workspace is made under the capture and lives on with the context."""
    case = Case(42, 2, nodes, 8, 2, [700, 77])
    args = case.arguments()
    want = case.context().tree_attn_packed(*args)
    ctx, out, graph = case.context(), torch.empty_like(want), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ctx.tree_attn_packed(*args, out=out)
    for _ in range(3):
        out.fill_(9)
        graph.replay()
        assert torch.equal(out, want)
    assert torch.equal(ctx.tree_attn_packed(*args), want)
    ctx.check()


def test_outputs_in_the_place_of_what_is_read():
    ctx = binding.Context(8, 2, 16, 512, max_nodes=4, n_layers=2, max_batch=2)
    codes, scales = ctx.new_packed_cache(3)
    tree = torch.ones((2, 2, 2, 2, 4, 128), dtype=torch.bfloat16, device="cuda")
    table, path, n, length = (dev(np.array(x, np.int32)) for x in ([[0], [1]], [[0, 1, -1, -1]] * 2, [2, 2], [5, 6]))
    for more in (dict(new_len=n), dict(new_len=length), dict(new_len=path.view(-1)[:2]), dict(new_len=table.view(-1))):
        with pytest.raises(binding.FspadError):
            ctx.kv_append_packed(codes, scales, table, tree, path, n, length, **more)
    k, v, slots = torch.ones((2, 5, 128), dtype=torch.bfloat16, device="cuda"), torch.ones((2, 5, 128), dtype=torch.bfloat16, device="cuda"), torch.arange(5, device="cuda")
    other = torch.empty_like(k)
    for kr, vr in ((v, k), (v, other), (other, k), (other, other)):
        with pytest.raises(binding.FspadError):
            ctx.kv_write_packed(k, v, slots, codes, scales, k_rounded=kr, v_rounded=vr)
    assert not codes.any() and not scales.any()
    ctx.kv_write_packed(k, v, slots, codes, scales, k_rounded=k, v_rounded=v)
    assert ctx.kv_append_packed(codes, scales, table, tree, path, n, length, rounded=tree).tolist() == [7, 8]
    ctx.check()
    # a block of ones has the scale 11/64, the e4m3 value nearest to 1/6 (10/64 is twice as far), and is kept as 6 * 11/64
    assert (k == 66 / 64).all() and (v == 66 / 64).all() and (tree[..., :2, :] == 66 / 64).all() and (tree[..., 2:, :] == 1).all()
