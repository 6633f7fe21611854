"""Attention over the 4-bit cache on the GPU: parts of several stretches, and trees that are none, in each of the kernels."""
import pytest
import torch

from tests.test_gpu_packed_attn import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,nodes,heads,lens", [
    (80, 60, (8, 2), lambda b: (53 * b) % 400),          # one tile of 240 rows; parts of two stretches, and of three
    (40, 65, (8, 2), lambda b: (53 * b) % 400),          # tiles of 256 and 4 rows: stretches with one row tile and with two in one part
    (40, 130, (8, 2), lambda b: (53 * b) % 130),         # tiles of 256, 256 and 8
    (16, 65, (16, 8), lambda b: 1280 - 20 * b if b < 4 else (37 * b) % 500),      # fewer runs than parts, but too ragged for equal pieces of each
    (20, 60, (32, 8), lambda b: (97 * b) % 600)])        # up to 32 sequences, more runs than parts
def test_parts_of_several_stretches(batch, nodes, heads, lens):
    """(At 148 parts.)  What a stretch leaves in the query tiles, barriers and partials is met by the next one of the same CTA."""
    case = Case(34, batch, nodes, *heads, [lens(b) for b in range(batch)])
    ctx, args = case.context(), case.arguments()
    out = ctx.tree_attn_packed(*args)
    ctx.check()
    case.check(out)
    for _ in range(5):
        assert torch.equal(ctx.tree_attn_packed(*args), out)


@pytest.mark.parametrize("nodes,heads", [(4, (2, 2)), (7, (1, 1)), (20, (2, 2)), (16, (4, 2)), (5, (8, 2)), (60, (4, 2)), (200, (1, 1))])
def test_a_malformed_parent_is_reported_by_every_kernel(nodes, heads):
    case = Case(35, 2, nodes, *heads, [100, 0])
    ctx = case.context()
    want = ctx.tree_attn_packed(*case.arguments())
    ctx.check()
    for node, parent in ((0, 0), (1, -1), (1, 1), (nodes - 1, nodes), (nodes - 1, -7), (nodes // 2, nodes - 1), (2, 2 ** 31 - 1), (2, -2 ** 31), (0, 1)):
        args = case.arguments()
        args[6][1, node] = parent
        got = ctx.tree_attn_packed(*args)
        assert ctx.status() == -8, (node, parent)
        assert torch.equal(got[0], want[0])              # (the other tree)
    assert torch.equal(ctx.tree_attn_packed(*case.arguments()), want)
    ctx.check()
