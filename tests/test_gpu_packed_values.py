"""Attention over the 4-bit cache on the GPU where values are out of the ordinary, against the 64-bit definition."""
import numpy as np
import pytest
import torch

from oracle import packed
from paper_2408_15562_b200 import synth
from tests.test_gpu_packed_attn import Case, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nodes,heads", [(1, (4, 1)), (7, (2, 1)), (20, (8, 8)), (60, (8, 2)), (130, (1, 1)), (150, (2, 1))])
@pytest.mark.parametrize("lens", [[0, 77], [2500, 300]])
@pytest.mark.parametrize("size", [2.0 ** 121, 2.0 ** -100])
def test_tree_rows_of_v_of_any_magnitude(nodes, heads, lens, size):
    """V rows of the tree up to 2^125 (normal ones of deviation 2^121): the sums of the weighted rows are finite, and so is the result.  And small ones."""
    case = Case(31, 2, nodes, *heads, lens)
    x = np.clip(packed.bf16(case.tv), -16, 16) * size
    case.tv = synth.f32_to_bf16_bits(x.astype(np.float32))
    out = _run(case)
    assert torch.isfinite(out).all()
    case.check(out)
