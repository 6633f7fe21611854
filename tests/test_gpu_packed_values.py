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


@pytest.mark.parametrize("nodes,group", [(1, 2), (7, 2), (20, 1), (60, 4), (130, 1)])
@pytest.mark.parametrize("lens", [[0, 0], [150, 1300]])
def test_one_infinite_element_of_a_tree_row_of_k(nodes, group, lens):
    """It acts through the score: where that is +infinity or no number the output is NaN, where it is -infinity the row has no weight, and who does not
    see it does not notice."""
    case = Case(32, 2, nodes, 2 * group, 2, lens)
    case.q[:, :, :, 5] |= 0x0080                       # (no zeros there: an infinity times one is no number)
    where, sign = nodes // 2, (0x7F80, 0xFF80)
    plain = case.tk.copy()
    for b in range(2):
        for h in range(2):
            case.tk[b, h, where, 5] = sign[(b + h) % 2]
    got = _run(case).float().cpu().numpy().astype(np.float64)

    def definition(tk):
        with np.errstate(invalid="ignore"):
            return packed.tree_attn(case.q, case.codes, case.scales, 0, case.table, tk, case.tv, case.parent, case.L)

    want, mass, _, all_v = definition(case.tk)
    odd = np.isnan(want)
    np.testing.assert_array_equal(np.isnan(got), odd)
    assert odd.any() and (nodes == 1 and lens[0] == 0 or not odd.all())
    # the others by `Case.check`'s bound; the magnitudes of the scores are those of finite rows (with the infinite one they would be infinite, but it has no weight)
    size = definition(plain)[2]
    bound = np.abs(want) * 2.0 ** -8 + (mass * (2.0 ** -8 + 2.0 ** -12 + 2.0 ** -15 * size[..., None]) + 2.0 ** -32 * all_v) * (1 + 2.0 ** -8)
    assert (np.abs(got - want) <= bound)[~odd].all()


@pytest.mark.parametrize("nodes,group", [(1, 2), (20, 1), (60, 4), (130, 1)])
def test_a_cached_row_of_k_that_is_no_number_is_seen_by_all_of_its_sequence(nodes, group):
    case = Case(33, 2, nodes, 2 * group, 2, [150, 700])
    case.scales[0, 0, case.table[1, 4], 1, 30, 6] = 0x7F
    got = _run(case).float().cpu().numpy()
    want = np.zeros(got.shape, bool)
    want[1, :, group:] = True
    np.testing.assert_array_equal(np.isnan(got), want)


@pytest.mark.parametrize("nodes,heads", [(1, (4, 2)), (20, (2, 2)), (60, (4, 2)), (130, (4, 2))])
def test_cached_v_of_the_least_and_the_largest_scales(nodes, heads):
    """Kept values from 2^-10 (fp16's least one, with the factor that the sums take) to 2688, a kv head of each kind."""
    case = Case(36, 2, nodes, *heads, [900, 130])
    real = case.scales != 0x7F
    case.codes[:, 1] = case.rng.integers(0, 256, case.codes[:, 1].shape, np.uint8)
    for h, (lo, hi) in enumerate(((1, 9), (118, 127))):
        s = case.rng.integers(lo, hi, case.scales[:, 1, :, h].shape).astype(np.uint8)
        case.scales[:, 1, :, h] = np.where(real[:, 1, :, h], s, 0x7F)
    case.tv[:, 0] = synth.f32_to_bf16_bits((packed.bf16(case.tv[:, 0]) * 2.0 ** -8).astype(np.float32))
    case.check(_run(case))
