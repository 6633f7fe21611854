"""Outputs of the calls around the 4-bit cache that lie where other parts of the call still read or write are refused, on the host and with nothing launched."""
import pytest

from tests.test_packed_host_side import BATCH, ERR, HKV, LAYERS, NODES, lib, run  # noqa: F401  (lib: the fixture)

A, B, C, D, E = (0x1000000 * (i + 1) for i in range(5))      # aligned addresses with room between them


@pytest.mark.parametrize("change,refused", [
    (dict(new_len=C), True), (dict(new_len=D), True), (dict(new_len=C + 4), True), (dict(new_len=D + 4), True), (dict(new_len=C - 4), True),
    (dict(new_len=B), True), (dict(new_len=B + 2 * NODES * 4 - 4), True), (dict(block_table=E + 8, new_len=E + 4), True),
    (dict(new_len=E), False), (dict(new_len=B + 2 * NODES * 4), False), (dict(block_table=E + 8, new_len=E), False), (dict(new_len=C + 8), False), (dict(new_len=D - 8), False), (dict(new_len=None), False)])
def test_new_lengths_of_an_append(lib, change, refused):  # noqa: F811
    """Every warp of a sequence reads its prefix length and its count; one of them writes the new length."""
    rc, log = run(lib, "kv_append_packed", **{**dict(tree_kv=A, accepted_path=B, n_accepted=C, prefix_len=D, batch=2), **change})
    assert (rc, len(log)) == ((ERR["RANGE"], 0) if refused else (0, 1))


ROWS = 7 * HKV * 256                       # bytes of k, of v, and of what is kept of them


@pytest.mark.parametrize("k,v,kr,vr,refused", [
    (A, B, A, B, False), (A, B, C, D, False), (A, B, C, C + ROWS, False), (A, A, C, D, False), (A, A + ROWS, A, A + ROWS, False),
    (A, B, B, D, True), (A, B, C, A, True), (A, B, B, A, True), (A, B, C, C, True), (A, A, A, A, True), (A, A, A, C, True), (A, A, C, A, True),
    (A, B, A + 16, D, True), (A, B, C, B + 16, True), (A, B, C, C + ROWS - 16, True), (A, B, A + ROWS, D, False), (A, B, A, A + ROWS, False),
    (A, B, B + ROWS - 16, D, True), (A, B, A - 16, B, True)])
def test_kept_values_of_a_write(lib, k, v, kr, vr, refused):  # noqa: F811
    """K and V go at the same time: what is kept of one must not lie where the other is read or written, and in its own rows' place only row by row."""
    rc, log = run(lib, "kv_write_packed", k=k, v=v, k_rounded=kr, v_rounded=vr)
    assert (rc, len(log)) == ((ERR["RANGE"], 0) if refused else (0, 1))


KEPT = LAYERS * 2 * 2 * HKV * NODES * 256  # bytes of tree_kv for two sequences


@pytest.mark.parametrize("rounded,refused", [(A, False), (B, False), (A + KEPT, False), (A + 16, True), (A - 16, True), (A + KEPT - 16, True)])
def test_kept_values_of_an_append(lib, rounded, refused):  # noqa: F811
    rc, log = run(lib, "kv_append_packed", tree_kv=A, rounded=rounded)
    assert (rc, len(log)) == ((ERR["RANGE"], 0) if refused else (0, 1))
