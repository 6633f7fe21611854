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
