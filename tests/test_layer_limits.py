"""Sizes past what the layer operators hold are refused before any GPU work (addresses here are
never dereferenced).  Runs without a GPU."""
import paper_2606_16824_amd as cwlib
from paper_2606_16824_amd import _lib as L


def _tables(n):
    """cw_build_step_tables of n sequences without a workspace, its arrays 64 GiB apart."""
    a = [0x100000 + (i << 36) for i in range(9)]
    return cwlib.library().cw_build_step_tables(a[0], a[1], n, a[2], 10, 16, a[3], 1, 20, a[4], a[5], a[6], a[7], a[8], None, 0,
                                                None)


def test_step_tables_of_more_sequences_than_their_indexes_hold():
    """Their kernels add up to 1024 to a sequence's 32-bit index; near 2^31 that turned negative and
    would have read in front of the lengths."""
    for n in ((1 << 30) + 1, (1 << 31) - 1000, (1 << 31) - 1):
        assert _tables(n) == L.CW_ERR_BAD_LENS
        assert "num_seqs" in cwlib.library().cw_last_error_message().decode()
    assert _tables(1 << 30) == L.CW_ERR_WORKSPACE  # accepted so far
