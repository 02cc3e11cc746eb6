"""CPU-side checks of the state space operators' ranges: numbers of sequences and of tensors next to 2^31."""

import pytest

from paper_2510_12128_amd import binding as B
from test_sequence_host import lib  # noqa: F401
from test_state_space_host import conv, conv_calls


@pytest.mark.parametrize("n_seqs", [(1 << 31) - 1, (1 << 31) - 3, (1 << 31) - 4])
@pytest.mark.parametrize("dim", [64, 65536])
def test_windows_of_as_many_sequences_as_there_can_be(lib, n_seqs, dim):  # noqa: F811
    """A workgroup for every four windows is more than one launch holds."""
    p = conv(n_seqs=n_seqs, dim=dim, workspace_bytes=1 << 62)
    assert list(conv_calls(lib, p, s1=1 << 20)) == [B.NUGPR_ERR_INVALID, B.NUGPR_ERR_INVALID]
    assert b"too many" in lib.nugpr_last_error_string()
