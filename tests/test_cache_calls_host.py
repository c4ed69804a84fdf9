"""What the cache and log-probability calls promise and refuse beyond single bad
arguments: workspaces kept for many calls, types of tensors, host lists, buffers
that share memory.  Nothing reaches a GPU; addresses are made up and every check
fails first."""

import ctypes as C

import pytest
import torch

import paper_2608_01821_amd as dv

EINVAL, ESHAPE, EDTYPE, ENOMEM = -1, -2, -3, -4
A = 1 << 20                                    # an aligned made-up address


@pytest.mark.parametrize("top", [0, 1, 5, 64])
@pytest.mark.parametrize("vocab", [1000, 16384, 32003, 126464, 1 << 24])
def test_a_log_probability_workspace_for_every_count_of_rows(vocab, top):
    """The header's bound for up to N rows, though fewer rows may need more."""
    most = 0
    for rows in range(1, 600):
        most = max(most, dv.davet_logprobs_workspace_bytes(rows, vocab, top))
        assert most <= (min(rows, 255) + 255) * (8 * top + 12)
    assert dv.davet_logprobs_workspace_bytes(1 << 22, vocab, top) <= most


def test_fewer_rows_than_the_workspace_was_asked_for():
    """255 rows are refused with what 256 need, which is nothing."""
    def f(rows, nb):
        return dv.raw().davet_token_logprobs(
            rows, 126464, A, dv.DAVET_F32, 126464, -1, A, A, None, 5, A, A, A, nb,
            None)
    assert dv.davet_logprobs_workspace_bytes(256, 126464, 5) == 0
    need = dv.davet_logprobs_workspace_bytes(255, 126464, 5)
    assert f(255, need - 1) == ENOMEM
    assert "%d bytes" % need in dv.raw().davet_last_error().decode()
