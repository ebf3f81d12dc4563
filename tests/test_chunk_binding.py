"""The binding of the chunk planner passes two arrays with one length: arrays that differ in length are refused, not read past
their end."""
import numpy as np
import pytest


@pytest.mark.parametrize("q_lens,seq_lens", [([1, 2, 3], [4, 5]), ([1], []), ([], [1]), ([[1, 2]], [[3, 4]]), (1, 2)])
def test_lengths_of_one_batch(lib, q_lens, seq_lens):
    with pytest.raises(ValueError):
        lib.libra_chunk_plan_host(148, 8, 2, q_lens, seq_lens)
    h = lib.Handle.__new__(lib.Handle)     # no GPU here: refused before the handle is used
    h._h = None
    with pytest.raises(ValueError):
        h.chunk_plan(np.asarray(q_lens, np.int32), np.asarray(seq_lens, np.int32), 256, 256, 0)


def test_equal_lengths_pass(lib):
    assert len(lib.libra_chunk_plan_host(148, 8, 2, [1, 2], [4, 5])["items"]) == 2
