"""Batches over a whole cluster of blocks whose lanes have different numbers of rows and pages to see to, at every kind of remainder."""
import numpy as np
import pytest

from test_gpu_cache_tables import Tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [8 * 1024 - 1, 8 * 1024 + 1, 8 * 8 * 1024 + 1, 2 * 8 * 8 * 1024 + 8 * 17 + 3])
def test_remainders(lib, rows):
    rng = np.random.default_rng(rows)
    cuts = np.sort(rng.integers(0, rows + 1, 6))
    new = np.diff(np.concatenate([[0], cuts, [rows]]))
    lens = rng.integers(0, 40, 7)
    t = Tables(lib, lens, -(-(int(new.max()) + 40) // 16), spare=rows // 16 + 20)
    for _ in range(2):
        t.rows_for(rows)
        t.extend(new)
        t.check_rows(*t.model_extend(new))
        t.check_state()
        t.trim(lens)
        t.model_trim(lens)
        t.check_state()
    assert int(t.err) == 0
    t.h.close()
