"""Passes over clusters of more queries than a wavefront counts at once, with counts that leave whole stretches of queries without rows."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import test_gpu_draft as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("queries,hq,hkv,R,cap", [(200, 8, 2, 3, 8), (321, 4, 1, 2, 5), (130, 8, 8, 1, 300), (193, 16, 2, 4, 6)])
def test_rows_are_found_wherever_they_are(queries, hq, hkv, R, cap):
    rng = np.random.default_rng(queries)
    labels = np.where(np.arange(queries) % 5 == 4, 1, 0)
    w = base._workload(hq=hq, hkv=hkv, prefix=(150, 70), labels=labels.tolist(), suffix=rng.integers(0, 20, size=queries).tolist())
    gen = base._generated(w, 2 * R)
    ref = base._oracle(w, gen)
    full = np.full(queries, R)
    with base._start(w, cap, R) as s:
        zero = np.zeros(queries, int)
        base._check(base._pass(s, gen, zero, None, R), ref, zero, full, base.TOL["bf16"])
        patterns = [rng.integers(0, R + 1, size=queries), np.where(np.arange(queries) < 70, 0, R), np.where(np.arange(queries) < queries - 3, 0, R),
                    np.where(np.arange(queries) % 67 == 5, 1, 0), np.where(np.arange(queries) < 66, R, 0)]
        for rows in patterns:
            done = rng.integers(0, R + 1, size=queries)
            done[0] = 0
            # (the last case's pages have room for 6 tokens: rows behind them are left as they were)
            base._check(base._pass(s, gen, done, rows, R), ref, done, np.minimum(rows, cap - done), base.TOL["bf16"])
