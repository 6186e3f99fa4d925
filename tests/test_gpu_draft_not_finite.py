"""A key or value that is not finite, among the tokens of a pass or those that stand, reaches the rows that see it and no others: not the
rows in front of it, not those of other queries of the cluster, which a kernel works on together."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import test_gpu_draft as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [9, 960])          # one launch; the two launches of long answers
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("what,bad", [(2, np.inf), (2, np.nan), (1, np.nan), (2, -np.inf)])
@pytest.mark.parametrize("hq,hkv,R", [(8, 2, 4), (12, 4, 7)])
def test_only_rows_that_see_it(hq, hkv, R, kv, what, bad, cap):
    w = base._workload(hq=hq, hkv=hkv, kv=kv)
    n = w.n_queries
    gen = base._generated(w, R + 2)
    ref = base._oracle(w, gen)
    hurt = {0: 1, 3: R - 1, 4: 0}                  # query: the token whose key or value is spoilt, in one channel (two queries of a cluster among them)
    spoilt = [x.copy() for x in gen]
    for query, token in hurt.items():
        spoilt[what][token, query, :, 5] = bad
    with base._start(w, max(cap, R + 2), R) as s:
        def check(got, done, rows):
            o, lse = got
            for i in range(n):
                for j in range(rows[i]):
                    t = done[i] + j
                    if i in hurt and t >= hurt[i]:
                        assert not np.isfinite(o[i, j]).all(), (i, j)
                        if what == 2:               # a value spoils its channel, and nothing else
                            assert (~np.isfinite(o[i, j])).nonzero()[1].tolist() == [5] * hq
                            good = np.delete(np.arange(w.head_dim), 5)
                            assert np.abs(o[i, j][:, good] - ref[0][t, i][:, good]).max() <= base.TOL[kv]
                    else:
                        assert np.isfinite(o[i, j]).all() and np.abs(o[i, j] - ref[0][t, i]).max() <= base.TOL[kv], (i, j)
                        assert np.abs(lse[:, i, j] - ref[1][t, :, i]).max() <= 5e-2, (i, j)
        zero = np.zeros(n, int)
        full = np.full(n, R)
        check(base._pass(s, spoilt, zero, None, R), zero, full)
        # the spoilt tokens stand in their queries' pages; the other queries go on beside them
        done = np.full(n, 2)
        check(base._pass(s, spoilt, done, None, R), done, full)
