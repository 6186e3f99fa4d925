"""Passes whose long prompts are split into ranges that the last one sums: captured, replayed and eager in turn, two layers' graphs of one plan,
with tiles that have no rows in between.  Every pass against the oracle, and replays against eager passes bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import test_gpu_draft as base
from paper_2505_10951_amd.harness import to_device, to_host_f32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("hq,hkv,R,prefix,labels", [(8, 2, 5, (2500, 333), (0, 1, 0, 0, 1)), (32, 8, 16, (6100,), (0, 0)), (64, 8, 9, (2100, 900, 0), (0, 1, 2, 0))])
def test_replays_and_eager_passes_in_turn(hq, hkv, R, prefix, labels, kv):
    n, cap = len(labels), 2 * R + 3
    w = base._workload(hq=hq, hkv=hkv, kv=kv, prefix=prefix, labels=labels, suffix=[3 * i for i in range(n)], layers=2)
    gens = [base._generated(w, cap, layer) for layer in (0, 1)]
    refs = [base._oracle(w, g, layer) for layer, g in enumerate(gens)]
    rng = np.random.default_rng(R)
    with base._start(w, cap, R, layers=(0, 1)) as s:
        done, rows = base._i32(np.zeros(n)), base._i32(np.full(n, R))
        held, graphs = [], []
        for layer in (0, 1):
            q, k, v = (to_device(x, "bf16") for x in base._rows(gens[layer], np.zeros(n, int), R))
            o, lse = torch.full_like(q, 7.0), torch.full((hq, n * R), 7.0, device=base.DEV)
            s.draft_step(done, rows, q, k, v, layer, do=o, dlse=lse)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                s.draft_step(done, rows, q, k, v, layer, do=o, dlse=lse)
            held.append((q, k, v, o, lse)), graphs.append(g)
        at = np.zeros(n, int)
        for i in range(6):
            r = rng.integers(0, R + 1, size=n) if i % 3 else np.full(n, R)
            if i == 2:
                r[np.array(labels) == 0] = 0                 # a cluster without rows
            if i == 4:
                r[:] = 0                                     # nobody has any
            r = np.minimum(r, cap - at)
            for layer in (0, 1):
                q, k, v, o, lse = held[layer]
                for t, x in zip((q, k, v), base._rows(gens[layer], at, R)):
                    t.copy_(to_device(x, "bf16"))
                done.copy_(base._i32(at)), rows.copy_(base._i32(r)), o.fill_(7.0), lse.fill_(7.0)
                graphs[layer].replay()
                torch.cuda.synchronize()
                replayed = to_host_f32(o), lse.cpu().numpy().reshape(hq, n, R)
                base._check(replayed, refs[layer], at, r, base.TOL[kv], (i, layer))
                eager = base._pass(s, gens[layer], at, r, R, layer)
                assert np.array_equal(replayed[0], eager[0]) and np.array_equal(replayed[1], eager[1]), (i, layer)
            at = at + np.minimum(r, 2)
