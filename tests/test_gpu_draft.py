"""Passes over drafted tokens against the fp64 oracle: token t that a query generates is row suffix + t of the oracle's suffix prefill
over [question; generated tokens], whichever pass brought it.  Bars as for decode steps: 2e-2 (16-bit cache), 6e-2 (fp8)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import oracle as orc
from paper_2505_10951_amd import sgc, workloads
from paper_2505_10951_amd.harness import Session, to_device, to_host_f32
from ref_util import oracle_caches

pytestmark = pytest.mark.gpu

TOL = {"bf16": 2e-2, "fp8_e4m3": 6e-2}
DEV = "cuda:0"


def _workload(name="draft", hq=8, hkv=2, kv="bf16", prefix=(200, 71, 0), labels=(0, 1, 0, 2, 1, 0, 2), suffix=(14, 16, 1, 30, 0, 47, 5), layers=1, seed=5):
    return workloads.custom(name, n_q_heads=hq, n_kv_heads=hkv, head_dim=128, rope_base=500000.0, io_dtype="bf16", kv_dtype=kv, n_layers=layers,
                            prefix_len=list(prefix), labels=list(labels), suffix_len=list(suffix), seed=seed)


def _start(w, cap, rows, kernel=sgc.SGC_KERNEL_MFMA, layers=(0,)):
    s = Session(w, kernel=kernel)
    for c in range(w.n_clusters):
        s.alloc_cluster(c)
    for layer in layers:
        s.prefix_prefill_batched(list(range(w.n_clusters)), layer)
    s.assign()
    s.enable_drafts(cap, rows)
    s.upload_plan()
    for layer in layers:
        if w.total_suffix_tokens:
            s.suffix_prefill(*(to_device(x, "bf16") for x in w.suffix_qkv(layer)), layer=layer)
    return s


def _generated(w, n, layer=0):
    """q, k, v of n generated tokens of every query: [n][n_queries][heads][d]"""
    return [np.stack(x) for x in zip(*(w.decode_qkv(t, layer) for t in range(n)))]


def _oracle(w, gen, layer=0, caches=None):
    """o [tokens][n_queries][Hq][d], lse [tokens][Hq][n_queries] of the generated tokens"""
    caches = oracle_caches(w, layer) if caches is None else caches
    n = gen[0].shape[0]
    o, lse = np.zeros((n, w.n_queries, w.n_q_heads, w.head_dim)), np.zeros((n, w.n_q_heads, w.n_queries))
    for i in range(w.n_queries):
        S = int(w.suffix_len[i])
        x = [np.concatenate([a, g[:, i]]) for a, g in zip(w.suffix_qkv_query(i, layer), gen)]
        oo, ll, _ = orc.suffix_prefill(*caches[int(w.labels[i])], *x, w.rope_base)
        o[:, i], lse[:, :, i] = oo[S:], ll[:, S:].T
    return o, lse


def _rows(gen, done, R):
    """Rows of a pass: [n_queries][R] from gen at done + j (the last token there is where there are no more)"""
    n = gen[0].shape[0]
    at = np.minimum(np.asarray(done)[:, None].clip(0) + np.arange(R), n - 1)
    return [np.stack([g[at[i], i] for i in range(g.shape[1])]) for g in gen]


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _pass(s, gen, done, rows, R, layer=0):
    q, k, v = (to_device(x, "bf16") for x in _rows(gen, done, R))
    o, lse = torch.full_like(q, 7.0), torch.full((q.shape[2], q.shape[0] * R), 7.0, device=DEV)
    s.draft_step(_i32(done), None if rows is None else _i32(rows), q, k, v, layer, do=o, dlse=lse)
    torch.cuda.synchronize()
    return to_host_f32(o), lse.cpu().numpy().reshape(q.shape[2], q.shape[0], R)


def _check(got, ref, done, rows, tol, what=""):
    (o, lse), (o_ref, lse_ref) = got, ref
    for i, (d, r) in enumerate(zip(done, rows)):
        r = max(0, r)
        err = np.abs(o[i, :r] - o_ref[d:d + r, i]).max() if r else 0.0
        lerr = np.abs(lse[:, i, :r].T - lse_ref[d:d + r, :, i]).max() if r else 0.0
        assert np.isfinite(o[i, :r]).all() and err <= tol and lerr <= 5e-2, (what, i, err, lerr)
        assert (o[i, r:] == 7.0).all() and (lse[:, i, r:] == 7.0).all(), (what, i, "rows behind the last")


@pytest.mark.parametrize("hq,hkv,R,kv,kernel", [
    (8, 2, 5, "bf16", "mfma"), (8, 2, 5, "fp8_e4m3", "mfma"), (4, 4, 1, "bf16", "mfma"), (8, 8, 16, "bf16", "mfma"), (12, 4, 7, "bf16", "mfma"),
    (32, 2, 16, "bf16", "mfma"), (32, 1, 3, "fp8_e4m3", "mfma"), (64, 8, 4, "bf16", "mfma"), (5, 1, 13, "bf16", "mfma")])
def test_passes_match_oracle(hq, hkv, R, kv, kernel):
    w = _workload(hq=hq, hkv=hkv, kv=kv)
    rng = np.random.default_rng(R)
    gen = _generated(w, 3 * R + 2)
    ref = _oracle(w, gen)
    wrong = [x[::-1] * 1.5 for x in gen]                  # drafts that will be refused: their keys are overwritten
    with _start(w, 3 * R + 2, R) as s:
        done = np.zeros(w.n_queries, int)
        for p in range(3):
            rows = rng.integers(0, R + 1, size=w.n_queries) if p else np.full(w.n_queries, R)
            _pass(s, wrong, done, None, R)
            got = _pass(s, gen, done, rows if p else None, R)
            _check(got, ref, done, rows, TOL[kv], f"pass {p}")
            again = _pass(s, gen, done, rows if p else None, R)
            assert np.array_equal(got[0], again[0]) and np.array_equal(got[1], again[1])
            done = done + np.minimum(rows, rng.integers(0, R + 1, size=w.n_queries))


@pytest.mark.parametrize("prefix,queries,hq,hkv,R", [((2500, 1100, 70), 7, 8, 2, 5), ((300, 40), 40, 8, 2, 4), ((9000,), 1, 8, 1, 5), ((6200, 129), 3, 32, 2, 2)])
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_long_prompts_and_many_queries(prefix, queries, hq, hkv, R, kv):
    rng = np.random.default_rng(queries)
    w = _workload(hq=hq, hkv=hkv, kv=kv, prefix=prefix, labels=[i % len(prefix) for i in range(queries)], suffix=rng.integers(1, 60, size=queries).tolist())
    gen = _generated(w, R + 7)
    ref = _oracle(w, gen)
    with _start(w, R + 7, R) as s:
        first = np.full(w.n_queries, R)
        _check(_pass(s, gen, np.zeros(w.n_queries, int), None, R), ref, np.zeros(w.n_queries, int), first, TOL[kv])
        done = rng.integers(0, R + 1, size=queries)
        _check(_pass(s, gen, done, None, R), ref, done, first, TOL[kv])


def test_first_product_on_the_codes():
    w = _workload(kv="fp8_e4m3", prefix=(6000, 2500), labels=[0, 1, 0], suffix=[14, 3, 40])
    gen = _generated(w, 8)
    ref = _oracle(w, gen)
    with _start(w, 8, 4, kernel=sgc.SGC_KERNEL_MFMA_FP8) as s:
        for done in ([0, 0, 0], [4, 2, 1]):
            _check(_pass(s, gen, done, None, 4), ref, done, [4, 4, 4], TOL["fp8_e4m3"])


def test_layers_keep_their_own_pages():
    w = _workload(layers=2)
    gens = [_generated(w, 9, layer) for layer in (0, 1)]
    refs = [_oracle(w, g, layer) for layer, g in enumerate(gens)]
    n = w.n_queries
    with _start(w, 9, 4, layers=(0, 1)) as s:
        for done in (np.zeros(n, int), np.arange(n) % 5):
            for layer in (1, 0):
                _check(_pass(s, gens[layer], done, None, 4, layer), refs[layer], done, [4] * n, TOL["bf16"])


def test_counts_outside_the_pages_leave_everything_as_it_was():
    w = _workload()
    cap, R = 10, 4
    gen = _generated(w, cap)
    ref = _oracle(w, gen)
    n = w.n_queries
    with _start(w, cap, R) as s:
        for d in range(0, cap, 2):
            _pass(s, gen, np.full(n, d), np.full(n, 2), R)                          # all keys are there
        done = np.array([6, 7, 9, 10, 11, -1, 1 << 30])                              # of the last ones: 1, 0, 0, 0, 0 rows fit
        got = _pass(s, gen, done, None, R)
        fit = np.array([4, 3, 1, 0, 0, 0, 0])
        _check(got, ref, np.minimum(np.maximum(done, 0), cap), fit, TOL["bf16"])
        for rows in ([-3, 0, 1 << 30, -(1 << 31), 1, 2, 0],):
            d = np.full(n, 3)
            _check(_pass(s, gen, d, rows, R), ref, d, np.clip(rows, 0, R), TOL["bf16"])
        # nothing of that has touched keys that stand: the last tokens again
        _check(_pass(s, gen, np.full(n, 8), np.full(n, 2), R), ref, np.full(n, 8), np.full(n, 2), TOL["bf16"])


def test_a_pass_of_one_row_is_a_decode_step():
    w = _workload()
    gen = _generated(w, 5)
    ref = _oracle(w, gen)
    n = w.n_queries
    with _start(w, 6, 3) as s:
        _check(_pass(s, gen, np.zeros(n, int), None, 3), ref, np.zeros(n, int), [3] * n, TOL["bf16"])
        # a decode step behind three drafted tokens, then a pass behind that
        q, k, v = (to_device(x[3], "bf16") for x in gen)
        o = to_host_f32(s.decode_step(3, q, k, v))
        assert np.abs(o - ref[0][3]).max() <= TOL["bf16"]
        _check(_pass(s, gen, np.full(n, 4), np.full(n, 1), 3), ref, np.full(n, 4), [1] * n, TOL["bf16"])


def test_no_question_tokens_anywhere_and_no_queries():
    w = _workload(labels=[0, 1, 2], suffix=[0, 0, 0])
    gen = _generated(w, 6)
    ref = _oracle(w, gen)
    with _start(w, 6, 3) as s:
        for done in ([0, 0, 0], [3, 1, 2]):
            _check(_pass(s, gen, done, None, 3), ref, done, [3, 3, 3], TOL["bf16"])
    # a plan without queries: nothing to do, whatever the arguments
    with Session(w) as s:
        for c in range(w.n_clusters):
            s.alloc_cluster(c)
        s.assign(labels=[], suffix_len=[])
        s.enable_drafts(6, 3)
        s.upload_plan()
        sgc.sgc_draft_step_batched(s.ctx, s.cache, s.plan, 0, 0, None, 0, 0, 0, 0)


def test_clusters_allocated_elsewhere_meanwhile():
    # the page table moves when another cluster comes or goes; a capture may not refresh it
    w = _workload(prefix=(200, 71, 40), labels=(0, 1, 0, 1, 1, 0, 1))
    gen = _generated(w, 8)
    ref = _oracle(w, gen)
    n = w.n_queries
    with Session(w, total_pages=60, max_clusters=4) as s:
        for c in range(3):
            s.alloc_cluster(c)
        s.prefix_prefill_batched([0, 1, 2], 0)
        s.assign()
        s.enable_drafts(8, 4)
        s.suffix_prefill(*(to_device(x, "bf16") for x in w.suffix_qkv(0)))
        _check(_pass(s, gen, np.zeros(n, int), None, 4), ref, np.zeros(n, int), [4] * n, TOL["bf16"])
        s.free_cluster(2)
        sgc.sgc_cache_alloc_cluster(s.ctx, s.cache, 3, 100)
        q, k, v = (to_device(x, "bf16") for x in _rows(gen, np.full(n, 4), 4))
        d, o = _i32(np.full(n, 4)), torch.empty_like(q)
        torch.cuda.synchronize()
        with pytest.raises(sgc.SgcError) as e:
            with torch.cuda.graph(torch.cuda.CUDAGraph()):
                s.draft_step(d, None, q, k, v, do=o)
        assert e.value.status == sgc.SGC_ESTATE
        _check(_pass(s, gen, np.full(n, 4), None, 4), ref, np.full(n, 4), [4] * n, TOL["bf16"])


def test_values_that_are_not_finite_stay_with_who_sees_them():
    # refused drafts of infinite value lie in the pages behind the keys that stand; a later query's pass does not see them
    w = _workload()
    R, n = 4, w.n_queries
    gen = _generated(w, 8)
    ref = _oracle(w, gen)
    poison = [gen[0], gen[1], np.full_like(gen[2], np.inf)]
    with _start(w, 8, R) as s:
        _pass(s, poison, np.zeros(n, int), None, R)
        for done, rows in ((np.zeros(n, int), np.full(n, 1)), (np.ones(n, int), np.full(n, 2)), (np.full(n, 3), np.full(n, 4))):
            _check(_pass(s, gen, done, rows, R), ref, done, rows, TOL["bf16"])


def test_outputs_over_inputs_are_refused():
    w = _workload(labels=[0, 1, 2], suffix=[3, 4, 5])
    with _start(w, 6, 3) as s:
        q, k, v = (to_device(x, "bf16") for x in _rows(_generated(w, 6), [0, 0, 0], 3))
        for o in (q, k, v):
            with pytest.raises(sgc.SgcError) as e:
                s.draft_step(_i32([0, 0, 0]), None, q, k, v, do=o)
            assert e.value.status == sgc.SGC_EINVAL


def test_captured_pass_replayed_with_counts_that_move():
    w = _workload()
    R, n = 4, w.n_queries
    gen = _generated(w, 12)
    ref = _oracle(w, gen)
    with _start(w, 12, R) as s:
        side = torch.cuda.Stream()
        q, k, v = (to_device(x, "bf16") for x in _rows(gen, np.zeros(n, int), R))
        o, lse = torch.full_like(q, 7.0), torch.full((w.n_q_heads, n * R), 7.0, device=DEV)
        done, rows = _i32(np.zeros(n)), _i32(np.full(n, R))
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            s.draft_step(done, rows, q, k, v, do=o, dlse=lse)
        at = np.zeros(n, int)
        rng = np.random.default_rng(3)
        for _ in range(4):
            r = np.minimum(rng.integers(1, R + 1, size=n), 12 - at)
            for t, x in zip((q, k, v), _rows(gen, at, R)):
                t.copy_(to_device(x, "bf16"))
            done.copy_(_i32(at)), rows.copy_(_i32(r)), o.fill_(7.0), lse.fill_(7.0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            replayed = to_host_f32(o), lse.cpu().numpy().reshape(w.n_q_heads, n, R)
            _check(replayed, ref, at, r, TOL["bf16"])
            eager = _pass(s, gen, at, r, R)
            assert np.array_equal(replayed[0], eager[0]) and np.array_equal(replayed[1], eager[1])
            at = at + np.minimum(r, 2)
