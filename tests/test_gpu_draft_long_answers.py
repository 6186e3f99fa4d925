"""Passes over drafted tokens of plans that allow long answers: the work of a pass is sized for what the pages may come to hold, so
that these small batches take the kernels that otherwise only large ones take.  The checks and their bars are those of short answers."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import test_gpu_draft as short
from paper_2505_10951_amd import sgc

pytestmark = pytest.mark.gpu

LONG = 960


@pytest.fixture(autouse=True)
def long_answers(monkeypatch):
    start = short._start
    monkeypatch.setattr(short, "_start", lambda w, cap, rows, **kw: start(w, max(cap, LONG), rows, **kw))


@pytest.mark.parametrize("hq,hkv,R,kv", [
    (8, 2, 5, "bf16"), (8, 2, 5, "fp8_e4m3"), (4, 4, 1, "bf16"), (8, 8, 16, "bf16"), (12, 4, 7, "bf16"),
    (32, 2, 16, "bf16"), (32, 1, 3, "fp8_e4m3"), (64, 8, 4, "bf16"), (5, 1, 13, "bf16")])
def test_passes_match_oracle(hq, hkv, R, kv):
    short.test_passes_match_oracle(hq, hkv, R, kv, "mfma")


@pytest.mark.parametrize("prefix,queries,hq,hkv,R", [((5000, 90), 5, 64, 8, 16), ((2500, 1100, 70), 24, 32, 8, 5), ((300, 40), 40, 8, 2, 4), ((2300,), 7, 32, 2, 16)])
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_long_prompts_and_many_queries(prefix, queries, hq, hkv, R, kv):
    rng = np.random.default_rng(queries)
    w = short._workload(hq=hq, hkv=hkv, kv=kv, prefix=prefix, labels=[i % len(prefix) for i in range(queries)], suffix=rng.integers(0, 60, size=queries).tolist())
    gen = short._generated(w, R + 4)
    ref = short._oracle(w, gen)
    with short._start(w, R + 4, R) as s:
        for done, rows in ((np.zeros(queries, int), np.full(queries, R)), (rng.integers(0, 5, size=queries), rng.integers(0, R + 1, size=queries))):
            short._check(short._pass(s, gen, done, rows, R), ref, done, rows, short.TOL[kv])


def test_first_product_on_the_codes():
    w = short._workload(kv="fp8_e4m3", prefix=(4000, 2500), labels=[0, 1, 0, 0, 1], suffix=[14, 3, 40, 0, 21], hq=64, hkv=8)
    gen = short._generated(w, 20)
    ref = short._oracle(w, gen)
    with short._start(w, 20, 16, kernel=sgc.SGC_KERNEL_MFMA_FP8) as s:
        for done in ([0, 0, 0, 0, 0], [4, 2, 1, 0, 3]):
            short._check(short._pass(s, gen, done, None, 16), ref, done, [16] * 5, short.TOL["fp8_e4m3"])


@pytest.mark.parametrize("test", [
    short.test_layers_keep_their_own_pages, short.test_a_pass_of_one_row_is_a_decode_step,
    short.test_no_question_tokens_anywhere_and_no_queries, short.test_values_that_are_not_finite_stay_with_who_sees_them], ids=lambda f: f.__name__[5:])
def test_as_with_short_answers(test):
    test()


def test_captured_pass_replayed_with_counts_that_move(monkeypatch):
    start = short._start

    def warm(w, cap, rows, **kw):
        # the rotary table grows to the longest answer with the first call, and a capture would be refused
        s = start(w, cap, rows, **kw)
        none = np.zeros(w.n_queries, int)
        short._pass(s, short._generated(w, rows), none, none, rows)
        return s

    monkeypatch.setattr(short, "_start", warm)
    short.test_captured_pass_replayed_with_counts_that_move()
