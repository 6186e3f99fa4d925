"""Verification of numbers of queries and lengths of rows where the kernels change hands, against the definition in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_draft_head import _same, _verify, _verify_ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,R,V", [(3, 2, 2047), (3, 2, 4096), (700, 2, 4095), (700, 2, 4097), (300, 2, 12287), (300, 3, 12289), (1100, 2, 9001), (2100, 2, 5000), (66000, 2, 33)])
@pytest.mark.parametrize("with_q", [False, True])
def test_verification(n, R, V, with_q):
    rng = np.random.default_rng(n + V)
    # weights that are not normalised, a twentieth of them large and a third nothing: multiples of 2^-20, whose sums in 64 bits are exact in any order
    p = rng.integers(0, 1 << 12, size=(n, R, V)).astype(np.float32)
    p[rng.random((n, R, V)) < 0.05] *= 64
    p[rng.random((n, R, V)) < 0.3] = 0
    q = np.roll(p[:, : R - 1], 1, axis=2) * np.float32(0.75)
    p, q = p * np.float32(2.0 ** -20), (q * np.float32(2.0 ** -20)).astype(np.float32)
    tokens = rng.integers(0, V, size=(n, R))
    u = rng.random((n, R)).astype(np.float32)
    u[:, R - 1][rng.random(n) < 0.1] = np.float32(1 - 2.0 ** -24)
    p[1] = 0                                             # no weight anywhere
    if n > 2:
        p[2], p[2, :, V - 1] = 0, np.float32(0.5)        # all of it on the last token
    rows, done = rng.integers(0, R + 1, size=n), rng.integers(0, 9, size=n)
    _same(_verify(p, q if with_q else None, tokens, rows, u, done, pad=V % 3), _verify_ref(p, q if with_q else None, tokens, rows, u, done))


def test_drafts_that_cover_the_target_leave_its_own_row():
    # the draft says twice what the target says, everywhere: refused by a large number, the token behind comes from the target's own row
    for n, V in ((2, 40000), (900, 9000)):
        rng = np.random.default_rng(V)
        p = rng.integers(1, 1 << 10, size=(n, 2, V)).astype(np.float32) * np.float32(2.0 ** -24)
        q = p[:, :1] * np.float32(2)
        tokens, u = rng.integers(0, V, size=(n, 2)), rng.random((n, 2)).astype(np.float32)
        rows, done = np.full(n, 2), np.zeros(n, int)
        _same(_verify(p, q, tokens, rows, u, done), _verify_ref(p, q, tokens, rows, u, done))


@pytest.mark.parametrize("n,V,with_q", [(5, 12288, True), (5, 12289, True), (5, 24576, False), (5, 24577, False), (256, 9000, True), (257, 9000, True), (6, 40000, True)])
def test_few_queries_at_the_second_launch(n, V, with_q):
    test_verification(n, 2, V, with_q)
