"""Probabilities of rows at the sizes where the kernels change hands: vectors of a thread, rows that just fit the registers or do not, rows shorter than a
vector, and numbers of rows from which a row is one workgroup's.  Bars as in the tests of the other sizes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_draft_head import DEV, TYPES, _probs_ref, _probs_tolerance, _token_probs

pytestmark = pytest.mark.gpu


def _check(x, T, pad, shift):
    got, xs = _token_probs(x.to(DEV), T, pad=pad, shift=shift), x.double().numpy()
    ref = _probs_ref(xs, T)
    assert (np.abs(got - ref) <= _probs_tolerance(xs, T, ref)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [
    (3, 7), (3, 8), (3, 9), (2, 15), (2, 4065), (2, 4066), (2, 8161), (2, 8162), (2, 16353), (2, 16384), (2, 16385),
    (17, 17000), (16, 16999), (34, 33000), (54, 53000), (66, 65505), (66, 65506), (82, 81889), (82, 81890)])
def test_rows_at_the_limits(rows, vocab, dtype):
    g = torch.Generator().manual_seed(vocab)
    x = (torch.randn((rows, vocab), generator=g) * 3).masked_fill(torch.rand((rows, vocab), generator=g) < 0.05, float("-inf")).to(TYPES[dtype][0])
    x[0, 0], x[-1, vocab - 1] = 21.0, 22.0               # the likeliest token first, and last
    for T, pad, shift in ((0.0, 1, 3), (0.9, 0, 0)):
        _check(x, T, pad, shift)


@pytest.mark.parametrize("rows,vocab", [(132, 131072), (132, 131011), (164, 163809), (164, 163810)])
def test_long_rows_of_16_bits(rows, vocab):
    x = (torch.randn((rows, vocab), generator=torch.Generator().manual_seed(vocab)) * 3).to(torch.bfloat16)
    x[3] = float("-inf")
    x[4, 7:] = float("nan")
    _check(x, 1.1, vocab % 2, 1)


def test_first_of_equal_logits_wherever_the_row_begins():
    for shift in range(0, 32, 5):
        for vocab in (300, 9000, 40000):
            x = torch.zeros((41, vocab))
            x[7, vocab - 3:] = 1.0
            x[8, ::41] = 1.0
            got = _token_probs(x.to(DEV), 0.0, pad=3, shift=shift)
            want = np.zeros(41, int)
            want[7] = vocab - 3
            assert np.array_equal(got.argmax(1), want) and np.array_equal(got.sum(1), np.ones(41))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(3, 32736), (3, 32737), (3, 32738), (2, 24001)])
def test_few_rows_at_the_second_launch(rows, vocab, dtype):
    x = (torch.randn((rows, vocab), generator=torch.Generator().manual_seed(vocab)) * 3).to(TYPES[dtype][0])
    x[0, vocab - 1] = 25.0
    for T in (0.0, 0.7):
        _check(x, T, 1, 2)
