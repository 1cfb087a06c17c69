"""Sums of exponentials of a beam search's rows on the GPU: a piece's largest terms in 64 bits, and what stands beside them in a run."""
import math

import numpy as np
import pytest

from kv_util import U32
from test_beam_gpu import DTYPES, _call

pytestmark = pytest.mark.gpu


def _check(x, beams, choices, dtype, scores=None, **more):
    """x: logits that dtype holds exactly.  Scores (None: those that leave the best continuation of a row at some 2^-24, where fp32 tells
    2^-47 apart) and the values against 64 bits, within what the terms that no list can hold may be off by."""
    x = x.astype(np.float64)
    top = x.max(axis=1, keepdims=True)
    logs = np.log(np.exp(x - top).sum(axis=1))
    scores = (logs if scores is None else np.asarray(scores)).astype(np.float32)
    held, (values, parents, tokens) = _call(x, beams, scores, choices, dtype=dtype, **more)
    assert np.array_equal(held, x)
    p = np.exp(x - top)
    listed = np.argsort(-x, axis=1, kind="stable")[:, :choices]  # (of the whole row: a piece lists these and perhaps more)
    np.put_along_axis(p, listed, 0.0, axis=1)
    d = np.where(p > 0, np.minimum(top - x, 1e30), 0.0)
    # A term not listed: its argument |d| log2(e), rounded as a product and by the logarithm's own rounding, 2.25 U32 |d| together, an exponential of
    # one unit in the last place, 2 U32, and seven additions of a run; all relative to the sum.  Terms in 64 bits and what is joined of pieces: below 2^-36.
    slack = U32 * (p * (10.0 + 4.0 * d)).sum(axis=1) / np.exp(logs) + 2.0 ** -36
    assert slack.max() < 2.0 ** -26, "nothing would be seen"
    for r in range(len(x) // beams):
        rows = slice(r * beams, (r + 1) * beams)
        want = scores[rows, None].astype(np.float64) + (x[rows] - top[rows]) - logs[rows, None]
        for v, b, t in zip(values[r].astype(np.float64), parents[r] - r * beams, tokens[r]):
            if b >= 0:
                assert abs(v - want[b, t]) <= U32 * abs(want[b, t]) * 1.01 + slack[r * beams + b], (r, b, t, v, want[b, t], slack[r * beams + b])
        order = sorted(((-want[b, t], b, t) for b in range(beams) for t in np.flatnonzero(np.isfinite(x[r * beams + b]))))[:choices]
        for i, (v, b, t) in enumerate(order):
            apart = 2.0 * slack[rows].max()
            if all(abs(v - order[j][0]) > apart for j in (i - 1, i + 1) if 0 <= j < len(order)) and i + 1 < len(order):
                assert (parents[r, i] - r * beams, tokens[r, i]) == (b, t), (r, i)
    return values, parents, tokens


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("choices", [1, 2, 5])
@pytest.mark.parametrize("vocab,offset", [(4, 0), (8, 0), (23, 1), (4099, 3), (16384, 0)])
def test_small_terms_beside_a_listed_one(dtype, choices, vocab, offset):
    rng = np.random.default_rng(vocab + choices)
    x = np.full((6, vocab), -math.inf)
    for i in range(6):
        start = int(rng.integers(0, max(vocab - 8, 0) + 1)) // 8 * 8  # (a run of 16 bits, two of 32)
        n = min(8, vocab - start)
        x[i, start:start + n] = -rng.integers(14 * 64, 18 * 64, n) / 64.0  # (whole 64ths: 16 bits hold them)
        x[i, start + rng.permutation(n)[:1 + i % min(choices, n)]] = rng.integers(-1, 1) / 64.0
    x = x if dtype != "bfloat16" else np.round(x * 8) / 8
    _check(x, 3, choices, dtype, offset=offset)


@pytest.mark.parametrize("dtype,far", [(t, False) for t in DTYPES] + [("float16", True), ("float32", True)])  # (bfloat16 holds multiples of 32 there at best)
@pytest.mark.parametrize("rising", [True, False])
def test_listed_terms_of_several_chunks(dtype, far, rising):
    # 32 beams and 64 choices leave a row 4 pieces, of several chunks each; each has larger terms than the one before it, or smaller ones, so that
    # sums go from one largest logit to the next.  `far`: logits past those whose exponentials are made by one operation
    rng = np.random.default_rng(3)
    vocab = 131072
    x = np.full((32, vocab), -math.inf)
    for i in range(32):
        for chunk in range(32):
            for _ in range(2 if chunk % 2 else 1):
                start = chunk * 4096 + 8 * int(rng.integers(0, 512))
                high = (chunk if rising else 31 - chunk) / 4.0
                x[i, start:start + 8] = high - 8.0 - rng.integers(14 * 4, 18 * 4, 8) / 4.0
                x[i, start + int(rng.integers(0, 8))] = high - 8.0 + rng.integers(0, 2) / 4.0
    if far:
        x += 8192.0 if dtype == "float32" else 4608.0
        x = np.round(x * (4 if dtype == "float32" else 0.25)) / (4 if dtype == "float32" else 0.25)
    _check(x, 32, 64, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_beams_that_differ_by_what_stands_beside_the_best(dtype):
    # ln(1 + 7 exp(-16)) = 7.9e-7: scores on both sides of it, a few 1e-8 away
    x = np.full((2, 64), -math.inf)
    x[0, 8], x[0, 9:16], x[1, 8] = 0.0, -16.0, 0.0
    for by in (-3e-8, -1e-9, 1e-9, 3e-8):
        values, parents, tokens = _check(x, 2, 2, dtype, scores=[0.0, -math.log1p(7 * math.exp(-16.0)) + by])
        assert parents[0].tolist() == ([1, 0] if by > 0 else [0, 1])
