"""Choice of the next token on the GPU where sums, slices and parameters end."""
import math

import numpy as np
import pytest

from test_sample_gpu import _check, _logits, _run

pytestmark = pytest.mark.gpu

# Rows of 262144 (of 57 to 93 in a call) and 524288 tokens (of 31 to 101) are cut into slices of 32768, the longest there are, and
# with a token more or less into slices of both neighbouring lengths.
WIDE = [(64, 262144), (64, 262143), (64, 262145), (31, 524288), (31, 524285)]


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("rows,vocab", WIDE)
def test_equal_logits_in_the_longest_slices(rows, vocab, dtype):
    # a slice lies in one bin as a whole, every token with the largest weight: the choice is exact, the number of the token
    x = np.full((rows, vocab), 3.25, dtype=np.float32)
    u = ((np.arange(rows) + 0.5) / rows).astype(np.float32)
    tokens, logprobs, _ = _run(x, 1.0, 0, 1.0, 0.0, u, dtype=dtype)
    assert tokens.tolist() == [int(float(v) * vocab) for v in u]
    # (as the test of equal logits in short slices: a logarithm and a sum in fp32)
    assert np.allclose(logprobs, -math.log(vocab), rtol=1e-6)
    k = 1 + np.arange(rows) * (vocab // rows)
    tokens, logprobs, _ = _run(x, 1.0, k, 1.0, 0.0, 1.0 - 2.0 ** -24, dtype=dtype)
    assert tokens.tolist() == (k - 1).tolist() and np.allclose(logprobs, -math.log(vocab), rtol=1e-6)
    # top-p on top of it: the shortest prefix that holds a half of k equal weights
    tokens, _, _ = _run(x, 1.0, k, 0.5, 0.0, 1.0 - 2.0 ** -24, dtype=dtype)
    assert tokens.tolist() == ((k + 1) // 2 - 1).tolist()


@pytest.mark.parametrize("rows,vocab", WIDE[:1] + WIDE[3:4])
def test_one_slice_above_the_others(rows, vocab):
    x = np.zeros((rows, vocab), dtype=np.float32)
    place = np.arange(rows) % (vocab // 32768) * 32768
    for r in range(rows):
        x[r, place[r]:place[r] + 32768] = 1.0
    tokens, logprobs, _ = _run(x, 1.0, 0, 1.0, 0.0, 0.0)
    assert tokens.tolist() == place.tolist()
    assert np.allclose(logprobs, -math.log(32768 + (vocab - 32768) / math.e), rtol=1e-6)
    # the weight of the slice in the whole is 0.28 or less: behind it the others follow by their numbers
    share = 32768 / (32768 + (vocab - 32768) / math.e)
    u = np.float32(0.9)
    rest = int((float(u) - share) / (1 - share) * (vocab - 32768))
    tokens, _, _ = _run(x, 1.0, 0, 1.0, 0.0, u)
    # (a weight of 1/e in units of 2^-31: 2^-31 of the sum off, a token of 2^19 at most)
    want = rest + np.where(rest >= place, 32768, 0)
    assert (np.abs(tokens - want) <= 1).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,vocab", WIDE[:3])
def test_every_filter_over_the_longest_slices(rows, vocab, dtype):
    rng = np.random.default_rng(vocab)
    x = _logits(rng, rows, vocab)
    t, k = rng.choice([0.0, 0.6, 1.0, 2.0], rows), rng.choice([0, 1, 50, 2000], rows)
    p, m, u = rng.choice([0.2, 0.95, 1.0], rows), rng.choice([0.0, 0.03], rows), rng.random(rows)
    sure, _ = _check(x, t, k, p, m, u, dtype=dtype)
    assert sure >= rows // 3


def _uniform(x, u):
    """Tokens of rows whose finite logits all weigh the same: by falling logit, equal ones by rising number."""
    out = []
    for row, v in zip(x, np.broadcast_to(np.asarray(u, dtype=np.float32), len(x))):
        n = int(np.isfinite(row).sum())
        out.append(int(np.lexsort((np.arange(row.size), -row.astype(np.float64)))[int(float(v) * n)]))
    return out


@pytest.mark.parametrize("temperature", [1e30, 3e38, math.inf])
@pytest.mark.parametrize("rows,vocab,finite", [(4, 100, 100), (4, 2048, 2048), (4, 2049, 2049), (4, 5000, 1500), (3, 131072, 700), (3, 131072, 2048),
                                               (2, 131072, 2049), (120, 1000, 1000), (64, 262144, 90)])
def test_temperatures_at_which_all_weigh_the_same(temperature, rows, vocab, finite):
    rng = np.random.default_rng(vocab + finite)
    x = np.full((rows, vocab), -math.inf, dtype=np.float32)
    for r in range(rows):
        x[r, rng.permutation(vocab)[:finite]] = rng.choice(rng.normal(0.0, 3.0, 50), finite)
    u = rng.random(rows).astype(np.float32)
    tokens, logprobs, _ = _run(x, temperature, 0, 1.0, 0.0, u)
    assert tokens.tolist() == _uniform(x, u)
    assert np.allclose(logprobs, -math.log(finite), rtol=1e-6)
    tokens, _, _ = _run(x, temperature, 1 + rng.integers(0, finite, rows), [1.0, 0.7][rows % 2], 0.5, 0.0)
    assert tokens.tolist() == _uniform(x, 0.0)
    tokens, _, _ = _run(x, temperature, finite, 1.0, 0.999, 1.0 - 2.0 ** -24)
    assert tokens.tolist() == _uniform(x, 1.0 - 2.0 ** -24)


@pytest.mark.parametrize("temperature", [1e-38, 4e-38, 1e-36, 1e-30])
def test_temperatures_near_the_least(temperature):
    # logits that lie a few temperatures apart, some of them no normal numbers; weights 1, 1/e, 1/e^2
    t = float(np.float32(temperature))
    x = np.float32(t) * np.array([[-1.0, 0.0, -2.0, -1e3], [0.0, -2.0, -1.0, -40.0]], dtype=np.float32)
    share = np.cumsum(np.exp([0.0, -1.0, -2.0])) / np.exp([0.0, -1.0, -2.0]).sum()
    for u, at in ((0.1, 0), (0.99 * share[0], 0), (1.01 * share[0], 1), (0.999 * share[1], 1), (1.001 * share[1], 2), (1.0 - 2.0 ** -24, 2)):
        tokens, logprobs, _ = _run(x, t, 0, 1.0, 0.0, u)
        assert tokens.tolist() == [[1, 0, 2][at], [0, 2, 1][at]], u
        # (a product of a denormal number and its temperature: 2^-22 of it)
        assert np.allclose(logprobs, -at - math.log(np.exp([0.0, -1.0, -2.0]).sum()), atol=1e-5)


def test_intervals_that_pass_the_range_of_fp32():
    x = np.array([[3.4e38, 3.3e38, 0.5e38, 0.0], [-3.3e38, -3.4e38, -3.35e38, -math.inf]], dtype=np.float32)
    for t in (1e37, 1e38, 3.4e38):
        _check(x, t, 0, 1.0, 0.0, [0.3, 0.9])
        _check(x, t, 2, 1.0, 0.0, [0.9, 0.6])


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows,vocab", [(3, 1000), (3, 131072), (120, 5000)])
def test_log_probabilities_of_ties_at_temperature_0(rows, vocab, dtype):
    # -ln of the number of tokens that share the largest logit, 0 where there is one
    rng = np.random.default_rng(vocab)
    x = rng.normal(size=(rows, vocab)).astype(np.float32)
    ties = rng.choice([1, 2, 7, 900], rows)
    first = []
    for r in range(rows):
        at = rng.permutation(vocab)[:ties[r]]
        x[r, at] = 9.5
        first.append(int(at.min()))
    tokens, logprobs, _ = _run(x, 0.0, 0, 1.0, 0.0, 0.7, dtype=dtype)
    assert tokens.tolist() == first
    assert (logprobs[ties == 1] == 0).all() and np.allclose(logprobs, -np.log(ties), rtol=1e-6)


@pytest.mark.parametrize("rows", [2, 120])
def test_log_probability_where_the_others_are_below_the_unit(rows):
    # one token with nearly all the weight: off by what the others lose or gain in whole units of 2^-31, 2^-32 for each at most
    vocab = 70000
    for other in (-24.0, -22.3, -22.0, -21.0, -20.0):
        x = np.full((rows, vocab), other, dtype=np.float32)
        x[:, 5] = 0.0
        tokens, logprobs, _ = _run(x, 1.0, 0, 1.0, 0.0, 0.0)
        want = -math.log1p((vocab - 1) * math.exp(other))
        assert (tokens == 5).all() and (np.abs(logprobs - want) <= vocab * 2.0 ** -32 + 1e-6 * abs(want)).all()
        units = (vocab - 1) * round(math.exp(other) * 2 ** 31) * 2.0 ** -31
        assert np.allclose(logprobs, -math.log1p(units), rtol=1e-6, atol=0.0)
