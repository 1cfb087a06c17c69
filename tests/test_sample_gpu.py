"""Choice of the next token on the GPU against the CPU oracle."""
import math

import numpy as np
import pytest

from oracle import sfmp_kv_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _run(x, temperature, top_k, top_p, min_p, u, dtype="float32", apart=0, offset=0):
    """x [rows, vocab] (numpy).  Returns (tokens, logprobs, the logits as the call saw them)."""
    import torch
    import paper_2602_01027_amd as S
    assert torch.cuda.is_available()
    rows, vocab = x.shape
    buffer = torch.zeros((rows, vocab + apart + offset), dtype=getattr(torch, dtype), device=DEV)
    logits = buffer[:, offset:offset + vocab]
    logits.copy_(torch.from_numpy(x).to(DEV))
    up = lambda a, t: None if a is None else torch.from_numpy(np.broadcast_to(np.asarray(a), (rows,)).astype(t)).to(DEV)  # noqa: E731
    tokens = torch.full((rows,), 12345, dtype=torch.int32, device=DEV)
    logprobs = torch.full((rows,), math.nan, dtype=torch.float32, device=DEV)
    ws = torch.full((S.sfmp_sample_workspace(rows, vocab),), 0xFF, dtype=torch.uint8, device=DEV)
    args = (logits, up(temperature, np.float32), up(top_k, np.int32), up(top_p, np.float32), up(min_p, np.float32), up(u, np.float32), tokens,
            logprobs, ws)
    S.sfmp_sample(*args)
    first = tokens.clone(), logprobs.clone()
    ws.fill_(0x55)
    S.sfmp_sample(*args)
    torch.cuda.synchronize()
    assert torch.equal(first[0], tokens) and torch.equal(first[1], logprobs)  # the same bits
    return tokens.cpu().numpy(), logprobs.cpu().numpy(), logits.float().cpu().numpy()


# Weights are computed in fp32 (each off by a few 2^-24 of itself) and held in units of 2^-31 of the largest: a decision that
# is nearer than 1e-5 of the whole weight, or, for min-p, of the difference of logits over temperature, may go either way.
NEAR = 1e-5


def _check(x, temperature, top_k, top_p, min_p, u, **more):
    tokens, logprobs, seen = _run(x, temperature, top_k, top_p, min_p, u, **more)
    rows = x.shape[0]
    at = lambda a, r, d: d if a is None else np.broadcast_to(np.asarray(a), (rows,))[r]  # noqa: E731
    f = lambda v: float(np.float32(v))  # noqa: E731
    sure = 0
    for r in range(rows):
        token, logprob, margin = O.sample(seen[r], f(at(temperature, r, 1.0)), int(at(top_k, r, 0)), f(at(top_p, r, 1.0)), f(at(min_p, r, 0.0)),
                                          f(at(u, r, 0)))
        if margin > NEAR:
            sure += 1
            assert tokens[r] == token, (r, tokens[r], token, margin)
            if token < 0:
                assert np.isneginf(logprobs[r])
            else:
                # (l - m) / T of a few U32, its exponential's sum, the logarithm; and the tokens below 2^-32 that weigh nothing
                assert abs(logprobs[r] - logprob) <= 2.0 ** -20 * (1 + abs(logprob)) + x.shape[1] * 2.0 ** -32, (r, logprobs[r], logprob)
    return sure, tokens


def _logits(rng, rows, vocab, std=2.0):
    x = rng.normal(0.0, std, size=(rows, vocab))
    x[:, rng.integers(0, vocab, max(1, vocab // 50))] += rng.exponential(3.0, size=max(1, vocab // 50))
    x[rng.random((rows, vocab)) < 0.01] = -math.inf
    x[:, 0] = 1.0
    return x.astype(np.float32)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows,vocab,apart,offset", [(1, 1, 0, 0), (3, 7, 0, 0), (5, 1000, 0, 0), (4, 4099, 3, 1), (24, 32000, 0, 0), (3, 131072, 0, 0),
                                                     (2, 100003, 5, 3), (70, 257, 1, 0)])
def test_every_filter(dtype, rows, vocab, apart, offset):
    rng = np.random.default_rng(rows + vocab)
    x = _logits(rng, rows, vocab)
    sure = all_ = 0
    for t, k, p, m in ((1.0, 0, 1.0, 0.0), (0.7, 40, 1.0, 0.0), (1.3, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.05), (0.9, 1000, 0.95, 0.02), (0.0, 5, 0.3, 0.1),
                       (2.0, 3, 0.5, 0.9), (1.0, vocab, 1.0, 1.0), (1.0, 2 ** 31 - 1, 0.0, 0.0), (1.0, -4, 2.0, -1.0)):
        u = rng.random(rows)
        s, _ = _check(x, t, k, p, m, u, dtype=dtype, apart=apart, offset=offset)
        sure, all_ = sure + s, all_ + rows
    assert sure > 0.5 * all_


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("rows,vocab,apart,offset", [(96, 3, 0, 0), (130, 5000, 1, 3), (100, 70001, 0, 0), (97, 140007, 2, 1)])
def test_many_rows(dtype, rows, vocab, apart, offset):
    # one workgroup per row, which keeps a part of it in registers: the same as the first rows alone, sliced, and as the oracle
    rng = np.random.default_rng(rows + vocab)
    x = _logits(rng, rows, vocab)
    t, k = rng.choice([0.0, 0.6, 1.0, 2.0], rows), rng.choice([0, 1, 50, 2000], rows)
    p, m, u = rng.choice([0.2, 0.95, 1.0], rows), rng.choice([0.0, 0.03], rows), rng.random(rows)
    all_, logprobs, _ = _run(x, t, k, p, m, u, dtype=dtype, apart=apart, offset=offset)
    some = slice(0, 40)
    few, few_logprobs, _ = _run(x[some], t[some], k[some], p[some], m[some], u[some], dtype=dtype)
    assert np.array_equal(all_[some], few) and np.array_equal(logprobs[some], few_logprobs)
    sure, tokens = _check(x[:96], t[:96], k[:96], p[:96], m[:96], u[:96], dtype=dtype, apart=apart, offset=offset)
    assert sure > 40 and np.array_equal(tokens, all_[:96])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,vocab,apart,offset", [(1, 38183, 0, 0), (40, 100003, 1, 2), (64, 131072, 0, 0), (2, 1000003, 5, 1)])
def test_slices_of_every_length(dtype, rows, vocab, apart, offset):
    # few to many slices of a row, of 4096 to 32768 tokens
    rng = np.random.default_rng(rows + vocab)
    x = _logits(rng, rows, vocab)
    t, k = rng.choice([0.0, 0.6, 1.0, 2.0], rows), rng.choice([0, 1, 50, 2000], rows)
    p, m, u = rng.choice([0.2, 0.95, 1.0], rows), rng.choice([0.0, 0.03], rows), rng.random(rows)
    sure, _ = _check(x, t, k, p, m, u, dtype=dtype, apart=apart, offset=offset)
    assert sure >= rows // 3


@pytest.mark.parametrize("vocab", [2049, 100000])
def test_many_rows_of_equal_logits(vocab):
    x = np.full((100, vocab), -1.5, dtype=np.float32)
    x[:, ::2] += 1e-4
    half = (vocab + 1) // 2
    tokens, _, _ = _run(x, 1.0, 1 + np.arange(100) * (half // 100), 1.0, 0.0, 1.0 - 2.0 ** -24)
    assert tokens.tolist() == [2 * i * (half // 100) for i in range(100)]


def test_defaults_and_parameters_by_row():
    rng = np.random.default_rng(0)
    x = _logits(rng, 40, 5000)
    _check(x, None, None, None, None, rng.random(40))
    _check(x, rng.choice([0.0, 0.5, 1.0, 3.0], 40), rng.choice([0, 1, 7, 100], 40), rng.choice([0.3, 0.9, 1.0], 40), rng.choice([0.0, 0.1], 40), rng.random(40))


@pytest.mark.parametrize("u", [0.0, 1.0 - 2.0 ** -24])
def test_ends_of_the_random_number(u):
    rng = np.random.default_rng(2)
    x = _logits(rng, 3, 3000)
    tokens, logprobs, seen = _run(x, 1.0, 20, 1.0, 0.0, u)
    for r in range(3):
        order = np.lexsort((np.arange(3000), -seen[r].astype(np.float64)))
        assert tokens[r] == (order[0] if u == 0.0 else order[19])


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("vocab", [100, 2048, 2049, 70000, 131072])
def test_rows_of_equal_logits(dtype, vocab):
    # every token is in one bin and in one tie: order by number alone
    x = np.full((4, vocab), 3.25, dtype=np.float32)
    u = np.array([0.0, 0.2501, 0.5, 0.99])
    tokens, logprobs, _ = _run(x, 1.0, 0, 1.0, 0.0, u, dtype=dtype)
    assert tokens.tolist() == [int(np.float32(v).astype(np.float64) * vocab) for v in u]
    assert np.allclose(logprobs, -math.log(vocab), rtol=1e-6)
    tokens, _, _ = _run(x, 1.0, [1, 2, 57, vocab - 1], 1.0, 0.0, 1.0 - 2.0 ** -24, dtype=dtype)
    assert tokens.tolist() == [0, 1, 56, vocab - 2]
    tokens, _, _ = _run(x, 0.0, 0, 1.0, 0.0, 0.9, dtype=dtype)
    assert (tokens == 0).all()


@pytest.mark.parametrize("vocab", [50000, 131072])
def test_rows_of_few_values_and_high_temperatures(vocab):
    # crowded bins, in which positions are narrowed digit by digit
    rng = np.random.default_rng(vocab)
    x = rng.choice([0.0, 0.001, 0.002, -0.0, 0.5], size=(6, vocab)).astype(np.float32)
    sure, _ = _check(x, 1.0, [0, 3, 30000, 0, 40000, 0], [1.0, 1.0, 1.0, 0.4, 0.7, 0.999], 0.0, rng.random(6))
    y = rng.normal(size=(6, vocab)).astype(np.float32)
    more, _ = _check(y, 200.0, [0, 3, 30000, 0, 40000, 0], [1.0, 1.0, 1.0, 0.4, 0.7, 0.999], [0, 0, 0, 0, 0, 0.98], rng.random(6))
    # (tokens of one 50000th each: a decision is seldom farther from its threshold than the tolerance)
    for k in (1, 2, 5000, 49999):
        tokens, _, _ = _run(y, 200.0, k, 1.0, 0.0, 1.0 - 2.0 ** -24)
        for r in range(6):
            assert tokens[r] == np.lexsort((np.arange(vocab), -y[r].astype(np.float64)))[k - 1]


def test_rows_with_nothing_infinities_and_nan():
    x = np.zeros((8, 600), dtype=np.float32)
    x[0] = -math.inf
    x[1] = math.nan
    x[2, 1:] = -math.inf
    x[3, 7] = math.nan
    x[3, 9] = 5.0
    x[4, [5, 50]] = math.inf
    x[5] = -3e38
    x[5, 11] = 3e38
    x[6] = -math.inf
    x[6, [3, 400]] = -3e38
    x[7, :] = np.where(np.arange(600) % 2, math.nan, -1e30)
    tokens, logprobs, _ = _run(x, 1.0, 0, 1.0, 0.0, 0.999)
    assert tokens.tolist() == [-1, -1, 0, 599, 50, 11, 400, 598]
    assert np.isneginf(logprobs[:2]).all() and logprobs[2] == 0 and np.isclose(logprobs[4], -math.log(2)) and logprobs[5] == 0
    tokens, _, _ = _run(x, 0.0, 0, 1.0, 0.0, 0.999)
    assert tokens.tolist() == [-1, -1, 0, 9, 5, 11, 3, 0]


def test_frequencies_follow_the_distribution():
    # 4096 evenly spread numbers over one row: each token as often as its weight says, to one count
    p = np.array([0.05, 0.3, 0.15, 0.4, 0.1])
    x = np.broadcast_to(np.log(p), (4096, 5)).astype(np.float32)
    tokens, _, _ = _run(x, 1.0, 0, 1.0, 0.0, (np.arange(4096) + 0.5) / 4096)
    assert np.abs(np.bincount(tokens, minlength=5) - 4096 * p).max() <= 1.01


def test_refusals_and_the_ctypes_path(monkeypatch):
    import torch
    import paper_2602_01027_amd as S
    rng = np.random.default_rng(5)
    x = _logits(rng, 3, 999)
    a = _run(x, 1.0, 10, 0.9, 0.0, 0.7, dtype="bfloat16", apart=2)
    monkeypatch.setattr(S.binding, "_LAUNCHER", (S.load_library(), S.binding._NoExtension))
    b = _run(x, 1.0, 10, 0.9, 0.0, 0.7, dtype="bfloat16", apart=2)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    monkeypatch.undo()
    l, i, f = torch.zeros((2, 9), device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV)
    w = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    good = dict(logits=l, temperature=f, top_k=i, top_p=f, min_p=f, uniform=f, tokens=i.clone(), logprobs=f.clone(), workspace=w)
    S.sfmp_sample(**good)
    for bad in (dict(logits=l.double()), dict(logits=l.t()), dict(logits=l[0]), dict(top_k=i.long()), dict(temperature=f[:1]), dict(uniform=f.half()),
                dict(tokens=i.float()), dict(logprobs=i)):
        with pytest.raises(ValueError):
            S.sfmp_sample(**{**good, **bad})
    for bad, code in ((dict(workspace=w[:0]), -5), (dict(uniform=None), -1), (dict(tokens=None), -1)):
        with pytest.raises(S.SfmpError) as e:
            S.sfmp_sample(**{**good, **bad})
        assert e.value.code == code
