"""The example of examples/: quantised projections, cache, attention, pages and sampling in one decoding loop."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _decoder(n, prompt, steps, format="int8"):
    import sample_continuations as E
    shape = E.Shape(layers=2, hidden=256, q_heads=4, kv_heads=2, head_dim=64, ffn=512, vocab=1024, theta=10000.0)
    each = (prompt + steps) // 64 + 2
    return E, E.Decoder(shape, pages=each * (n + 1), sequences=n + 1, table_pages=each, seed=3, format=format)


def _plain_logits(decoder, tokens):
    """Logits after the last of `tokens` in float64, from the matrices' codes, with keys and values that were never rounded."""
    s = decoder.shape

    def product(m, x):
        p = m.problem
        w = np.repeat(p.scales.astype(np.float64), p.group, 0).T * p.codes + np.repeat(p.zeros.astype(np.float64), p.group, 0).T
        y = np.empty((x.shape[0], p.N))
        y[:, p.row_perm] = x[:, p.col_perm] @ w.T
        return y

    def norm(x):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-5)

    def turn(x):
        angle = np.arange(x.shape[0])[:, None, None] * s.theta ** (-np.arange(0, s.head_dim, 2) / s.head_dim)
        a, b = np.split(x, 2, -1)
        return np.concatenate((a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)), -1)

    n = len(tokens)
    x = decoder.embedding.cpu().numpy().astype(np.float64)[tokens]
    for m in decoder.layers:
        q, k, v = np.split(product(m["qkv"], norm(x)).reshape(n, -1, s.head_dim), (s.q_heads, s.q_heads + s.kv_heads), 1)
        q, k = turn(q), turn(k)
        out = np.empty_like(q)
        for h in range(s.q_heads):
            kv = h // (s.q_heads // s.kv_heads)
            score = q[:, h] @ k[:, kv].T / np.sqrt(s.head_dim)
            score[np.triu_indices(n, 1)] = -np.inf
            e = np.exp(score - score.max(1, keepdims=True))
            out[:, h] = e @ v[:, kv] / e.sum(1, keepdims=True)
        x = x + product(m["out"], out.reshape(n, -1))
        gate, up = np.split(product(m["up"], norm(x)), 2, -1)
        x = x + product(m["down"], gate / (1 + np.exp(-gate)) * up)
    return product(decoder.head, norm(x[-1:]))[0]


def test_a_replayed_step_samples_what_a_launched_one_does():
    import torch
    results = []
    for graph in (False, True):
        E, decoder = _decoder(6, 100, 40)
        prompt = torch.randint(0, 1024, (100,), generator=torch.Generator().manual_seed(5)).cuda()
        results.append(E.sample_continuations(decoder, prompt, 6, 40, E.Sampling(temperature=1.0, top_k=0, top_p=1.0), seed=9, graph=graph))
        assert decoder.tables.lengths.tolist() == [0] + [139] * 6
        # 100 tokens: one page that all share, the second copied for five of them, a third for each
        assert int((decoder.tables.refs > 0).sum()) == 13 and decoder.tables.refs.max() == 6
        assert E.give_back(decoder, [1, 3, 5]) == 7 and int((decoder.tables.refs[:7] > 0).sum()) == 7
        assert E.give_back(decoder, [2, 4, 6]) == 0
    (a, p), (b, q) = results
    assert torch.equal(a, b) and torch.equal(p, q)
    assert len({tuple(r) for r in a.T.tolist()}) == 6  # (continuations of their own)


@pytest.mark.parametrize("format", ["int8", "fp8"])
@pytest.mark.parametrize("temperature,top_k", [(0.0, 0), (1.0, 1)])
def test_continuations_follow_the_decoder(format, temperature, top_k):
    """After a prompt and greedy tokens, logits are those of the plain decoder on the same tokens, up to the cache's rounding: a key or
    value of eight bits is off by its page's maximum / 254 (int8) or 1/16 of itself (fp8) at most, in root mean square 1% or
    4% of a typical value with the rewriting of growing pages, which softmax averages and two layers pass on once each."""
    import torch
    E, decoder = _decoder(3, 70, 12, format)
    prompt = torch.randint(0, 1024, (70,), generator=torch.Generator().manual_seed(6)).cuda()
    tokens, logprobs = E.sample_continuations(decoder, prompt, 3, 12, E.Sampling(temperature=temperature, top_k=top_k, top_p=1.0), seed=1)
    assert (tokens == tokens[:, :1]).all()
    so_far = prompt.tolist()
    for t, lp in zip(tokens[:, 0].tolist(), logprobs[:, 0].tolist()):
        want = _plain_logits(decoder, np.array(so_far))
        spread = np.abs(want - want.mean()).mean()
        tolerance = {"int8": 0.05, "fp8": 0.2}[format] * max(spread, 1e-3) * 4
        assert want.max() - want[t] <= 2 * tolerance
        # (the first token alone has weight at temperature 0; what top_k leaves out counts)
        ln = want[t] - want.max() - np.log(np.exp(want - want.max()).sum()) if temperature else 0.0
        assert abs(ln - lp) <= (2 * tolerance if temperature else 0.0)
        so_far.append(t)


@pytest.mark.parametrize("prompt,steps,message", [(129, 2, "prompt: the page table"), (128, 3, "token: the page table"), (64, 5, None)])
def test_what_finds_no_room_is_refused(prompt, steps, message):
    import contextlib
    import torch
    E, decoder = _decoder(1, 10, 10)  # (tables of two pages)
    with pytest.raises(RuntimeError, match=message) if message else contextlib.nullcontext():
        E.sample_continuations(decoder, torch.zeros(prompt, dtype=torch.int64, device="cuda"), 1, steps, E.Sampling())


def test_a_pool_without_pages_is_refused():
    import torch
    E, decoder = _decoder(6, 100, 40)
    others = torch.ones(decoder.layout.pages - 5, dtype=torch.int32)
    decoder.tables.refs[:len(others)] = others.cuda()  # (held by someone else)
    with pytest.raises(RuntimeError, match="token: 2 pages are missing"):  # 2 for the prompt, 5 copies of the second
        E.sample_continuations(decoder, torch.zeros(100, dtype=torch.int64, device="cuda"), 6, 3, E.Sampling())
