"""The examples with shared pages, a window with first tokens, and beam search: whole decoding loops."""
import numpy as np
import pytest

from test_example_gpu import _decoder, _plain_logits

pytestmark = pytest.mark.gpu


def _beams(n, prompt, steps, format="int8"):
    E, decoder = _decoder(n, prompt, steps, format)
    import beam_search as B
    return E, B, decoder


@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 0), (50, 7)])
def test_continuations_that_share_pages(window, sinks):
    """Long enough a prompt for a plan; the tokens of the greedy continuation are those without sharing, where no two logits lie closer
    together than the order of sums can move them."""
    import torch
    results = []
    for share, graph in ((False, True), (True, False), (True, True)):
        E, decoder = _decoder(24, 2500, 9)
        decoder.window, decoder.sinks = window, sinks
        prompt = torch.randint(0, 1024, (2500,), generator=torch.Generator().manual_seed(5)).cuda()
        results.append(E.sample_continuations(decoder, prompt, 24, 9, E.Sampling(temperature=0.0), graph=graph, share=share))
    (a, _), (b, _), (c, _) = results
    assert torch.equal(b, c) and (b == b[:, :1]).all() and torch.equal(a[:1], b[:1])
    assert (a == b).float().mean() > 0.8


def test_a_window_with_first_tokens_follows_the_decoder():
    import torch
    E, decoder = _decoder(2, 70, 6)
    decoder.window, decoder.sinks = 20, 4
    prompt = torch.randint(0, 1024, (70,), generator=torch.Generator().manual_seed(6)).cuda()
    tokens, _ = E.sample_continuations(decoder, prompt, 2, 6, E.Sampling(temperature=0.0), share=True)
    triu = np.triu_indices
    so_far = prompt.tolist()
    for t in tokens[:, 0].tolist():
        n = len(so_far)
        i, j = np.indices((n, n))
        hidden = np.nonzero((j > i) | ((j <= i - 20) & (j >= 4)))
        try:
            np.triu_indices = lambda *_, hidden=hidden: hidden  # (what the plain decoder masks)
            want = _plain_logits(decoder, np.array(so_far))
        finally:
            np.triu_indices = triu
        # as without a window: the cache's rounding, 5 % of the logits' spread, twice over
        assert want.max() - want[t] <= 2 * 0.05 * max(np.abs(want - want.mean()).mean(), 1e-3) * 4
        so_far.append(t)


def test_a_replayed_beam_search_is_a_launched_one():
    import torch
    results = []
    for graph in (False, True):
        E, B, decoder = _beams(5, 100, 30)
        prompt = torch.randint(0, 1024, (100,), generator=torch.Generator().manual_seed(5)).cuda()
        results.append(B.beam_search(decoder, prompt, 5, 30, end_token=2, graph=graph))
        assert decoder.tables.lengths.tolist() == [0] + [129] * 5
        # holders of pages: as many as rows of the table name them
        held = [decoder.tables.page_table[s, :3] for s in range(1, 6)]
        want = torch.bincount(torch.cat(held).long().cpu(), minlength=decoder.layout.pages)
        assert torch.equal(decoder.tables.refs.cpu().long(), want) and want.max() == 5
        assert E.give_back(decoder, [1, 2, 3, 4, 5]) == 0
    for x, y in zip(*results):
        assert torch.equal(x, y)
    tokens, scores, lengths = results[0]
    assert len({tuple(t) for t in tokens.tolist()}) == 5 and torch.isfinite(scores).all()


@pytest.mark.parametrize("format", ["int8", "fp8"])
def test_scores_of_a_beam_search_are_those_of_its_tokens(format):
    """The log-probabilities of a beam's tokens after one another, by the plain decoder in 64 bits: the cache's rounding moves a logit by some 5 % (int8)
    or 20 % (fp8) of their spread at most, its log-probability by twice that."""
    import torch
    E, B, decoder = _beams(3, 70, 8, format)
    prompt = torch.randint(0, 1024, (70,), generator=torch.Generator().manual_seed(6)).cuda()
    end = 5
    tokens, scores, lengths = B.beam_search(decoder, prompt, 3, 8, end_token=end, penalty=0.7)
    ranks = scores / lengths.float() ** 0.7
    assert (ranks[:-1] >= ranks[1:]).all()
    for row, score, length in zip(tokens.tolist(), scores.tolist(), lengths.tolist()):
        assert row[length:] == [end] * (8 - length) and end not in row[:length - 1]
        so_far, total, slack = prompt.tolist(), 0.0, 0.0
        for t in row[:length]:
            want = _plain_logits(decoder, np.array(so_far))
            slack += 2 * {"int8": 0.05, "fp8": 0.2}[format] * max(np.abs(want - want.mean()).mean(), 1e-3) * 4
            total += want[t] - want.max() - np.log(np.exp(want - want.max()).sum())
            so_far.append(t)
        assert abs(total - score) <= slack


def test_one_beam_is_the_greedy_continuation():
    import torch
    E, B, decoder = _beams(1, 90, 12)
    prompt = torch.randint(0, 1024, (90,), generator=torch.Generator().manual_seed(8)).cuda()
    tokens, _, _ = B.beam_search(decoder, prompt, 1, 12, end_token=1023)
    E.give_back(decoder, [1])
    greedy, _ = E.sample_continuations(decoder, prompt, 1, 12, E.Sampling(temperature=0.0))
    n = tokens[0].tolist().index(1023) + 1 if 1023 in tokens[0].tolist() else 12
    assert tokens[0, :n].tolist() == greedy[:n, 0].tolist()


def test_a_beam_search_without_room_is_refused():
    import torch
    E, B, decoder = _beams(2, 10, 10)  # (tables of two pages)
    with pytest.raises(RuntimeError, match="prompt: the page table"):
        B.beam_search(decoder, torch.zeros(129, dtype=torch.int64, device="cuda"), 2, 3, 1)
    with pytest.raises(RuntimeError, match="token: the page table"):
        B.beam_search(decoder, torch.zeros(127, dtype=torch.int64, device="cuda"), 2, 4, 1)
