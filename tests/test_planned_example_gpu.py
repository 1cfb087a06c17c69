"""The examples' loops where attention runs by a plan: reserve with copy on write, share, planned layers, choice, reorder, launched one by one and replayed."""
import numpy as np
import pytest

from test_example_gpu import _decoder, _plain_logits

pytestmark = pytest.mark.gpu


@pytest.fixture
def planned(monkeypatch):
    """Numbers of calls of sfmp_kv_attention_shared that use a plan, and of those that do not (these need no more of it than its head)."""
    import paper_2602_01027_amd as S
    call, found = S.sfmp_kv_attention_shared, [0, 0]

    def watched(cache, layer, tables, slots, row_start, groups, Q, O, max_rows, max_tokens, scale, plan, workspace, **more):
        args = (cache, layer, tables, slots, row_start, groups, Q, O, max_rows, max_tokens, scale)
        try:
            call(*args, plan[:256], workspace, **more)
            found[1] += 1
        except S.SfmpError as e:
            assert e.code == -5
            found[0] += 1
            call(*args, plan, workspace, **more)
    monkeypatch.setattr(S, "sfmp_kv_attention_shared", watched)
    return found


def _promised(decoder, max_tokens):
    """Steps are told of longer sequences than there are, as a loop with room for them would: then a plan is worth its while."""
    attention = decoder.attention
    decoder.attention = lambda slots, row_start, rows, max_rows, most, groups: attention(slots, row_start, rows, max_rows,
                                                                                       most if groups is None else max(most, max_tokens), groups)
    return decoder


def _forced(decoder, prompt, tokens):
    """Logits [steps, n, vocab] in front of each of `tokens` [steps, n] behind the prompt; every sequence attends for itself.  The decoder is empty
    before and after."""
    import torch
    import sample_continuations as E
    steps, n = tokens.shape
    numbers = lambda a, b: torch.arange(a, b, dtype=torch.int32, device="cuda")  # noqa: E731
    slots, logits = numbers(1, n + 1), [decoder.prefill(0, prompt).expand(n, -1).float()]
    E.S.sfmp_kv_fork(decoder.cache, decoder.tables, torch.zeros(n, dtype=torch.int32, device="cuda"), slots)
    E.S.sfmp_kv_free(decoder.cache, decoder.tables, numbers(0, 1))
    for i in range(steps - 1):
        decoder.reserve(slots)
        positions = decoder.tables.lengths[1:n + 1] - 1
        x = decoder.run(tokens[i], positions, slots, None, 1, prompt.shape[0] + steps)
        logits.append(decoder.logits(x).float())
    assert E.give_back(decoder, list(range(1, n + 1))) == 0
    return torch.stack(logits)


def _off(logits):
    """How far the logits of a step may lie from those of the same tokens with sums in another order.  An attention result is off by its rounding to fp16
    and its weights', 2^-11 each; two layers of five products and sums of fp16 results and the head pass that on, and round it as often:
    some 22 times 2^-11 where all of it adds up, 1 % of the logits' spread (four times what they lie from their mean)."""
    return 0.01 * 4 * (logits - logits.mean(-1, keepdim=True)).abs().mean(-1)


@pytest.mark.parametrize("window,sinks", [(0, 0), (5000, 0), (5000, 7)])
def test_planned_continuations(planned, window, sinks):
    import torch
    n, steps, tokens = 24, 9, 6000
    prompt = torch.randint(0, 1024, (tokens,), generator=torch.Generator().manual_seed(5)).cuda()
    results = []
    for graph in (False, True):
        E, decoder = _decoder(n, tokens, steps)
        decoder.window, decoder.sinks = window, sinks
        results.append(E.sample_continuations(decoder, prompt, n, steps, E.Sampling(temperature=0.0), graph=graph, share=True)[0])
        assert E.give_back(decoder, list(range(1, n + 1))) == 0
    assert planned[0] and not planned[1]
    assert torch.equal(*results)
    logits = _forced(decoder, prompt, results[0])
    chosen = logits.gather(2, results[0].long()[..., None])[..., 0]
    assert (logits.amax(2) - chosen <= 2 * _off(logits)).all()


@pytest.mark.parametrize("format", ["int8", "fp8"])
@pytest.mark.parametrize("beams,tokens,steps", [(4, 300, 70), (8, 191, 40), (2, 70, 140)])
def test_a_planned_beam_search(planned, format, beams, tokens, steps):
    """Beams part, die out and take over each other's pages within and over page ends; a score is that of its tokens when every beam attends
    for itself."""
    import torch
    prompt = torch.randint(0, 1024, (tokens,), generator=torch.Generator().manual_seed(beams)).cuda()
    results = []
    for graph in (False, True):
        E, decoder = _decoder(beams, tokens, steps, format)
        import beam_search as B
        results.append(B.beam_search(_promised(decoder, 60000), prompt, beams, steps, end_token=3, penalty=0.7, graph=graph))
        refs = torch.zeros(decoder.layout.pages, dtype=torch.int64)
        for s in range(1, beams + 1):
            held = decoder.tables.page_table[s, :-(-(tokens + steps - 1) // 64)].long().cpu()
            refs += torch.bincount(held, minlength=len(refs))
        assert torch.equal(decoder.tables.refs.cpu().long(), refs)
        assert decoder.tables.lengths.tolist() == [0] + [tokens + steps - 1] * beams
        assert E.give_back(decoder, list(range(1, beams + 1))) == 0
    assert planned[0] and not planned[1]
    for x, y in zip(*results):
        assert torch.equal(x, y)
    history, scores, lengths = results[0]
    assert len({tuple(t) for t in history.tolist()}) == beams
    logits = _forced(decoder, prompt, history.T.contiguous())
    each = torch.log_softmax(logits.double(), 2).gather(2, history.T.long()[..., None])[..., 0]
    counted = torch.arange(steps, device="cuda")[:, None] < lengths
    want, slack = (each * counted).sum(0), (2 * _off(logits) * counted).sum(0)
    assert (want - scores.double()).abs().le(slack + 2.0 ** -20 * scores.abs()).all()


def test_scores_of_a_planned_beam_search_are_those_of_its_tokens(planned):
    """Against the plain decoder in 64 bits: the cache's rounding moves a logit by some 5 % of their spread at most, its log-probability by twice that."""
    import torch
    E, decoder = _decoder(3, 130, 8)
    import beam_search as B
    prompt = torch.randint(0, 1024, (130,), generator=torch.Generator().manual_seed(6)).cuda()
    tokens, scores, lengths = B.beam_search(_promised(decoder, 60000), prompt, 3, 8, end_token=5)
    assert planned[0] and not planned[1]
    for row, score, length in zip(tokens.tolist(), scores.tolist(), lengths.tolist()):
        so_far, total, slack = prompt.tolist(), 0.0, 0.0
        for t in row[:length]:
            want = _plain_logits(decoder, np.array(so_far))
            slack += 2 * 0.05 * max(np.abs(want - want.mean()).mean(), 1e-3) * 4
            total += want[t] - want.max() - np.log(np.exp(want - want.max()).sum())
            so_far.append(t)
        assert abs(total - score) <= slack
