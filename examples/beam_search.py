"""Beam search with the decoder of sample_continuations.py: quantised projections, the 8-bit paged cache, attention that reads the
pages which the beams share once for all of them.

    python examples/beam_search.py [--prompt 1000] [--beams 4] [--steps 64] [--penalty 1.0] [--eager]

The prompt is put into one sequence and forked into the beams.  A step reserves a token for each beam, finds what the beams share (the
prompt's pages, and what they have not parted in since) and plans their attention once, runs the layers, chooses the best
continuations of all beams and lets the sequences become their parents' (sfmp_kv_reorder: pages change hands, nothing is copied but
the last page of beams with one parent, when the next token is reserved).  Nothing in a step asks the host, so it is captured once as a graph."""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from sample_continuations import Decoder, S, Shape, give_back, room  # noqa: E402


def beam_search(decoder, prompt, beams, steps, end_token, penalty=1.0, graph=True):
    """(tokens int32 [beams, steps], scores [beams], lengths [beams]), the best first by score / length^penalty; a beam that has chosen end_token
    is left as it is from there on (end_token to the end).  Sequences 0 .. beams of the decoder have to be empty; the beams are left in 1 .. beams."""
    device, vocab = decoder.device, decoder.shape.vocab
    numbers = lambda a, b: torch.arange(a, b, dtype=torch.int32, device=device)  # noqa: E731
    zeros = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device=device)  # noqa: E731
    slots, groups = numbers(1, beams + 1), torch.tensor([0, beams], dtype=torch.int32, device=device)
    tokens, parents, ended, failed = zeros(1, beams), zeros(1, beams), zeros(beams), zeros(1)
    lengths, weights, history, place = zeros(beams, dtype=torch.float32), zeros(beams, dtype=torch.float32), zeros(beams, steps), zeros(1)
    scores, next_scores = zeros(beams, dtype=torch.float32), zeros(1, beams, dtype=torch.float32)
    workspace = torch.empty(S.sfmp_beam_select_workspace(1, beams, vocab, beams), dtype=torch.uint8, device=device)
    max_tokens = prompt.shape[0] + steps

    def choose(logits):
        """The best continuations, and everything that a beam has taken over from its parent."""
        weights.copy_((lengths + (ended == 0)) ** -penalty)
        S.sfmp_beam_select(logits, beams, scores, weights, ended, end_token, next_scores, parents, tokens, workspace)
        S.sfmp_kv_reorder(decoder.cache, decoder.tables, slots, parents[0])
        parent, token = parents[0].clamp(min=0).long(), tokens[0].clamp(min=0)  # (-1: no continuation is left; its score is -infinity)
        tokens[0].copy_(token)
        history.copy_(history[parent].scatter(1, place.expand(beams)[:, None].long(), token[:, None]))
        place.add_(1)
        lengths.copy_(lengths[parent] + (ended[parent] == 0))
        ended.copy_(ended[parent] | (token == end_token).int())
        scores.copy_(next_scores[0])

    def step():
        decoder.reserve(slots)
        failed.copy_(torch.where(failed == 0, decoder.status, failed))
        positions = decoder.tables.lengths[1:beams + 1] - 1
        choose(decoder.logits(decoder.run(tokens[0], positions, slots, None, 1, max_tokens, groups)))

    first = decoder.prefill(0, prompt)
    if int(decoder.status):  # (a prompt without room: nothing was reserved, and nothing may be appended for good)
        raise RuntimeError(f"no room for the prompt: {room(decoder.status)}")
    S.sfmp_kv_fork(decoder.cache, decoder.tables, torch.zeros(beams, dtype=torch.int32, device=device), slots)
    S.sfmp_kv_free(decoder.cache, decoder.tables, numbers(0, 1))  # (its pages are the beams' now)
    scores[1:] = float("-inf")  # (all beams are the same so far)
    choose(first.expand(beams, vocab).contiguous())
    captured = None
    for i in range(1, steps):
        if captured is not None:
            captured.replay()
        else:
            step()
            if graph:  # (the eager step has loaded every kernel; recording runs nothing)
                captured = torch.cuda.CUDAGraph()
                with torch.cuda.graph(captured):
                    step()
    if int(failed):  # (a step without room changes no length: the steps after it wrote over the last token)
        raise RuntimeError(f"no room for a token: {room(failed)}")
    return history, scores, lengths.long()


def main():
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--prompt", type=int, default=1000, help="tokens of the prompt")
    a.add_argument("--beams", type=int, default=4)
    a.add_argument("--steps", type=int, default=64)
    a.add_argument("--layers", type=int, default=2)
    a.add_argument("--penalty", type=float, default=1.0, help="beams rank by score / length^penalty")
    a.add_argument("--eager", action="store_true", help="launch every step instead of replaying a graph")
    a = a.parse_args()
    shape = Shape(layers=a.layers)
    each = (a.prompt + a.steps) // 64 + 2
    decoder = Decoder(shape, pages=each * (a.beams + 1), sequences=a.beams + 1, table_pages=each)
    prompt = torch.randint(0, shape.vocab, (a.prompt,), generator=torch.Generator().manual_seed(1)).to(decoder.device)
    for _ in range(2):  # (the first turn loads the kernels)
        torch.cuda.synchronize()
        start = time.perf_counter()
        tokens, scores, lengths = beam_search(decoder, prompt, a.beams, a.steps, 2, a.penalty, graph=not a.eager)
        torch.cuda.synchronize()
        took = time.perf_counter() - start
        held = int((decoder.tables.refs > 0).sum())
        print(f"{a.beams} beams x {a.steps} tokens after {a.prompt}: {took * 1e3:.1f} ms, scores {[round(x, 3) for x in scores.tolist()]}, {held} pages held "
              f"by sequences of {decoder.tables.lengths[1:].tolist()} tokens")
        print("  first tokens:", tokens[:, :6].tolist())
        give_back(decoder, list(range(1, a.beams + 1)))


if __name__ == "__main__":
    main()
