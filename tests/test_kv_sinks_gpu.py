"""Attention over a sliding window and the first tokens on the GPU, against the CPU oracle."""
import math

import numpy as np
import pytest

from kv_many_util import DEV, activations, compare, dev, modules, starts
from kv_util import PAGE, make_pool, make_tables, pages_of, stale_slots, upload

pytestmark = pytest.mark.gpu


def _attend(fmt, dim, heads, group, dtype, entries, window, sinks, seed=0, slots=True, apart=8, max_tokens=None, change=None):
    """entries: (rows, tokens).  Runs the call, compares it with the oracle, returns what a test may look at."""
    torch, S = modules()
    rng = np.random.default_rng(3000 + seed)
    counts, lengths = [n for n, _ in entries], [t for _, t in entries]
    pages = sum(pages_of(t) for t in lengths) + 3
    pool = make_pool(rng, 2, pages, heads, dim, fmt)
    order = rng.permutation(len(entries)) if slots else np.arange(len(entries))
    by_slot = np.zeros(len(entries), dtype=int)
    by_slot[order] = lengths
    tables = make_tables(rng, by_slot, max(1, max(pages_of(t) for t in lengths)), pages)
    stale_slots(pool, tables, fmt, dim)
    if change:
        change(pool, tables, order)
    cache, dt = upload(S, pool, tables, fmt)
    start = starts(counts)
    rows, q_heads = int(start[-1]), heads * group
    Q, q = activations(torch, rng, rows, q_heads, dim, dtype, apart)
    out = torch.full((rows, q_heads * dim + apart), math.nan, dtype=getattr(torch, dtype), device=DEV)
    got = out[:, :q_heads * dim].view(rows, q_heads, dim)
    lse = torch.full((rows, q_heads), math.nan, dtype=torch.float32, device=DEV)
    most, tokens = max(counts), max_tokens or max(1, max(lengths))
    ws = torch.full((S.sfmp_kv_attention_workspace(cache.layout, len(entries), rows, q_heads, most, tokens),), 0xFF, dtype=torch.uint8, device=DEV)
    scale = 1.0 / math.sqrt(dim)
    ragged = any(n != 1 for n in counts) or not slots
    args = (cache, 1, dt, dev(torch, order.astype(np.int32)) if slots else None, dev(torch, start) if ragged else None, Q, got, most, tokens, scale,
            ws, window, sinks)
    S.sfmp_kv_attention_sinks(*args, lse=lse)
    torch.cuda.synchronize()
    assert torch.isnan(out[:, q_heads * dim:]).all() or apart == 0
    compare(pool, tables, order, start, q, got, lse, fmt, dtype, scale, window, sinks)
    return args, got, lse


TOKENS = [(1, 1), (1, 63), (1, 64), (1, 65), (1, 500), (1, 1000), (1, 2)]
DRAFTS = [(3, 3), (4, 64), (1, 200), (0, 70), (5, 266), (4, 700), (2, 1), (3, 0)]
CHUNKS = [(40, 40), (17, 130), (1, 300), (33, 397), (0, 5), (64, 64), (9, 4), (65, 600)]
MANY = [(40, 40), (1, 130), (33, 64), (40, 365), (17, 128), (0, 100), (39, 229), (40, 500)] * 4
# nothing between window and first tokens, a page or many; first tokens that end inside, at and behind a page; of a window of one token
MASKS = [(1, 1), (1, 64), (70, 3), (64, 65), (100, 200), (300, 5), (33, 128), (5000, 7), (40, 5000)]


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("window,sinks", MASKS)
@pytest.mark.parametrize("dim,heads,group,dtype", [(128, 2, 4, "float16"), (64, 1, 5, "bfloat16"), (256, 1, 17, "float16"), (128, 1, 20, "bfloat16")])
def test_single_tokens(fmt, window, sinks, dim, heads, group, dtype):
    _attend(fmt, dim, heads, group, dtype, TOKENS, window, sinks, seed=dim + group)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("window,sinks", [(1, 1), (70, 3), (64, 65), (100, 130)])
@pytest.mark.parametrize("dim,heads,group,dtype", [(128, 2, 4, "bfloat16"), (64, 2, 3, "float16"), (256, 1, 2, "float16"), (128, 1, 7, "float16")])
def test_a_few_rows(fmt, window, sinks, dim, heads, group, dtype):
    _attend(fmt, dim, heads, group, dtype, DRAFTS, window, sinks, seed=dim + group + window)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,entries,max_tokens", [(2, 4, TOKENS, 20000), (8, 2, TOKENS, 60000), (2, 6, DRAFTS, 20000), (8, 6, DRAFTS, 60000),
                                                            (4, 4, MANY, None), (2, 4, CHUNKS, None), (2, 4, CHUNKS, 9000), (4, 4, MANY, 9000)])
@pytest.mark.parametrize("window,sinks", [(60, 70), (130, 2)])
def test_every_form(fmt, dim, heads, group, entries, max_tokens, window, sinks):
    _attend(fmt, dim, heads, group, "float16" if dim == 128 else "bfloat16", entries, window, sinks, max_tokens=max_tokens, seed=dim + heads)


@pytest.mark.parametrize("rows,tokens,heads,group,window,sinks", [(1, 9000, 1, 8, 100, 4), (2, 9000, 2, 4, 5000, 500), (130, 3000, 1, 4, 200, 130),
                                                                  (257, 900, 1, 8, 300, 65), (300, 1500, 4, 4, 64, 64), (1, 9000, 1, 4, 4500, 4400)])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_one_sequence(fmt, rows, tokens, heads, group, window, sinks):
    _attend(fmt, 128, heads, group, "float16", [(rows, tokens)], window, sinks, seed=tokens)


def test_pages_between_first_tokens_and_window_are_not_read():
    # their scales are NaN, and their place in the table names no page
    def change(pool, tables, order):
        for s, n in enumerate(tables["lengths"]):
            for place in range(2, (n - 200) // PAGE - 1):
                pool["scales"][:, tables["table"][s, place]] = math.nan
    for entries in ([(1, 2000), (1, 777)], [(30, 2000), (9, 777)], [(100, 1500)]):
        args, got, lse = _attend("int8", 128, 2, 4, "float16", entries, 64, 128, change=change)
        first, flse = got.clone(), lse.clone()
        table = args[2].page_table
        for b, (_, n) in enumerate(entries):
            table[int(args[3][b]), 2:(n - 200) // PAGE - 1] = -1
        got.fill_(math.nan)
        modules()[1].sfmp_kv_attention_sinks(*args, lse=lse)
        assert modules()[0].equal(got, first) and modules()[0].equal(lse, flse)


@pytest.mark.parametrize("entries", [TOKENS, DRAFTS, [(200, 900)]])
def test_without_first_tokens_or_window_it_is_the_other_call(entries):
    torch, S = modules()
    for window, sinks in ((0, 9), (70, 0), (2 ** 31 - 1, 5), (0, 0)):
        args, got, lse = _attend("fp8", 128, 2, 2, "bfloat16", entries, window, sinks)
        other, olse = torch.empty_like(got), torch.empty_like(lse)
        S.sfmp_kv_attention(*args[:6], other, *args[7:11], window=window, lse=olse)
        assert torch.equal(got, other) and torch.equal(lse, olse)
    args, got, lse = _attend("fp8", 128, 2, 2, "bfloat16", entries, 1, 2 ** 31 - 1)  # (every token is a first one)
    S.sfmp_kv_attention(*args[:6], other, *args[7:11], lse=olse)
    assert torch.allclose(got.float(), other.float(), rtol=2.0 ** -7, atol=2.0 ** -10)


@pytest.mark.parametrize("entries", [[(1, 5000)] * 3, DRAFTS, CHUNKS])
def test_the_same_bits_every_time_and_on_any_stream(entries):
    torch, S = modules()
    args, got, lse = _attend("int8", 128, 2, 4, "float16", entries, 300, 70, seed=4)
    first, flse = got.clone(), lse.clone()
    side = torch.cuda.Stream()
    for stream in (None, side):
        got.fill_(math.nan)
        args[10].fill_(0x7F)
        if stream:
            stream.wait_stream(torch.cuda.current_stream())
        S.sfmp_kv_attention_sinks(*args, lse=lse, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got, first) and torch.equal(lse, flse)
