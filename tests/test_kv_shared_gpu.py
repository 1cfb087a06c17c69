"""Attention over pages that sequences share on the GPU, against the CPU oracle."""
import math

import numpy as np
import pytest

from kv_many_util import DEV, Groups, dev, modules
from kv_util import PAGE

pytestmark = pytest.mark.gpu

# prompts of no page, of whole pages, that end inside one; alone in their group; sequences that end at the prompt's end
TOKENS = [(640, [(1, 5), (1, 70), (1, 1)]), (130, [(1, 3)]), (50, [(1, 9), (1, 90)]), (1000, [(1, 24), (1, 25), (1, 200), (1, 1), (1, 64)]), (64, [(1, 1), (1, 0)])]
DRAFTS = [(640, [(3, 5), (0, 70), (4, 4)]), (300, [(2, 3)]), (150, [(5, 9), (5, 90), (1, 1)]), (0, [(2, 2), (3, 1), (2, 70)]), (700, [(4, 130), (2, 2), (3, 0)])]
ONE = [(900, [(1, 1 + 11 * i) for i in range(23)])]
SMALL = [(128 + 64 * i, [(1, 3), (1, 40)]) for i in range(9)]


def _run(groups, fmt, dim, heads, group, dtype, window=0, sinks=0, seed=0, planned=True, **more):
    g = Groups(groups, fmt, dim, heads, group, dtype, seed, **more)
    if planned is not None:
        assert g.planned(window, sinks) == planned
    g.share(window, sinks)
    g.attend(window, sinks)
    g.check(window, sinks)
    assert g.prefix.tolist() == g.common_tokens()
    return g


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("groups", [TOKENS, DRAFTS, ONE, SMALL])
@pytest.mark.parametrize("dim,heads,group,dtype", [(128, 2, 4, "float16"), (128, 1, 1, "bfloat16"), (64, 3, 5, "bfloat16"), (64, 1, 12, "float16"),
                                                   (256, 2, 2, "float16"), (256, 1, 7, "bfloat16"), (128, 1, 11, "bfloat16")])
def test_against_the_oracle(fmt, groups, dim, heads, group, dtype):
    _run(groups, fmt, dim, heads, group, dtype, seed=dim + group)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (70, 0), (700, 0), (70, 3), (200, 65), (30, 5000), (10000, 4)])
@pytest.mark.parametrize("groups", [TOKENS, DRAFTS, ONE])
@pytest.mark.parametrize("dim,group", [(64, 2), (128, 4), (256, 3)])
def test_with_a_window_and_first_tokens(fmt, window, sinks, groups, dim, group):
    # (a short window leaves too little to read for a plan)
    _run(groups, fmt, dim, 2, group, "float16", window, sinks, seed=dim + window, planned=None)


@pytest.mark.parametrize("window,sinks", [(2100, 0), (2100, 3), (1950, 65), (30, 5000), (1100, 1000), (1600, 700)])
@pytest.mark.parametrize("rows,dim,group,fmt", [(1, 64, 4, "int8"), (1, 128, 8, "fp8"), (3, 128, 4, "int8"), (1, 256, 4, "fp8"), (2, 128, 16, "fp8")])
def test_planned_with_a_window_and_first_tokens(rows, dim, group, fmt, window, sinks):
    groups = [(2000, [(rows, rows + 11 * i) for i in range(20)]), (1400, [(rows, 5 + 70 * i) for i in range(12)]), (2200, [(rows, 80)])]
    _run(groups, fmt, dim, 8, group, "float16", window, sinks, seed=dim + window, planned=True)


@pytest.mark.parametrize("groups", [TOKENS, DRAFTS, ONE])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
def test_short_calls_run_without_a_plan(groups, window, sinks):
    _run(groups, "int8", 64, 2, 2, "float16", window, sinks, max_tokens=None, planned=False)  # (8 us by themselves)
    g = Groups(groups, "int8", 128, 2, 40, "float16", 1)  # (neither do rows that fill large tiles by themselves)
    assert g.planned(window, sinks) == (40 * max(g.counts) <= 64 and not window)


@pytest.mark.parametrize("rows,each", [(1, 40), (2, 20), (5, 3)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_tall_groups(rows, each, dim):
    _run([(2000, [(rows, rows + 3 * i) for i in range(each)])], "int8", dim, 2, 12 if rows < 5 else 8, "bfloat16", seed=rows, planned=True)


def test_sequences_without_slots_and_with_room_in_max_tokens():
    _run(TOKENS, "int8", 128, 2, 4, "float16", slots=False, max_tokens=70000, apart=0)
    _run(DRAFTS, "fp8", 64, 2, 2, "bfloat16", slots=False, max_tokens=19000, apart=0)


def test_many_sequences():
    rng = np.random.default_rng(2)
    groups = [(int(rng.integers(0, 400)), [(1, int(rng.integers(1, 90))) for _ in range(int(rng.integers(0, 9)))]) for _ in range(300)]
    _run(groups, "int8", 64, 1, 2, "float16")


def test_entries_of_no_group_attend_for_themselves():
    g = Groups(ONE + TOKENS, "int8", 128, 2, 4, "float16", 3)
    # the groups cover the entries 2 .. 20 alone, and one of them is empty
    g.starts, g.group_start = dev(g.torch, np.array([2, 9, 9, 21], dtype=np.int32)), np.array([2, 9, 9, 21])
    g.prefix = g.prefix[:3].contiguous()
    g.share()
    g.attend()
    g.check()
    assert g.prefix.tolist() == g.common_tokens()


def test_pages_past_the_first_difference_are_not_shared():
    # (the same page again behind one that differs; ids that differ in the first place)
    def change(pool, tables, order):
        tables["table"][order[3], 4] = tables["table"][order[3], 11]
        tables["table"][order[24], 0] = tables["table"][order[24], 1]
    g = _run(ONE + [(200, [(1, 5), (1, 6)])], "int8", 128, 2, 4, "float16", change=change)
    assert g.prefix.tolist() == [256, 0]


def test_a_page_that_reads_as_nan_reaches_the_sequences_that_hold_it():
    def change(pool, tables, order):
        pool["scales"][:, tables["table"][order[2], tables["lengths"][order[2]] // PAGE]] = math.nan  # (the last one of a sequence)
    _run(ONE, "int8", 128, 1, 4, "float16", change=change)
    def shared(pool, tables, order):  # noqa: E306
        pool["scales"][:, tables["table"][order[2], 3], 0] = math.nan
        pool["scales"][:, tables["table"][order[2], 5], 1] = 0.0
    _run(ONE, "fp8", 128, 2, 4, "float16", change=shared)


def test_a_plan_for_other_numbers_is_not_used():
    g = Groups(ONE, "int8", 128, 2, 4, "float16", 1)
    for plan in ("none", "window"):
        if plan == "window":
            g.share(window=100)
        g.attend()
        g.torch.cuda.synchronize()
        assert g.torch.isnan(g.got).all() and g.torch.isnan(g.lse).all()
    g.share()
    g.attend()
    g.check()


def test_group_starts_that_do_not_ascend():
    # (the same entries in two groups: unspecified results at most)
    g = Groups(TOKENS + ONE, "int8", 128, 2, 4, "float16", 1)
    g.starts = dev(g.torch, np.array([3, 20, 1, 30, -5, 99, 7], dtype=np.int32))
    g.prefix = g.torch.zeros(6, dtype=g.torch.int32, device=DEV)
    g.share()
    g.attend()
    g.torch.cuda.synchronize()
    assert g.torch.isnan(g.out[:, g.q_heads * g.dim:]).all()


@pytest.mark.parametrize("groups", [TOKENS, DRAFTS, ONE])
def test_the_same_bits_every_time_and_on_any_stream(groups):
    g = _run(groups, "int8", 128, 2, 4, "float16", seed=4)
    first, flse = g.got.clone(), g.lse.clone()
    side = g.torch.cuda.Stream()
    for stream in (None, side):
        g.got.fill_(math.nan)
        g.plan.fill_(0x7F)
        g.workspace.fill_(0x7F)
        if stream:
            stream.wait_stream(g.torch.cuda.current_stream())
        g.share(stream=stream)
        g.attend(stream=stream)
        g.torch.cuda.synchronize()
        assert g.torch.equal(g.got, first) and g.torch.equal(g.lse, flse)


def test_one_plan_for_all_layers_in_a_graph():
    g = Groups(TOKENS + ONE, "fp8", 128, 2, 4, "bfloat16", 8)
    outs = [g.torch.empty_like(g.got) for _ in range(2)]

    def step():
        g.share()
        for layer in range(2):
            g.attend(layer=layer)
            outs[layer].copy_(g.got)
    step()
    eager = [o.clone() for o in outs]
    graph = g.torch.cuda.CUDAGraph()
    with g.torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for o in outs:
            o.fill_(math.nan)
        g.plan.fill_(0)
        graph.replay()
        g.torch.cuda.synchronize()
        assert all(g.torch.equal(o, e) for o, e in zip(outs, eager))
        (g.Q.float() * 2).sum().item()  # (eager work between the replays)
    g.got.copy_(outs[0])
    g.attend(layer=0)
    g.check(layer=0)


@pytest.mark.parametrize("dim,heads,group", [(64, 2, 4), (64, 2, 1), (128, 1, 8), (256, 1, 4), (256, 2, 1)])
def test_sequences_that_end_with_the_shared_pages(dim, heads, group):
    # (no sequence has a page of its own)
    _run([(640, [(1, 0)] * 40), (1280, [(1, 0)] * 3)], "int8", dim, heads, group, "float16", seed=dim)


@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
def test_more_groups_and_sequences_than_threads_plan_them(window, sinks):
    rng = np.random.default_rng(3)
    groups = [(int(64 * rng.integers(0, 4)), [(1, int(rng.integers(1, 90))) for _ in range(2 if i % 5 else 0)]) for i in range(1500)]
    _run(groups, "int8", 64, 1, 2, "float16", window, sinks, planned=None if window else True)


def test_rows_of_no_sequence_are_left_as_they_were():
    g = _run(DRAFTS, "int8", 128, 2, 4, "float16")  # (the plan knows all rows, and keeps its contents)
    for rows in (g.rows - 1, g.rows - 7, 0):
        g.start = np.minimum(g.start, rows)
        g.row_start = dev(g.torch, g.start)
        g.got.fill_(math.nan)
        g.lse.fill_(math.nan)
        g.share()
        g.attend()
        g.check()
        assert g.torch.isnan(g.got[rows:]).all() and g.torch.isnan(g.lse[rows:]).all()


def test_a_plan_for_one_row_more():
    # (other lengths than the plan's last ones, in the same memory)
    g = _run(ONE, "fp8", 128, 2, 4, "float16", seed=2)
    lengths = g.tables["lengths"]
    grows = [s for s in g.order if lengths[s] % PAGE]
    lengths[grows] -= 1
    g.dt.lengths.copy_(g.torch.from_numpy(lengths))
    g.share()
    g.attend()
    g.check()


@pytest.mark.parametrize("differs", [False, True])
def test_more_sequences_in_a_group_than_are_held(differs):
    def change(pool, tables, order):
        if differs:
            tables["table"][order[1090], 1] = tables["table"][order[1090], 3]
    g = _run([(192, [(1, 1 + i % 70) for i in range(1100)])], "int8", 64, 1, 1, "float16", change=change)
    assert g.prefix.tolist() == [64 if differs else 192]
