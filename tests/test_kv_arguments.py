"""What the binding of the cache and sampling calls does with arguments before the library sees them (no GPU)."""
import math
import random

import numpy as np
import pytest

from oracle import sfmp_kv_oracle as O
import paper_2602_01027_amd as S


def test_a_workspace_has_to_be_contiguous_memory_of_the_gpu():
    import torch
    for bad in (torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8).expand(1 << 16), 1 << 20):
        with pytest.raises(ValueError, match="workspace has to be"):
            S.kv._workspace(bad)
    assert S.kv._workspace(None) == (None, 0) and S.kv._workspace(torch.zeros(0)) == (None, 0)


def test_a_workspace_is_enough_for_smaller_calls():
    """Forms that need none and forms that need much follow each other as a call grows: 512 sequences of 8192 tokens are cut into parts, 513 are
    not; 77 rows of 131072 tokens are cut into slices, 78 are not."""
    L = S.sfmp_kv_query(16, 8, 128)
    assert S.sfmp_kv_attention_workspace(L, 513, 513, 32, 1, 8192) >= S.sfmp_kv_attention_workspace(L, 512, 512, 32, 1, 8192) > 4 << 20
    assert S.sfmp_sample_workspace(78, 131072) >= S.sfmp_sample_workspace(77, 131072) > 7 << 20
    assert S.sfmp_sample_workspace(1, 1000) == 256 and S.sfmp_kv_attention_workspace(L, 1, 1, 32, 1, 64) == 256


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_workspaces_never_fall_as_calls_grow(dim):
    rng = random.Random(dim)
    log = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))  # noqa: E731
    seen = set()
    for _ in range(4000):
        heads, group = rng.choice((1, 2, 8, 16)), rng.choice((1, 2, 4, 5, 8, 16, 40))
        L = S.sfmp_kv_query(16, heads, dim)
        big = [log(1, 700), log(1, 300), log(1, 40000)]  # entries, rows of one, tokens
        for k in range(3):
            if rng.random() < 0.2:
                big[k] = rng.choice(((255, 256, 257, 511, 512, 513), (16, 17, 32, 64, 65), (64, 1024, 1025, 2048, 2049))[k])
        small = [max(1, log(1, n)) if rng.random() < 0.6 else max(1, n - 1) for n in big]
        size = lambda b, r, t: S.sfmp_kv_attention_workspace(L, b, b * r, heads * group, r, t)  # noqa: E731
        assert size(*small) <= size(*big), (heads, group, small, big)
        assert S.sfmp_kv_attention_workspace(L, small[0], small[0] + small[1] - 1, heads * group, small[1], small[2]) <= size(*big)
        seen.add(size(*small))
    assert len(seen) >= 3


def test_workspaces_of_sampling_never_fall_as_calls_grow():
    rng = random.Random(3)
    for _ in range(4000):
        rows, vocab = rng.randint(1, 130), int(math.exp(rng.uniform(0, math.log(1 << 24))))
        assert S.sfmp_sample_workspace(rng.randint(0, rows), rng.randint(1, vocab)) <= S.sfmp_sample_workspace(rows, vocab)
        assert S.sfmp_sample_workspace(rows - 1, vocab) <= S.sfmp_sample_workspace(rows, vocab)


def test_rows_of_a_head_stay_below_2_to_the_30():
    # (rows of an entry times query heads of a key head are counted in 32 bits)
    L = S.sfmp_kv_query(16, 1, 64)
    assert S.sfmp_kv_attention_workspace(L, 1, 2 ** 28, 4, 2 ** 28, 64) > 0
    for rows, heads in ((2 ** 28 + 1, 4), (2 ** 30, 2), (2 ** 29, 4), (2 ** 26, 64)):
        with pytest.raises(S.SfmpError) as e:
            S.sfmp_kv_attention_workspace(L, 1, rows, heads, rows, 64)
        assert e.value.code == -2


@pytest.mark.parametrize("past", [2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 31 - 1, 2 ** 64 + 4])
def test_numbers_that_do_not_fit_32_bits_are_refused_not_cut_off(past):
    L = S.sfmp_kv_query(4, 2, 64)
    calls = [lambda k=k: S.sfmp_kv_query(*[past if i == k else (4, 2, 64, 0, 1)[i] for i in range(5)]) for k in range(5)]
    calls += [lambda k=k: S.sfmp_kv_attention_workspace(L, *[past if i == k else (1, 4, 2, 4, 100)[i] for i in range(5)]) for k in range(5)]
    calls += [lambda: S.sfmp_sample_workspace(past, 100), lambda: S.sfmp_sample_workspace(1, past),
              lambda: S.kv._batch(None, None, None, 1, past), lambda: S.kv._batch(None, None, None, past, 1)]
    for call in calls:
        with pytest.raises(ValueError, match="fit 32 bits"):
            call()


def test_slots_and_row_starts_have_to_be_vectors():
    import torch
    for bad in ([0], 3, torch.zeros((), dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int32)):
        for slots, row_start in ((bad, None), (None, bad)):
            with pytest.raises(ValueError, match="has to be a vector"):
                S.kv._batch(None, slots, row_start, 1, 1)


def test_sizes_past_the_limits_of_the_header():
    L = S.sfmp_kv_query(16, 8, 128)
    size = lambda batch=1, q_heads=8, tokens=64: S.sfmp_kv_attention_workspace(L, batch, batch, q_heads, 1, tokens)  # noqa: E731
    assert size(batch=65535) and size(q_heads=65536) and size(tokens=2 ** 26) and S.sfmp_sample_workspace(65535, 2 ** 24)
    for past in (lambda: size(batch=65536), lambda: size(q_heads=65544), lambda: size(q_heads=12), lambda: size(tokens=2 ** 26 + 1), lambda: size(tokens=0),
                 lambda: S.sfmp_sample_workspace(65536, 10), lambda: S.sfmp_sample_workspace(1, 2 ** 24 + 1), lambda: S.sfmp_sample_workspace(-1, 10),
                 lambda: S.sfmp_sample_workspace(1, 0)):
        with pytest.raises(S.SfmpError) as e:
            past()
        assert e.value.code == -2


def test_log_probability_of_a_tie_at_temperature_0():
    x = np.array([1.0, 7.0, 7.0, -3.0, 7.0, 6.99])
    assert O.sample(x, 0.0, 0, 1.0, 0.0, 0.9)[:2] == (1, pytest.approx(-math.log(3)))
    assert O.sample(x[:2], 0.0, 0, 1.0, 0.0, 0.9)[:2] == (1, 0.0)
