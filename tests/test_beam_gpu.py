"""One step of a beam search on the GPU, against the CPU oracle."""
import math

import numpy as np
import pytest

from oracle import sfmp_kv_oracle as O
from kv_util import U32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = ("float16", "bfloat16", "float32")


def _torch():
    import torch
    assert torch.cuda.is_available()
    import paper_2602_01027_amd as S
    return torch, S


def _call(x, beams, scores, choices, weights=None, ended=None, end_token=0, dtype="float32", offset=0, gap=0, stream=None, fill=0xFF):
    """x float [rows, vocab] as numpy.  Rows of the call lie `gap` elements apart, the first one `offset` behind an aligned address."""
    torch, S = _torch()
    rows, vocab = x.shape
    flat = torch.full((offset + rows * (vocab + gap),), math.nan, dtype=getattr(torch, dtype), device=DEV)
    logits = flat[offset:].view(rows, vocab + gap)[:, :vocab]
    logits.copy_(torch.from_numpy(x.astype(np.float32)))
    up = lambda a, t: None if a is None else torch.from_numpy(np.asarray(a).astype(t)).to(DEV)  # noqa: E731
    requests = rows // beams
    out = [torch.full((requests, choices), 77, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    ws = torch.full((S.sfmp_beam_select_workspace(requests, beams, vocab, choices),), fill, dtype=torch.uint8, device=DEV)
    S.sfmp_beam_select(logits, beams, up(scores, np.float32), up(weights, np.float32), up(ended, np.int32), end_token, *out, ws, stream=stream)
    torch.cuda.synchronize()
    return logits.float().cpu().numpy(), [o.cpu().numpy() for o in out]


def _check(x, beams, scores, choices, weights=None, ended=None, end_token=0, exact=False, **more):
    """exact: the oracle's own ties are the kernel's (equal rows, or all terms in 64 bits)."""
    scores = np.asarray(scores, dtype=np.float32)
    weights = None if weights is None else np.asarray(weights, dtype=np.float32)
    held, (values, parents, tokens) = _call(x, beams, scores, choices, weights, ended, end_token, **more)
    for r in range(len(x) // beams):
        rows = slice(r * beams, (r + 1) * beams)
        of = lambda a: None if a is None else a[rows]  # noqa: E731
        want, sums, slopes = O.beam_select(held[rows], scores[rows], choices, of(weights), of(ended), end_token)
        got = [(float(v), int(p) - r * beams, int(t)) for v, p, t in zip(values[r], parents[r], tokens[r])]
        assert all(p == (-math.inf, -1 - r * beams, -1) for p in got[len(want):]), got[len(want):]
        # a term of the sum carries the rounding of its argument, |d| log2(e) in fp32 with the product of the logarithm's lower half, some two
        # U32 of |d|, the difference's own U32, and three U32 of the exponential and of the sum of a run; in 64 bits everything else is less than 2^-40
        slack = U32 * (4.0 * slopes + 6.0) + 2.0 ** -36
        for (v, b, t), (gv, gb, gt) in zip(want, got):
            assert abs(gv - v) <= U32 * abs(v) * 1.01 + slack[b] + slack[gb] + (0 if gb == b else abs(gv) * U32), (r, v, b, t, gv, gb, gt)
        if exact:
            assert [w[1:] for w in want] == [g[1:] for g in got[:len(want)]], (r, want, got)
            continue
        # where the values around a rank lie further apart than they can be off, the continuation is the oracle's
        w = [1.0 if weights is None else float(weights[rows][b]) for _, b, _ in want]
        keys = [v * k for (v, _, _), k in zip(want, w)]
        for i, (v, b, t) in enumerate(want):
            clear = all(abs(keys[i] - keys[j]) > 4 * w[i] * (slack[b] + slack[want[j][1]]) or b == want[j][1] for j in (i - 1, i + 1) if 0 <= j < len(want))
            if clear and i + 1 < len(want):
                assert got[i][1:] == (b, t), (r, i, want, got)
        assert len(set(g[1:] for g in got[:len(want)])) == len(want)
    return values, parents, tokens


def _logits(rng, rows, vocab, beams, std=2.0):
    x = rng.normal(0.0, std, (rows, vocab))
    x += np.repeat(np.where(rng.random((rows // beams, vocab)) < min(0.25, 300 / vocab), rng.exponential(3.0, (rows // beams, vocab)), 0.0), beams, axis=0)
    x[rng.random((rows, vocab)) < 0.01] = -math.inf
    return x


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("requests,beams,vocab,choices,offset,gap", [
    (1, 4, 32000, 8, 0, 0), (1, 1, 1, 1, 0, 0), (2, 1, 7, 3, 1, 0), (3, 5, 1003, 10, 3, 5), (1, 32, 5000, 64, 0, 1), (2, 3, 4095, 6, 7, 0), (2, 3, 4097, 6, 0, 1),
    (1, 2, 16384, 64, 0, 0), (40, 8, 9001, 16, 0, 0), (7, 32, 20011, 32, 5, 3), (700, 3, 300, 3, 0, 0), (1, 8, 131072, 16, 0, 0)])
def test_against_the_oracle(dtype, requests, beams, vocab, choices, offset, gap):
    rng = np.random.default_rng(vocab + beams)
    rows = requests * beams
    x = _logits(rng, rows, vocab, beams)
    _check(x, beams, rng.normal(-40.0, 3.0, rows), choices, dtype=dtype, offset=offset, gap=gap)


@pytest.mark.parametrize("dtype", DTYPES)
def test_pieces_of_several_chunks(dtype):
    rng = np.random.default_rng(3)
    _check(_logits(rng, 2, 1500007, 2), 2, [-3.0, -4.0], 64, dtype=dtype)       # few rows: 128 pieces of each
    _check(_logits(rng, 4 * 32, 70001, 32), 32, rng.normal(-9, 2, 128), 64, dtype=dtype)  # 8 pieces of each
    rising = np.sort(rng.normal(0.0, 3.0, (2, 600011)), axis=1)                  # every chunk has larger ones
    _check(rising, 2, [-3.0, -3.1], 64, dtype=dtype)
    _check(rising[:, ::-1].copy(), 2, [-3.0, -3.1], 64, dtype=dtype)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
def test_ended_beams_and_weights(dtype, weighted):
    rng = np.random.default_rng(8)
    requests, beams, vocab = 6, 6, 3001
    rows = requests * beams
    ended = rng.random(rows) < 0.4
    ended[:beams] = True   # a request of which all have
    ended[beams:2 * beams] = False
    weights = 1.0 / rng.integers(5, 60, rows) if weighted else None
    _check(_logits(rng, rows, vocab, beams), beams, rng.normal(-30.0, 4.0, rows), 12, weights, ended, 2, dtype=dtype)


def test_fewer_continuations_than_wanted():
    x = np.full((6, 50), -math.inf)
    x[0, [3, 7]] = 1.0, 2.0
    x[2, 49] = -5.0
    x[4] = 0.0
    x[5] = math.nan
    values, parents, tokens = _check(x, 2, [0.0, -1.0, -2.0, -3.0, -math.inf, -1.0], 4, exact=True)
    assert parents.tolist() == [[0, 0, -1, -1], [2, -1, -1, -1], [-1] * 4] and tokens[0].tolist() == [7, 3, -1, -1]
    values, parents, tokens = _check(x, 3, [math.nan] * 3 + [0.0, 0.0, 0.0], 3, exact=True)
    assert parents.tolist() == [[-1] * 3, [4] * 3]


@pytest.mark.parametrize("dtype", DTYPES)
def test_equal_continuations_come_in_the_order_of_rows_and_tokens(dtype):
    rng = np.random.default_rng(1)
    for vocab in (5, 700, 40007, 300011):
        flat = np.zeros((4, vocab))
        for choices in (1, 4, 64):
            _check(flat, 4, [-1.0] * 4, choices, dtype=dtype, exact=True, gap=1, offset=1)
        few = np.tile(rng.integers(0, 3, (1, vocab)), (8, 1)).astype(float)  # equal rows of three values
        _check(few, 4, [-1.0] * 8, 64, dtype=dtype, exact=True, gap=3)
        _check(few, 4, [-1.0, -1.0, -3.0, -1.0] * 2, 30, dtype=dtype, exact=True, offset=5)
    x = np.zeros((1, 100))
    x[0, 40:60] = -0.0
    _check(x, 1, [0.0], 64, dtype=dtype, exact=True)


@pytest.mark.parametrize("rows,beams,vocab", [(4, 2, 9001), (64, 4, 70001), (256, 8, 33000), (2, 1, 20)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_which_few_tokens_are_left(dtype, rows, beams, vocab):
    # (all logits of a few threads are larger than the rest)
    rng = np.random.default_rng(11)
    for choices, left in ((64, 3900), (64, 66), (17, 500), (5, 130), (2, 9)):
        x = np.full((rows, vocab), -math.inf)
        start = rng.integers(0, max(vocab - left, 1), rows)
        for i in range(rows):
            x[i, start[i]:start[i] + left] = rng.normal(0.0, 2.0, x[i, start[i]:start[i] + left].shape)
        scores = rng.normal(-5.0, 1.0, rows)
        _check(x[:2 * beams], beams, scores[:2 * beams], choices, dtype=dtype)
        if choices != 64:
            _check(x, beams, scores, choices, dtype=dtype)
        x[:] = np.where(np.isfinite(x[0]), 3.0, -math.inf)  # equal ones in equal rows
        _check(x[:2 * beams], beams, [-1.0] * 2 * beams, choices, dtype=dtype, exact=True)


def test_many_beams_of_short_pieces():
    rng = np.random.default_rng(12)
    _check(_logits(rng, 32, 50000, 32), 32, rng.normal(-9, 2, 32), 64, dtype="float16")
    _check(_logits(rng, 32, 50000, 32, std=0.01), 32, [-3.0] * 32, 64, dtype="bfloat16")  # (close together: many equal logits)
    _check(_logits(rng, 32, 3000, 32), 32, [0.0] + [-math.inf] * 31, 64)


def test_infinities_and_no_numbers():
    rng = np.random.default_rng(4)
    for dtype in DTYPES:
        x = _logits(rng, 4, 9001, 2)
        x[0, [5, 8000]] = math.inf
        x[1, ::3] = math.nan
        x[2, 77] = math.nan
        x[3] = math.inf
        _check(x, 2, [-1.0, -2.0, -3.0, -4.0], 20, dtype=dtype)


def test_values_closer_together_than_fp32_tells_apart():
    # log-probabilities of 1/2 and 1/3, scores whose difference is that of the two, rounded to fp32: only 64 bits see which is larger
    x = np.full((2, 64), -math.inf)
    x[0, :2], x[1, :3] = 0.0, 0.0
    for low in (-3.0, -17.3, -50.7, -80.1):
        a = np.float32(low)
        b = np.float32(float(a) + math.log(3) - math.log(2))
        for s in (b, np.nextafter(b, np.float32(0)), np.nextafter(b, np.float32(-99))):
            _check(x, 2, [a, s], 5, exact=True)


def test_rows_of_large_and_small_spread():
    rng = np.random.default_rng(6)
    _check(rng.normal(0.0, 1e4, (4, 5003)), 2, [-1.0] * 4, 9, dtype="float16")
    _check(rng.normal(0.0, 1e36, (4, 5003)), 2, [-1.0] * 4, 9, dtype="bfloat16")
    _check(rng.normal(0.0, 1e-6, (4, 70001)), 2, [-1.0, -1.5] * 2, 9)
    _check(rng.normal(-300.0, 0.3, (4, 70001)), 2, [-1e5, -1e5 + 1, 0.0, 3.0], 9)


def test_the_same_bits_every_time_on_any_stream_and_in_a_graph():
    torch, S = _torch()
    rng = np.random.default_rng(5)
    x, scores = _logits(rng, 24, 50021, 6), rng.normal(-40, 3, 24)
    first = _call(x, 6, scores, 12, dtype="bfloat16")[1]
    side = torch.cuda.Stream()
    again = _call(x, 6, scores, 12, dtype="bfloat16", stream=side, fill=0x11)[1] if side.wait_stream(torch.cuda.current_stream()) is None else None
    assert all(np.array_equal(a, b) for a, b in zip(first, again))
    logits = torch.from_numpy(x).to(DEV).bfloat16()
    s = torch.from_numpy(scores.astype(np.float32)).to(DEV)
    out = [torch.zeros((4, 12), dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    ws = [torch.empty(S.sfmp_beam_select_workspace(4, 6, 50021, 12), dtype=torch.uint8, device=DEV) for _ in range(2)]
    S.sfmp_beam_select(logits, 6, s, None, None, 0, *out, ws[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.sfmp_beam_select(logits, 6, s, None, None, 0, *out, ws[0])
    for _ in range(3):
        for o in out:
            o.zero_()
        other = [torch.zeros_like(o) for o in out]
        with torch.cuda.stream(side):
            S.sfmp_beam_select(logits, 6, s, None, None, 0, *other, ws[1])  # (a second call meanwhile)
        graph.replay()
        torch.cuda.synchronize()
        for o, p, f in zip(out, other, first):
            assert np.array_equal(o.cpu().numpy(), f) and np.array_equal(p.cpu().numpy(), f)


# ---- reordering ---------------------------------------------------------------------------------------------------------

def _reorder(n, sequences, table_pages, seed, parents=None, shared=True):
    torch, S = _torch()
    rng = np.random.default_rng(seed)
    pages = 40 + n * (table_pages + 1)
    table = np.full((sequences, table_pages), -1, dtype=np.int32)
    lengths, refs = np.zeros(sequences, dtype=np.int32), np.zeros(pages, dtype=np.int32)
    free = rng.permutation(pages).tolist()
    common = [free.pop() for _ in range(table_pages)]
    for s in range(sequences):
        lengths[s] = rng.integers(0, 64 * table_pages + 1) if s % 5 else 0
        k = O.pages_of(int(lengths[s]))
        same = int(rng.integers(0, k + 1)) if shared else 0
        mine = common[:same] + [free.pop() if len(free) else common[i] for i in range(same, k)]
        table[s, :k] = mine
        for page in mine:
            refs[page] += 1
    slots = rng.permutation(sequences)[:n].astype(np.int32)
    parents = rng.integers(-1, n, n).astype(np.int32) if parents is None else np.asarray(parents, dtype=np.int32)
    tables = dict(table=table, lengths=lengths, refs=refs)
    up = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    layout = S.sfmp_kv_query(pages, 1, 64)
    cache, dt = S.make_kv_cache(layout), S.DeviceKvTables(up(table), up(lengths), up(refs))
    S.sfmp_kv_reorder(cache, dt, up(slots), up(parents))
    O.reorder(tables, slots.tolist(), parents.tolist())
    assert np.array_equal(dt.lengths.cpu().numpy(), tables["lengths"])
    assert np.array_equal(dt.refs.cpu().numpy(), tables["refs"])
    assert np.array_equal(dt.page_table.cpu().numpy(), tables["table"])


@pytest.mark.parametrize("n,sequences,table_pages", [(1, 1, 1), (4, 9, 17), (8, 8, 3), (64, 64, 40), (64, 70, 300), (130, 150, 127), (1000, 1024, 16), (1024, 1024, 33),
                                                     (3, 3, 6000)])
@pytest.mark.parametrize("shared", [True, False])
def test_reorder(n, sequences, table_pages, shared):
    _reorder(n, sequences, table_pages, n + table_pages, shared=shared)


def test_reorder_with_given_parents():
    _reorder(6, 9, 20, 1, parents=[0, 1, 2, 3, 4, 5])
    _reorder(6, 9, 20, 2, parents=[1, 2, 3, 4, 5, 0])
    _reorder(6, 9, 20, 3, parents=[3] * 6)
    _reorder(6, 9, 20, 4, parents=[-1, 6, 2 ** 31 - 1, -2 ** 31, 4, 4])


def test_reorder_refuses_no_slot_but_leaves_those_out_of_range():
    torch, S = _torch()
    layout = S.sfmp_kv_query(8, 1, 64)
    cache, dt = S.make_kv_cache(layout), S.make_kv_tables(layout, 3, 4)
    up = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    dt.page_table[0, 0], dt.page_table[1, 0], dt.lengths[0], dt.lengths[1] = 5, 6, 10, 20
    dt.refs[5] = dt.refs[6] = 1
    S.sfmp_kv_reorder(cache, dt, up([0, -4, 1, 99]), up([2, 0, 1, 0]))  # (what a slot out of range was is nothing)
    assert dt.lengths.tolist() == [20, 0, 0] and dt.refs.tolist() == [0, 0, 0, 0, 0, 0, 1, 0] and dt.page_table[0, 0] == 6


def test_reorder_in_a_graph():
    torch, S = _torch()
    up = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    layout = S.sfmp_kv_query(600, 1, 64)
    cache, dt = S.make_kv_cache(layout), S.make_kv_tables(layout, 200, 100)
    slots, parents = torch.arange(200, dtype=torch.int32, device=DEV), torch.roll(torch.arange(200, dtype=torch.int32, device=DEV), 1)
    dt.lengths.copy_(torch.arange(200) * 3)
    dt.page_table.copy_(torch.arange(200)[:, None] % 600)
    graph = torch.cuda.CUDAGraph()
    S.sfmp_kv_reorder(cache, dt, slots, up(list(range(200))))
    with torch.cuda.graph(graph):
        S.sfmp_kv_reorder(cache, dt, slots, parents)
    for i in range(1, 4):
        graph.replay()
        assert dt.lengths.tolist() == [3 * ((s - i) % 200) for s in range(200)]
