"""More requests than one reordering takes: choice for all of them, sequences that change places in several calls of whole requests."""
import numpy as np
import pytest

from oracle import sfmp_kv_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_reordering_in_calls_of_whole_requests():
    import torch
    import paper_2602_01027_amd as S
    rng = np.random.default_rng(1)
    requests, beams, vocab, table_pages = 300, 5, 700, 7  # (1500 sequences)
    rows = requests * beams
    lengths = rng.integers(0, 64 * table_pages + 1, rows).astype(np.int32)
    pages = int(sum(O.pages_of(int(n)) for n in lengths)) + 5
    table, refs, free = np.full((rows, table_pages), -1, dtype=np.int32), np.zeros(pages, dtype=np.int32), rng.permutation(pages).tolist()
    for s, n in enumerate(lengths):
        k = O.pages_of(int(n))
        table[s, :k] = [free.pop() for _ in range(k)]
        refs[table[s, :k]] += 1
    tables = dict(table=table, lengths=lengths, refs=refs)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    layout = S.sfmp_kv_query(pages, 1, 64)
    cache, dt = S.make_kv_cache(layout), S.DeviceKvTables(up(table), up(lengths), up(refs))
    x = rng.normal(0.0, 2.0, (rows, vocab)).astype(np.float32)
    x[rng.random(rows) < 0.3] = -np.inf  # (rows without a continuation: beams that are left empty where a request has too few)
    x[:beams] = -np.inf
    x[beams, :3] = 1.0, 2.0, 3.0
    x[beams:2 * beams, 3:] = -np.inf
    x[beams + 1:2 * beams] = -np.inf
    scores = rng.normal(-9.0, 1.0, rows).astype(np.float32)
    out = [torch.zeros((requests, beams), dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    ws = torch.empty(S.sfmp_beam_select_workspace(requests, beams, vocab, beams), dtype=torch.uint8, device=DEV)
    S.sfmp_beam_select(up(x), beams, up(scores), None, None, 0, *out, ws)
    slots, parents, each = torch.arange(rows, dtype=torch.int32, device=DEV), out[1].flatten(), 1000 // beams * beams
    for first in range(0, rows, each):
        part = slice(first, min(first + each, rows))
        S.sfmp_kv_reorder(cache, dt, slots[part], parents[part] - first)
    expected = np.full((requests, beams), -1)
    for r in range(requests):
        want, _, _ = O.beam_select(x[r * beams:(r + 1) * beams], scores[r * beams:(r + 1) * beams], beams)
        expected[r, :len(want)] = [b + r * beams for _, b, _ in want]
    assert (expected[0] == -1).all() and (expected[1] == [beams] * 3 + [-1] * 2).all()
    assert np.array_equal(parents.cpu().numpy(), expected.flatten())
    for r in range(requests):
        O.reorder(tables, list(range(r * beams, (r + 1) * beams)), [p - r * beams if p >= 0 else -1 for p in expected[r]])
    assert np.array_equal(dt.lengths.cpu().numpy(), tables["lengths"]) and np.array_equal(dt.refs.cpu().numpy(), tables["refs"])
    assert np.array_equal(dt.page_table.cpu().numpy(), tables["table"])
