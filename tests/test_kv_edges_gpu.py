"""The cache and sampling calls on the GPU where sizes and arguments end."""
import numpy as np
import pytest

from kv_util import U16, UB16, attention_bound, make_pool, make_tables, upload
from oracle import sfmp_kv_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _torch():
    import torch
    assert torch.cuda.is_available()
    import paper_2602_01027_amd as S
    return torch, S


def test_workspaces_that_are_not_contiguous_gpu_memory_are_refused():
    torch, S = _torch()
    layout = S.sfmp_kv_query(4, 2, 64)
    cache, tables = S.make_kv_cache(layout), S.make_kv_tables(layout, 2, 3)
    x = torch.zeros((2, 2, 64), dtype=torch.float16, device=DEV)
    i, f = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV)
    calls = (lambda w: S.sfmp_kv_attention(cache, 0, tables, i, None, x, x.clone(), 1, 64, 1.0, w),
             lambda w: S.sfmp_kv_reserve(cache, tables, i[:0], None, i[:1], w), lambda w: S.sfmp_kv_compact(cache, tables, i[:1], w),
             lambda w: S.sfmp_sample(torch.zeros((2, 9), device=DEV), None, None, None, None, f, i, f.clone(), w))
    host = torch.zeros((1 << 16) + 256, dtype=torch.uint8)
    host = host[-host.data_ptr() % 256:][:1 << 16]  # (on an address that the library would take)
    for call in calls:
        call(torch.zeros(1 << 16, dtype=torch.uint8, device=DEV))
        for bad in (host, torch.zeros(1, dtype=torch.uint8, device=DEV).expand(1 << 16)):
            with pytest.raises(ValueError, match="workspace has to be"):
                call(bad)
    torch.cuda.synchronize()


def test_one_workspace_for_a_batch_that_shrinks():
    # made for the largest step of a program (whose form needs none), used by the smaller ones (whose forms cut the work into parts)
    torch, S = _torch()
    rng = np.random.default_rng(12)
    n, dim, heads, group, tokens = 520, 64, 2, 2, 9000
    lengths = rng.integers(1, 130, n)
    lengths[0] = 1000
    pool = make_pool(rng, 1, int((-(-lengths // 64)).sum()), heads, dim, "int8")
    tables = make_tables(rng, lengths, 16, pool["codes"].shape[1])
    cache, dt = upload(S, pool, tables, "int8")
    most = 40  # rows of an entry
    size = S.sfmp_kv_attention_workspace(cache.layout, n, n * most, heads * group, most, tokens)
    canary = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    for batch, rows in ((n, 1), (512, 1), (100, 1), (3, 1), (1, 1), (3, 8), (2, most), (100, 12), (n, 3), (300, most)):
        start = (np.arange(batch + 1) * rows).astype(np.int32)
        q = rng.normal(size=(batch * rows, heads * group, dim)).astype(np.float16)
        Q, got = torch.from_numpy(q).to(DEV), torch.full((batch * rows, heads * group, dim), float("nan"), dtype=torch.float16, device=DEV)
        S.sfmp_kv_attention(cache, 0, dt, None if batch == n else torch.arange(batch, dtype=torch.int32, device=DEV), torch.from_numpy(start).to(DEV),
                            Q, got, rows, tokens, 0.125, canary[:size])
        a = got.float().cpu().numpy()
        for b in sorted({0, batch - 1, batch // 2}):
            k, v = O.dense(pool, 0, tables, b, "int8", dim)
            r = slice(b * rows, (b + 1) * rows)
            want, _, spread, products = O.attention(q[r].astype(np.float64), k, v, 0.125)
            assert (np.abs(a[r] - want) <= attention_bound(U16, want, spread, products)).all(), (batch, rows, b)
    assert (canary[size:] == 0x5A).all()
    # likewise rows of logits
    rows, vocab = 130, 140000
    size = S.sfmp_sample_workspace(rows, vocab)
    canary = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    logits = torch.from_numpy(rng.normal(0.0, 3.0, size=(rows, vocab)).astype(np.float32)).to(DEV)
    u = torch.from_numpy(rng.random(rows).astype(np.float32)).to(DEV)
    tokens = torch.empty(rows, dtype=torch.int32, device=DEV)
    S.sfmp_sample(logits, None, None, None, None, u, tokens, None, canary[:size])
    for n in (109, 80, 79, 64, 33, 1):
        few = torch.empty(n, dtype=torch.int32, device=DEV)
        S.sfmp_sample(logits[:n], None, None, None, None, u[:n], few, None, canary[:size])
        assert torch.equal(few, tokens[:n])
    assert (canary[size:] == 0x5A).all()


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 100, 64 * 2 ** 20])
@pytest.mark.parametrize("entries,max_tokens", [([(8, 3), (2, 2), (30, 20)], None), ([(8, 3), (1, 700), (3, 0)], 20000), ([(300, 40), (200, 190)], None),
                                                ([(70, 20), (200, 190)], 9000)])
def test_windows_that_reach_past_every_sequence(entries, max_tokens, window):
    # rows that stand before the first token, and a window whose end lies 2^31 before the others: the same bits as without a window
    torch, S = _torch()
    rng = np.random.default_rng(21)
    heads, group, dim = 2, 2, 128
    lengths, counts = [t for _, t in entries], [n for n, _ in entries]
    tokens = max_tokens or max(lengths)
    pages = sum(-(-t // 64) for t in lengths)
    cache, dt = upload(S, make_pool(rng, 1, pages, heads, dim, "int8"), make_tables(rng, lengths, -(-max(lengths) // 64), pages), "int8")
    start = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(DEV)
    q = torch.from_numpy(rng.normal(size=(sum(counts), heads * group, dim)).astype(np.float16)).to(DEV)
    ws = torch.empty(S.sfmp_kv_attention_workspace(cache.layout, len(entries), sum(counts), heads * group, max(counts), tokens), dtype=torch.uint8,
                     device=DEV)
    results = []
    for w in (0, window):
        out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device=DEV)
        S.sfmp_kv_attention(cache, 0, dt, None, start, q, out, max(counts), tokens, 0.09, ws, window=w, lse=lse)
        results.append((out, lse))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    assert not torch.isneginf(results[0][1][-1]).any() or lengths[-1] == 0


def test_numbers_of_a_call_that_do_not_fit_32_bits_are_refused():
    torch, S = _torch()
    layout = S.sfmp_kv_query(4, 2, 64)
    cache, tables = S.make_kv_cache(layout), S.make_kv_tables(layout, 2, 3)
    x = torch.zeros((2, 2, 64), dtype=torch.float16, device=DEV)
    i, w = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)
    for past in (2 ** 32, 2 ** 32 + 1, -2 ** 32):
        for layer, max_rows, tokens, window in ((past, 1, 64, 0), (0, past, 64, 0), (0, 1, past, 0), (0, 1, 64, past)):
            with pytest.raises(ValueError, match="fit 32 bits"):
                S.sfmp_kv_attention(cache, layer, tables, i, None, x, x.clone(), max_rows, tokens, 1.0, w, window=window)
        for layer, max_rows in ((past, 1), (0, past)):
            with pytest.raises(ValueError, match="fit 32 bits"):
                S.sfmp_kv_append(cache, layer, tables, i, None, x, x, max_rows)
            with pytest.raises(ValueError, match="fit 32 bits"):
                S.sfmp_kv_gather(cache, layer, tables, i, i, None, x, x.clone(), max_rows)


def test_calls_on_pages_refuse_what_is_no_vector():
    torch, S = _torch()
    layout = S.sfmp_kv_query(4, 2, 64)
    cache, tables = S.make_kv_cache(layout), S.make_kv_tables(layout, 2, 3)
    i, w = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)
    for bad in (None, [0], 0, i[0], i[None]):
        for call in (lambda: S.sfmp_kv_reserve(cache, tables, bad, None, i, w), lambda: S.sfmp_kv_fork(cache, tables, bad, i),
                     lambda: S.sfmp_kv_free(cache, tables, bad)):
            with pytest.raises(ValueError, match="has to be a vector"):
                call()


def _weights_floor(q, k, v, scale):
    """What weights held in units of 2^-38 of their page's largest add to a result: 2^-39 of that largest weight for every token of the
    page, times the token's value."""
    n, heads, dim = q.shape
    t, group = k.shape[0], heads // k.shape[1]
    out = np.zeros((n, heads, dim))
    for i in range(n):
        p = t - n + i
        for h in range(heads):
            z = scale * (k[:p + 1, h // group] @ q[i, h].astype(np.float64))
            w = np.exp(z - z.max())
            for page in range(0, p + 1, 64):
                part = slice(page, min(page + 64, p + 1))
                out[i, h] += 2.0 ** -39 * w[part].max() / w.sum() * np.abs(v[part, h // group]).sum(0)
    return out


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("entries,max_tokens", [([(1, 500), (1, 1000), (1, 130)], 1000), ([(1, 500), (1, 1000), (1, 130)], 40000),
                                                ([(40, 300), (33, 97), (70, 200)], 2000), ([(40, 300), (33, 97), (70, 200)], 9000)])
@pytest.mark.parametrize("powers", [[60], [12, 30], [-30, 0, 60, 90]])
def test_attention_over_values_of_great_magnitude(fmt, entries, max_tokens, powers):
    # the least weights' rounding in proportion to the values that they multiply, where an absolute term does not cover it
    torch, S = _torch()
    rng = np.random.default_rng(len(powers) + max_tokens)
    heads, group, dim = 2, 2, 128
    lengths, counts = [t for _, t in entries], [n for n, _ in entries]
    pages = sum(-(-t // 64) for t in lengths)
    pool, tables = make_pool(rng, 1, pages, heads, dim, fmt), make_tables(rng, lengths, -(-max(lengths) // 64), pages)
    pool["scales"][..., 1] = 2.0 ** rng.choice(powers, size=pool["scales"].shape[:3])
    cache, dt = upload(S, pool, tables, fmt)
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    Q = torch.from_numpy(rng.normal(0.0, 4.0, size=(sum(counts), heads * group, dim)).astype(np.float32)).bfloat16().to(DEV)
    q, out = Q.float().cpu().numpy(), torch.full_like(Q, float("nan"))
    ws = torch.empty(S.sfmp_kv_attention_workspace(cache.layout, len(entries), sum(counts), heads * group, max(counts), max_tokens), dtype=torch.uint8,
                     device=DEV)
    S.sfmp_kv_attention(cache, 0, dt, None, torch.from_numpy(start).to(DEV), Q, out, max(counts), max_tokens, 0.09, ws)
    got = out.float().cpu().numpy().astype(np.float64)
    for b in range(len(entries)):
        k, v = O.dense(pool, 0, tables, b, fmt, dim)
        r = slice(start[b], start[b + 1])
        want, _, spread, products = O.attention(q[r], k, v, 0.09)
        bound = attention_bound(UB16, want, spread, products) + _weights_floor(q[r], k, v, 0.09)
        assert (np.abs(got[r] - want) <= bound).all(), (b, (np.abs(got[r] - want) / bound).max())
