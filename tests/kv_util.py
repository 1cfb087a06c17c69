"""Helpers of the cache and sampling tests: pools and tables on both sides, and bounds derived from the kernels' arithmetic."""
import numpy as np

PAGE = 64
U16, UB16, U32 = 2.0 ** -11, 2.0 ** -8, 2.0 ** -24  # unit roundoffs of fp16, bf16, fp32


def pages_of(tokens):
    return -(-tokens // PAGE)


def random_codes(rng, shape, fmt):
    """Any byte that stands for a number (for fp8 not the two patterns that do not)."""
    codes = rng.integers(1 if fmt == "int8" else 0, 256, size=shape, dtype=np.uint8)
    if fmt == "fp8":
        codes[(codes & 0x7F) == 0x7F] = 0x70
    return codes


def make_pool(rng, layers, pages, heads, dim, fmt):
    codes = random_codes(rng, (layers, pages, heads, 2, PAGE * dim), fmt)
    spread = np.exp(rng.normal(0.0, 0.7, size=codes.shape[:4]))
    scales = spread / 64.0 if fmt == "int8" else 2.0 ** np.rint(np.log2(spread) - 7)
    return dict(codes=codes, scales=scales.astype(np.float32).astype(np.float64))


def make_tables(rng, lengths, table_pages, pages, spare=0):
    """Sequences of these lengths in pages taken at random."""
    table = np.full((len(lengths) + spare, table_pages), -1, dtype=np.int32)
    refs = np.zeros(pages, dtype=np.int32)
    free = rng.permutation(pages)
    at = 0
    for s, n in enumerate(lengths):
        k = pages_of(n)
        table[s, :k] = free[at:at + k]
        at += k
    refs[free[:at]] = 1
    return dict(table=table, lengths=np.array(list(lengths) + [0] * spare, dtype=np.int32), refs=refs)


def stale_slots(pool, tables, fmt, dim):
    """What no sequence has written holds the worst there is: for fp8 the pattern that stands for no number."""
    bad = 0x7F if fmt == "fp8" else 0xFF
    for s, n in enumerate(tables["lengths"]):
        if n % PAGE:
            page = pool["codes"][:, tables["table"][s, n // PAGE]]
            page[:, :, 0].reshape(*page.shape[:2], PAGE, dim)[:, :, n % PAGE:] = bad
            page[:, :, 1].reshape(*page.shape[:2], dim, PAGE)[:, :, :, n % PAGE:] = bad
            pool["codes"][:, tables["table"][s, n // PAGE]] = page


def upload(S, pool, tables, fmt, device="cuda:0"):
    import torch
    layers, pages, heads, _, block = pool["codes"].shape
    layout = S.sfmp_kv_query(pages, heads, block // PAGE, fmt, layers)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)  # noqa: E731
    cache = S.DeviceKvCache(layout, up(pool["codes"]), up(pool["scales"].astype(np.float32)))
    return cache, S.DeviceKvTables(up(tables["table"]), up(tables["lengths"]), up(tables["refs"]))


def attention_bound(out_unit, O, spread, products):
    """Elementwise bound of |O - O of the oracle|.

    Weights: each is rounded to fp16 (U16 of itself, or 2^-25 in units of 2^-14 of the largest weight where it is a denormal), and
    carries the error of its score: a sum of fp32 products, below (dim + 8) U32 <= 2^-15.9 of the sum of magnitudes
    `products`, plus the exponential's few U32.  The same relative error enters the sum of weights.  Then the result's own
    rounding."""
    score = 2.0 ** -15 * products[..., None] + 2.0 ** -20
    return spread * (2.0 * np.expm1(score) + U16 + 2.0 ** -20) + out_unit * np.abs(O) * 1.01 + 2.0 ** -24


def lse_bound(lse, products):
    return 2.0 ** -15 * products + 2.0 ** -20 + 2.0 ** -21 * np.abs(lse)
