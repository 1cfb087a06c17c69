"""Cache and sampling calls, host side (no GPU): struct sizes, sizes, and every refusal of the library and of the binding."""
import ctypes as C
import math

import pytest

import paper_2602_01027_amd as S
from paper_2602_01027_amd.binding import SfmpKvBatch, SfmpKvTables

NULL, SHAPE, WORKSPACE, LAYOUT, ALIGN = -1, -2, -5, -8, -9
P = 1 << 20  # an address that no check follows


def test_struct_sizes():
    assert C.sizeof(S.SfmpKvLayout) == 48 and C.sizeof(SfmpKvTables) == 32 and C.sizeof(SfmpKvBatch) == 32


def test_query():
    L = S.sfmp_kv_query(10, 8, 128, "fp8", 3)
    assert (L.pages, L.kv_heads, L.head_dim, L.format, L.layers, L.reserved) == (10, 8, 128, 1, 3, 0)
    assert L.page_bytes == 8 * 2 * 64 * 128 and L.codes_bytes == 30 * L.page_bytes and L.scales_bytes == 30 * 8 * 2 * 4
    big = S.sfmp_kv_query(2 ** 31 - 1, 1024, 256, "int8", 1)
    assert big.codes_bytes == (2 ** 31 - 1) * 1024 * 2 * 64 * 256


@pytest.mark.parametrize("args,code", [((0, 8, 128, 0, 1), SHAPE), ((1, 0, 128, 0, 1), SHAPE), ((1, 1025, 128, 0, 1), SHAPE),
                                       ((1, 8, 96, 0, 1), SHAPE), ((1, 8, 128, 0, 0), SHAPE), ((1, 8, 128, 2, 1), LAYOUT),
                                       ((2 ** 31 - 1, 1024, 256, 0, 2 ** 31 - 1), SHAPE)])
def test_query_refuses(args, code):
    with pytest.raises(S.SfmpError) as e:
        S.sfmp_kv_query(*args)
    assert e.value.code == code


def call(name, **change):
    """Status of a call with valid-looking arguments, some of them changed.  (Nothing is launched where a check refuses; a call
    that none refuses ends at the missing device.)"""
    lib = S.load_library()
    L = S.sfmp_kv_query(16, 4, 128, "int8", 2)
    for k in ("pages", "kv_heads", "head_dim", "format", "page_bytes", "scales_bytes"):
        if k in change:
            setattr(L, k, change.pop(k))
    t = SfmpKvTables(P, P, P, 5, 9)
    b = SfmpKvBatch(P, P, 3, 6, 4, 0)
    for obj, names in ((t, ("page_table", "lengths", "refs", "sequences", "table_pages")),
                       (b, ("slots", "row_start", "batch", "rows", "max_rows"))):
        for k in names:
            if k in change:
                setattr(obj, k, change.pop(k))
    a = dict(layer=1, codes=P, scales=P, K=P, V=P, first=P, dtype=0, k_stride=512, v_stride=512, Q=P, O=P, lse=P, q_heads=8,
             q_stride=1024, o_stride=1024, max_tokens=300, window=0, scale=0.1, workspace=P, bytes=1 << 40, index=P, other=P, n=3,
             status=P, logits=P, type=0, count=4, vocab=1000, stride=1000, temperature=P, top_k=P, top_p=P, min_p=P, uniform=P,
             tokens=P, logprobs=P)
    layout, tables, batch = C.byref(L), C.byref(t), C.byref(b)
    if change.pop("no_layout", False):
        layout = None
    if change.pop("no_tables", False):
        tables = None
    if change.pop("no_batch", False):
        batch = None
    assert set(change) <= set(a), change
    a.update(change)
    rows = (layout, a["layer"], a["codes"], a["scales"], tables, batch)
    args = {
        "append": (*rows, a["K"], a["V"], a["dtype"], a["k_stride"], a["v_stride"]),
        "gather": (*rows, a["first"], a["K"], a["V"], a["dtype"], a["k_stride"], a["v_stride"]),
        "attention": (*rows, a["Q"], a["q_heads"], a["dtype"], a["q_stride"], a["max_tokens"], a["window"], a["scale"], a["O"],
                      a["o_stride"], a["lse"], a["workspace"], a["bytes"]),
        "reserve": (layout, a["codes"], a["scales"], tables, a["index"], a["other"], a["n"], a["status"], a["workspace"], a["bytes"]),
        "fork": (layout, tables, a["index"], a["other"], a["n"]),
        "free": (layout, tables, a["index"], a["other"], a["n"]),
        "compact": (layout, a["codes"], a["scales"], tables, a["status"], a["workspace"], a["bytes"]),
        "sample": (a["logits"], a["type"], a["count"], a["vocab"], a["stride"], a["temperature"], a["top_k"], a["top_p"], a["min_p"],
                   a["uniform"], a["tokens"], a["logprobs"], a["workspace"], a["bytes"]),
    }[name]
    return getattr(lib, "sfmp_" + name if name == "sample" else "sfmp_kv_" + name)(*args, None)


ROWS = [(dict(no_layout=True), NULL), (dict(no_tables=True), NULL), (dict(no_batch=True), NULL), (dict(codes=None), NULL),
        (dict(scales=None), NULL), (dict(page_table=None), NULL), (dict(lengths=None), NULL), (dict(layer=2), SHAPE),
        (dict(layer=-1), SHAPE), (dict(codes=P + 8), ALIGN), (dict(scales=P + 4), ALIGN), (dict(lengths=P + 2), ALIGN),
        (dict(slots=P + 1), ALIGN), (dict(row_start=P + 2), ALIGN), (dict(sequences=0), SHAPE), (dict(table_pages=0), SHAPE),
        (dict(table_pages=2 ** 20 + 1), SHAPE), (dict(batch=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(max_rows=7), SHAPE),
        (dict(rows=2 ** 30 + 1), SHAPE), (dict(row_start=None), SHAPE), (dict(slots=None, batch=6), SHAPE), (dict(page_bytes=1), LAYOUT),
        (dict(scales_bytes=1), LAYOUT), (dict(head_dim=32), SHAPE), (dict(format=5), LAYOUT), (dict(dtype=7), LAYOUT)]
WRITE = [(dict(K=None), NULL), (dict(V=None), NULL), (dict(K=P + 2), ALIGN), (dict(V=P + 8), ALIGN), (dict(k_stride=511), SHAPE),
         (dict(k_stride=516), SHAPE), (dict(v_stride=504), SHAPE)]
REFUSED = {
    "append": ROWS + WRITE + [(dict(dtype=2), LAYOUT)],
    "gather": ROWS + WRITE + [(dict(first=None), NULL), (dict(first=P + 2), ALIGN)],
    "attention": ROWS + [(dict(Q=None), NULL), (dict(O=None), NULL), (dict(Q=P + 8), ALIGN), (dict(O=P + 2), ALIGN), (dict(lse=P + 2), ALIGN),
                         (dict(q_heads=6), SHAPE), (dict(q_heads=0), SHAPE), (dict(q_stride=1016), SHAPE), (dict(o_stride=1028), SHAPE),
                         (dict(max_tokens=0), SHAPE), (dict(window=-1), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=-1.0), SHAPE),
                         (dict(scale=math.nan), SHAPE), (dict(scale=math.inf), SHAPE), (dict(workspace=None), WORKSPACE),
                         (dict(workspace=P + 16), WORKSPACE), (dict(bytes=0), WORKSPACE), (dict(dtype=2), LAYOUT),
                         (dict(max_tokens=64 * 2 ** 20, max_rows=2 ** 20, rows=2 ** 20), SHAPE)],
    "reserve": [(dict(no_layout=True), NULL), (dict(no_tables=True), NULL), (dict(refs=None), NULL), (dict(refs=P + 2), ALIGN),
                (dict(codes=None), NULL), (dict(index=None), NULL), (dict(index=P + 2), ALIGN), (dict(other=P + 1), ALIGN),
                (dict(status=None), NULL), (dict(status=P + 2), ALIGN), (dict(n=-1), SHAPE), (dict(n=1025), SHAPE),
                (dict(workspace=None), WORKSPACE), (dict(workspace=P + 64), WORKSPACE), (dict(bytes=64), WORKSPACE)],
    "fork": [(dict(no_layout=True), NULL), (dict(refs=None), NULL), (dict(index=None), NULL), (dict(other=None), NULL),
             (dict(other=P + 2), ALIGN), (dict(n=-1), SHAPE)],
    "free": [(dict(no_tables=True), NULL), (dict(refs=None), NULL), (dict(index=None), NULL), (dict(index=P + 3), ALIGN), (dict(n=-5), SHAPE)],
    "compact": [(dict(no_layout=True), NULL), (dict(scales=None), NULL), (dict(status=None), NULL), (dict(refs=None), NULL),
                (dict(status=P + 1), ALIGN), (dict(bytes=8), WORKSPACE)],
    "sample": [(dict(logits=None), NULL), (dict(uniform=None), NULL), (dict(tokens=None), NULL), (dict(type=3), LAYOUT),
               (dict(vocab=0), SHAPE), (dict(vocab=2 ** 24 + 1, stride=2 ** 25), SHAPE), (dict(stride=999), SHAPE), (dict(count=-1), SHAPE),
               (dict(count=65536), SHAPE), (dict(logits=P + 1), ALIGN), (dict(logits=P + 2, type=2), ALIGN), (dict(uniform=P + 2), ALIGN),
               (dict(top_k=P + 2), ALIGN), (dict(tokens=P + 2), ALIGN), (dict(workspace=None), WORKSPACE), (dict(bytes=0), WORKSPACE)],
}


@pytest.mark.parametrize("name,change,code", [(n, c, k) for n, cases in REFUSED.items() for c, k in cases])
def test_library_refuses(name, change, code):
    assert call(name, **change) == code


@pytest.mark.parametrize("name,change", [("append", dict(rows=0, max_rows=0, K=None, V=None)), ("gather", dict(batch=0, rows=0, max_rows=0)),
                                         ("attention", dict(batch=0, rows=0, max_rows=0, Q=None, O=None)), ("fork", dict(n=0)), ("free", dict(n=0)),
                                         ("sample", dict(count=0, logits=None))])
def test_calls_with_nothing_to_do(name, change):
    assert call(name, **change) == 0


def test_binding_refuses_what_is_no_gpu_tensor_of_the_right_kind():
    import torch
    layout = S.sfmp_kv_query(4, 2, 64)
    cache, tables = S.make_kv_cache(layout, "cpu"), S.make_kv_tables(layout, 2, 3, "cpu")
    x = torch.zeros((1, 2, 64), dtype=torch.float16)
    i = torch.zeros(1, dtype=torch.int32)
    w = torch.zeros(1024, dtype=torch.uint8)
    for f in (lambda: S.sfmp_kv_append(cache, 0, tables, None, None, x, x, 1),
              lambda: S.sfmp_kv_gather(cache, 0, tables, None, i, None, x, x, 1),
              lambda: S.sfmp_kv_attention(cache, 0, tables, None, None, x, x, 1, 64, 1.0, w),
              lambda: S.sfmp_kv_reserve(cache, tables, i, None, i, w), lambda: S.sfmp_kv_fork(cache, tables, i, i),
              lambda: S.sfmp_kv_free(cache, tables, i), lambda: S.sfmp_kv_compact(cache, tables, i, w),
              lambda: S.sfmp_sample(torch.zeros((1, 9)), None, None, None, None, i, i, None, w)):
        with pytest.raises(ValueError, match="on the GPU"):
            f()
