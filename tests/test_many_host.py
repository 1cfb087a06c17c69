"""Attention over shared pages and first tokens, beam selection and reordering, host side (no GPU): every refusal of the library and of the
binding, sizes of plans and workspaces."""
import ctypes as C
import math
import random

import numpy as np
import pytest

from oracle import sfmp_kv_oracle as O
import paper_2602_01027_amd as S
from paper_2602_01027_amd.binding import SfmpKvBatch, SfmpKvTables

NULL, SHAPE, WORKSPACE, HIP, LAYOUT, ALIGN = -1, -2, -5, -6, -8, -9
P = 1 << 20  # an address that no check follows


def call(name, **change):
    """Status of a call with valid-looking arguments, some of them changed.  (Nothing is launched where a check refuses; a call
    that none refuses ends at the missing device.)"""
    lib = S.load_library()
    L = change.pop("L", None) or S.sfmp_kv_query(16, 4, 128, "int8", 2)
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
    a = dict(layer=1, codes=P, scales=P, dtype=0, Q=P, O=P, lse=P, q_heads=8, q_stride=1024, o_stride=1024, max_tokens=300, window=70, sinks=4,
             scale=0.1, workspace=P, bytes=1 << 40, plan=P, plan_bytes=1 << 40, group_start=P, groups=2, prefix=P, index=P, other=P, n=3,
             logits=P, type=0, requests=2, beams=3, vocab=1000, stride=1000, scores=P, weights=P, ended=P, end_token=2, choices=6, next_scores=P,
             parents=P, tokens=P)
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
    end = (a["scale"], a["O"], a["o_stride"], a["lse"])
    args = {
        "kv_attention_sinks": (*rows, a["Q"], a["q_heads"], a["dtype"], a["q_stride"], a["max_tokens"], a["window"], a["sinks"], *end, a["workspace"],
                               a["bytes"]),
        "kv_share": (layout, tables, batch, a["group_start"], a["groups"], a["q_heads"], a["max_tokens"], a["window"], a["sinks"], a["prefix"], a["plan"],
                     a["plan_bytes"]),
        "kv_attention_shared": (*rows, a["group_start"], a["groups"], a["Q"], a["q_heads"], a["dtype"], a["q_stride"], a["max_tokens"], a["window"],
                                a["sinks"], *end, a["plan"], a["plan_bytes"], a["workspace"], a["bytes"]),
        "kv_reorder": (layout, tables, a["index"], a["other"], a["n"]),
        "beam_select": (a["logits"], a["type"], a["requests"], a["beams"], a["vocab"], a["stride"], a["scores"], a["weights"], a["ended"],
                        a["end_token"], a["choices"], a["next_scores"], a["parents"], a["tokens"], a["workspace"], a["bytes"]),
    }[name]
    return getattr(lib, "sfmp_" + name)(*args, None)


TABLES = [(dict(no_layout=True), NULL), (dict(no_tables=True), NULL), (dict(page_table=None), NULL), (dict(lengths=None), NULL),
          (dict(lengths=P + 2), ALIGN), (dict(sequences=0), SHAPE), (dict(table_pages=0), SHAPE), (dict(table_pages=2 ** 20 + 1), SHAPE),
          (dict(page_bytes=1), LAYOUT), (dict(scales_bytes=1), LAYOUT), (dict(head_dim=32), SHAPE), (dict(format=5), LAYOUT)]
BATCH = TABLES + [(dict(no_batch=True), NULL), (dict(slots=P + 1), ALIGN), (dict(row_start=P + 2), ALIGN), (dict(batch=-1), SHAPE), (dict(rows=-1), SHAPE),
                  (dict(max_rows=7), SHAPE), (dict(rows=2 ** 30 + 1), SHAPE), (dict(row_start=None), SHAPE), (dict(slots=None, batch=6), SHAPE),
                  (dict(q_heads=6), SHAPE), (dict(q_heads=0), SHAPE), (dict(max_tokens=0), SHAPE), (dict(max_tokens=2 ** 26 + 1), SHAPE),
                  (dict(window=-1), SHAPE), (dict(sinks=-1), SHAPE), (dict(window=0, sinks=-1), SHAPE)]
ATTENTION = BATCH + [(dict(codes=None), NULL), (dict(scales=None), NULL), (dict(layer=2), SHAPE), (dict(layer=-1), SHAPE), (dict(codes=P + 8), ALIGN),
                     (dict(scales=P + 4), ALIGN), (dict(Q=None), NULL), (dict(O=None), NULL), (dict(Q=P + 8), ALIGN), (dict(O=P + 2), ALIGN),
                     (dict(lse=P + 2), ALIGN), (dict(q_stride=1016), SHAPE), (dict(o_stride=1028), SHAPE), (dict(scale=0.0), SHAPE),
                     (dict(scale=math.nan), SHAPE), (dict(scale=math.inf), SHAPE), (dict(dtype=2), LAYOUT), (dict(workspace=None), WORKSPACE),
                     (dict(workspace=P + 16), WORKSPACE), (dict(bytes=0), WORKSPACE)]
GROUPS = [(dict(groups=-1), SHAPE), (dict(groups=65536), SHAPE), (dict(group_start=None), NULL), (dict(group_start=P + 2), ALIGN), (dict(plan=None), WORKSPACE),
          (dict(plan=P + 128), WORKSPACE), (dict(plan_bytes=0), WORKSPACE)]
LARGE = dict(max_tokens=60000, table_pages=1000)  # (a call that is worth a plan)
REFUSED = {
    "kv_attention_sinks": ATTENTION,
    "kv_share": BATCH + GROUPS + [(dict(prefix=P + 1), ALIGN), (dict(plan_bytes=1024, window=0, **LARGE), WORKSPACE)],
    "kv_attention_shared": ATTENTION + GROUPS + [({**LARGE, "window": 0, **c}, k) for c, k in ATTENTION[-20:]] + [(dict(plan_bytes=1024, window=0, **LARGE),
                                                                                                                   WORKSPACE)],
    "kv_reorder": TABLES + [(dict(refs=None), NULL), (dict(refs=P + 2), ALIGN), (dict(index=None), NULL), (dict(other=None), NULL), (dict(index=P + 1), ALIGN),
                            (dict(other=P + 2), ALIGN), (dict(n=-1), SHAPE), (dict(n=1025), SHAPE)],
    "beam_select": [(dict(logits=None), NULL), (dict(scores=None), NULL), (dict(next_scores=None), NULL), (dict(parents=None), NULL), (dict(tokens=None), NULL),
                    (dict(type=3), LAYOUT), (dict(type=-1), LAYOUT), (dict(requests=-1), SHAPE), (dict(beams=0), SHAPE), (dict(beams=33), SHAPE),
                    (dict(requests=65536, beams=1), SHAPE), (dict(requests=2 ** 31 - 1, beams=32), SHAPE), (dict(choices=0), SHAPE), (dict(choices=65), SHAPE),
                    (dict(vocab=0), SHAPE), (dict(vocab=2 ** 24 + 1, stride=2 ** 25), SHAPE), (dict(stride=999), SHAPE), (dict(stride=2 ** 62), SHAPE),
                    (dict(end_token=-1), SHAPE), (dict(end_token=1000), SHAPE), (dict(logits=P + 1), ALIGN), (dict(logits=P + 2, type=2), ALIGN),
                    (dict(scores=P + 2), ALIGN), (dict(weights=P + 1), ALIGN), (dict(ended=P + 2), ALIGN), (dict(next_scores=P + 2), ALIGN),
                    (dict(parents=P + 2), ALIGN), (dict(tokens=P + 3), ALIGN), (dict(workspace=None), WORKSPACE), (dict(workspace=P + 16), WORKSPACE),
                    (dict(bytes=100), WORKSPACE)],
}


@pytest.mark.parametrize("name,change,code", [(n, c, k) for n, cases in REFUSED.items() for c, k in cases])
def test_library_refuses(name, change, code):
    assert call(name, **change) == code


@pytest.mark.parametrize("name,change", [("kv_attention_sinks", dict(batch=0, rows=0, max_rows=0, Q=None, O=None)), ("kv_reorder", dict(n=0)),
                                         ("kv_share", dict(groups=0, group_start=None)), ("kv_share", dict(prefix=None)),
                                         ("kv_attention_shared", dict(batch=0, rows=0, max_rows=0, Q=None, O=None)),
                                         ("beam_select", dict(requests=0, logits=None, scores=None))])
def test_nothing_to_do(name, change):
    assert call(name, **change) == 0


def test_queries_refuse():
    L = S.sfmp_kv_query(16, 8, 128)
    for ask in (S.sfmp_kv_share_plan, S.sfmp_kv_attention_shared_workspace):
        assert ask(L, 0, 0, 0, 8, 0, 64) >= 256
        for bad in ((-1, 1, 1, 8, 1, 64), (65536, 65536, 1, 8, 1, 64), (2, 2, -1, 8, 1, 64), (2, 2, 65536, 8, 1, 64), (2, 2, 1, 12, 1, 64),
                    (2, 2, 1, 8, 3, 64), (2, 2, 1, 8, 1, 0)):
            with pytest.raises(S.SfmpError) as e:
                ask(L, *bad)
            assert e.value.code == SHAPE
    for bad in ((-1, 1, 10, 1), (1, 33, 10, 1), (1, 0, 10, 1), (1, 1, 0, 1), (1, 1, 2 ** 24 + 1, 1), (1, 1, 10, 0), (1, 1, 10, 65), (65536, 1, 10, 1)):
        with pytest.raises(S.SfmpError) as e:
            S.sfmp_beam_select_workspace(*bad)
        assert e.value.code == SHAPE
    for k in range(4):
        with pytest.raises(ValueError, match="fit 32 bits"):
            S.sfmp_beam_select_workspace(*[2 ** 32 + 1 if i == k else 1 for i in range(4)])
    for k in range(6):
        with pytest.raises(ValueError, match="fit 32 bits"):
            S.sfmp_kv_share_plan(L, *[2 ** 31 if i == k else 8 for i in range(6)])


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_plans_and_workspaces_are_enough_for_smaller_calls(dim):
    """Of a call whose plan or workspace is too small nothing is launched; one whose is not ends at the missing device, or at an
    address that is none."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("launches what no check refuses")
    rng = random.Random(dim)
    log = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))  # noqa: E731
    shared = 0
    for _ in range(1500):
        heads, group = rng.choice((1, 2, 8, 16)), rng.choice((1, 2, 4, 5, 8, 16, 40))
        L = S.sfmp_kv_query(16, heads, dim)
        batch, rows, groups, tokens = log(2, 400), log(1, 90), log(1, 90), log(64, 60000)
        small = [log(1, batch), log(1, rows), log(1, groups), log(1, tokens)]
        sizes = (L, batch, batch * rows, groups, heads * group, rows, tokens)
        plan, space = S.sfmp_kv_share_plan(*sizes), S.sfmp_kv_attention_shared_workspace(*sizes)
        for b, r, g, t in ((batch, rows, groups, tokens), small):
            width = heads * group * dim
            args = dict(L=L, layer=0, sequences=1000, table_pages=1000, batch=b, rows=b * r, max_rows=r, groups=g, q_heads=heads * group, q_stride=width,
                        o_stride=width, max_tokens=t, plan_bytes=plan, bytes=space)
            for window in (0, 500):
                assert call("kv_share", window=window, **args) in (0, HIP)
                assert call("kv_attention_shared", window=window, **args) in (0, HIP)
                shared += call("kv_attention_shared", window=window, **{**args, "plan_bytes": 256}) == WORKSPACE
    assert shared > 100


def test_workspaces_of_beam_selection_are_enough_for_smaller_calls():
    import torch
    if torch.cuda.is_available():
        pytest.skip("launches what no check refuses")
    rng = random.Random(1)
    log = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))  # noqa: E731
    for _ in range(3000):
        big = [log(1, 2000), log(1, 32), log(1, 2 ** 24), log(1, 64)]
        space = S.sfmp_beam_select_workspace(*big)
        for r, b, v, c in (big, [log(1, n) for n in big]):
            for dtype in (0, 1, 2):
                assert call("beam_select", requests=r, beams=b, vocab=v, stride=v, choices=c, type=dtype, end_token=0, bytes=space) in (0, HIP)


def test_the_binding_refuses_tensors_of_other_kinds():
    import torch
    cpu = torch.zeros((4, 8))
    with pytest.raises(ValueError, match="logits has to be a tensor on the GPU"):
        S.sfmp_beam_select(cpu, 2, cpu, None, None, 0, cpu, cpu, cpu, cpu)
    for bad in ([0, 1], None, torch.zeros((1, 1), dtype=torch.int32)):
        with pytest.raises(ValueError, match="group_start has to be a vector"):
            S.kv._groups(bad)
    with pytest.raises(ValueError, match="end of the last group"):
        S.kv._groups(torch.zeros(0, dtype=torch.int32))
    with pytest.raises(ValueError, match="group_start has to be a tensor on the GPU"):
        S.kv._groups(torch.zeros(3, dtype=torch.int32))


# ---- the oracle --------------------------------------------------------------------------------------------------------

def test_oracle_of_a_window_with_first_tokens():
    rng = np.random.default_rng(0)
    Q, K, V = rng.normal(size=(2, 1, 8)), rng.normal(size=(9, 1, 8)), rng.normal(size=(9, 1, 8))
    got = O.attention(Q, K, V, 0.3, 2, 3)[0]
    for i, seen in enumerate(([0, 1, 2, 6, 7], [0, 1, 2, 7, 8])):  # (positions 7 and 8)
        w = np.exp(0.3 * K[seen, 0] @ Q[i, 0])
        assert np.allclose(got[i, 0], w @ V[seen, 0] / w.sum())
    whole = O.attention(Q, K, V, 0.3)[0]
    assert np.allclose(O.attention(Q, K, V, 0.3, 2, 99)[0], whole) and np.allclose(O.attention(Q, K, V, 0.3, 0, 3)[0], whole)


def test_oracle_of_beam_selection():
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.1, 0.8, 0.1]]))
    got, _, _ = O.beam_select(x, [math.log(0.4), math.log(0.3)], 4)
    assert [g[1:] for g in got] == [(1, 1), (0, 0), (0, 1), (0, 2)] and np.allclose([math.exp(g[0]) for g in got], [0.24, 0.2, 0.1, 0.1])
    got, _, _ = O.beam_select(x, [math.log(0.4), math.log(0.3)], 3, weights=[0.1, 1.0], ended=[1, 0], end_token=2)
    assert [g[1:] for g in got] == [(0, 2), (1, 1), (1, 0)] and got[0][0] == math.log(0.4)


def test_oracle_of_reordering():
    t = dict(table=np.array([[0, 1], [0, 2], [3, -1]]), lengths=np.array([100, 70, 5]), refs=np.array([2, 1, 1, 1]))
    O.reorder(t, [0, 1, 2], [1, 1, 0])
    assert t["table"].tolist() == [[0, 2], [0, 2], [0, 1]] and t["lengths"].tolist() == [70, 70, 100] and t["refs"].tolist() == [3, 1, 2, 0]
