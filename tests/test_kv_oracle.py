"""Pins of the oracle of the 8-bit cache and of sampling that do not go through itself (no GPU)."""
import math

import numpy as np
import pytest

from oracle import sfmp_kv_oracle as O


def test_fp8_values_and_encoding_are_those_of_torch():
    import torch
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(O.fp8_values(), want, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 4001), np.random.default_rng(0).normal(0, 2.0 ** -8, 4000)]).astype(np.float32)
    # (halves between neighbours too: ties)
    v = np.sort(want[np.isfinite(want)])
    x = np.concatenate([x, ((v[1:] + v[:-1]) / 2).astype(np.float32)])
    got = O.encode(x, "fp8")
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(O.decode(got, "fp8"), O.decode(ref, "fp8"))


def test_int8_codes():
    assert O.encode(np.array([0.0, 0.5, 1.5, -0.5, 126.6, 300.0, -300.0]), "int8").tolist() == [128, 128, 130, 128, 255, 255, 1]
    assert O.decode(np.array([1, 128, 255], dtype=np.uint8), "int8").tolist() == [-127.0, 0.0, 127.0]


@pytest.mark.parametrize("largest,want", [(448.0, 1.0), (448.1, 2.0), (1.0, 2.0 ** -8), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7),
                                          (0.0, 0.0), (2.0 ** -101, 0.0), (math.inf, math.nan)])
def test_scale_of_fp8_is_the_least_power_of_two_that_fits(largest, want):
    got = O.scale_for(largest, "fp8")
    assert got == want or (math.isnan(got) and math.isnan(want))


@pytest.mark.parametrize("window", [0, 1, 5])
def test_attention_equals_masked_softmax(window):
    import torch
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(4, 6, 8)), rng.normal(size=(9, 2, 8)), rng.normal(size=(9, 2, 8))
    out, lse, _, _ = O.attention(q, k, v, 0.3, window)
    kk = torch.from_numpy(k).repeat_interleave(3, dim=1).permute(1, 0, 2)
    vv = torch.from_numpy(v).repeat_interleave(3, dim=1).permute(1, 0, 2)
    z = torch.matmul(torch.from_numpy(q).permute(1, 0, 2), kk.transpose(1, 2)) * 0.3
    at, key = torch.arange(5, 9)[:, None], torch.arange(9)[None, :]
    seen = (key <= at) & ((key > at - window) if window else torch.ones_like(key, dtype=torch.bool))
    z = z.masked_fill(~seen, -math.inf)
    want = torch.matmul(torch.softmax(z, dim=-1), vv).permute(1, 0, 2).numpy()
    assert np.allclose(out, want, atol=1e-12) and np.allclose(lse, torch.logsumexp(z, -1).T.numpy(), atol=1e-12)


def test_attention_of_rows_before_the_first_token_is_zero():
    out, lse, _, _ = O.attention(np.ones((3, 2, 4)), np.ones((1, 1, 4)), np.ones((1, 1, 4)), 1.0)
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and (out[2] == 1).all()


def test_append_then_dense_by_hand():
    # two tokens of one head: the second one doubles the scale of the page
    pool = dict(codes=np.full((1, 1, 1, 2, 64 * 2), 9, dtype=np.uint8), scales=np.full((1, 1, 1, 2), 7.0))
    t = dict(table=np.zeros((1, 1), dtype=np.int32), lengths=np.array([1]), refs=np.ones(1, dtype=np.int32))
    O.append(pool, 0, t, [0], [0, 1], np.array([[[12.7, -6.3]]]), np.array([[[1.27, 0.0]]]), "int8")
    assert pool["codes"][0, 0, 0, 0, :4].tolist() == [255, 65, 128, 128]
    assert pool["codes"][0, 0, 0, 1, [0, 64]].tolist() == [255, 128]
    t["lengths"][0] = 2
    O.append(pool, 0, t, [0], [0, 1], np.array([[[25.4, 0.0]]]), np.array([[[0.5, 0.0]]]), "int8")
    assert pool["codes"][0, 0, 0, 0, :4].tolist() == [128 + 64, 128 - 32, 255, 128]  # 63.5 and -31.5: to the even
    assert pool["scales"][0, 0, 0, 0] == np.float32(25.4 / 127) and pool["scales"][0, 0, 0, 1] == np.float32(1.27 / 127)
    k, v = O.dense(pool, 0, t, 0, "int8", 2)
    assert k.shape == (2, 1, 2) and np.isclose(k[1, 0, 0], 25.4) and np.isclose(v[1, 0, 0], 0.5, atol=0.006)


def test_pages_by_hand():
    pool = dict(codes=np.arange(6, dtype=np.uint8).reshape(1, 6, 1, 1, 1), scales=np.zeros((1, 6, 1, 1)))
    t = dict(table=np.full((4, 3), -1, dtype=np.int32), lengths=np.zeros(4, dtype=np.int32), refs=np.zeros(6, dtype=np.int32))
    assert O.reserve(pool, t, [0], [100]) == 0 and t["table"][0].tolist() == [0, 1, -1]
    O.fork(t, [0, 0], [1, 2])
    assert t["refs"].tolist() == [3, 3, 0, 0, 0, 0]
    # three holders of the partly filled page 1 grow: two get copies, the last keeps it
    assert O.reserve(pool, t, [1, 0, 2], [1, 1, 30]) == 0
    assert t["table"][:3].tolist() == [[0, 3, -1], [0, 2, -1], [0, 1, 4]]
    assert t["refs"].tolist() == [3, 1, 1, 1, 1, 0] and pool["codes"].reshape(-1).tolist() == [0, 1, 1, 1, 4, 5]
    assert O.reserve(pool, t, [3], [129]) == 2 and t["lengths"][3] == 0
    assert O.reserve(pool, t, [3], [64 * 4]) == -1
    O.free(t, [0, 2], [64, 130])
    assert t["refs"].tolist() == [3, 1, 1, 0, 1, 0] and t["lengths"].tolist() == [64, 101, 130, 0]
    O.free(t, [1])
    assert t["refs"].tolist() == [2, 1, 0, 0, 1, 0]
    assert O.compact(pool, t) == 3 and t["refs"].tolist() == [2, 1, 1, 0, 0, 0]
    assert t["table"][2].tolist() == [0, 1, 2] and pool["codes"].reshape(-1)[2] == 4


def test_sample_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.1, 0.25, 0.15]))
    pick = lambda **k: O.sample(x, **dict(dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0), **k))[0]  # noqa: E731
    # order 1, 3, 4, 0, 2 with running sums 0.4, 0.65, 0.8, 0.9, 1
    assert [pick(u=u) for u in (0.0, 0.39, 0.41, 0.7, 0.85, 0.95)] == [1, 1, 3, 4, 0, 2]
    assert pick(u=0.95, top_k=2) == 3 and pick(u=0.99, top_k=1) == 1 and pick(u=0.99, temperature=0.0) == 1
    assert pick(u=0.99, top_p=0.6) == 3 and pick(u=0.99, top_p=0.66) == 4 and pick(u=0.99, top_p=0.0) == 1
    assert pick(u=0.99, min_p=0.5) == 3 and pick(u=0.99, min_p=1.0) == 1
    # top-p is taken of what top-k left: 0.6 of (0.4 + 0.25)
    assert pick(u=0.99, top_k=2, top_p=0.6) == 1
    assert O.sample(np.full(3, -math.inf), 1.0, 0, 1.0, 0.0, 0.5)[0] == -1
    assert O.sample(x, 1.0, 0, 1.0, 0.0, 0.5)[1] == pytest.approx(math.log(0.25))
