"""Helpers of the tests of attention over shared pages and over first tokens: calls, and their comparison with the oracle."""
import math

import numpy as np

from oracle import sfmp_kv_oracle as O
from kv_util import PAGE, U16, UB16, attention_bound, lse_bound, make_pool, pages_of, stale_slots, upload

DEV = "cuda:0"


def modules():
    import torch
    assert torch.cuda.is_available()
    import paper_2602_01027_amd as S
    return torch, S


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def starts(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def activations(torch, rng, rows, heads, dim, dtype, apart, std=1.5):
    """(tensor whose rows lie `apart` elements further from each other than they are long, its exact values)."""
    t = torch.from_numpy(rng.normal(0.0, std, size=(rows, heads * dim + apart)).astype(np.float32)).to(getattr(torch, dtype)).to(DEV)
    t = t[:, :heads * dim].view(rows, heads, dim)
    return t, t.float().cpu().numpy()


def compare(pool, tables, order, start, q, got, lse, fmt, dtype, scale, window, sinks, layer=1):
    """Rows start[b] .. start[b + 1] - 1 are those of sequence order[b]; within the bounds that the kernels' arithmetic gives."""
    dim = q.shape[2]
    a, z = got.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    for b, slot in enumerate(order):
        r = slice(int(start[b]), int(start[b + 1]))
        if r.start == r.stop:
            continue
        k, v = O.dense(pool, layer, tables, slot, fmt, dim)
        want, wlse, spread, products = O.attention(q[r], k, v, scale, window, sinks)
        none, nan = np.isneginf(wlse), np.isnan(wlse)
        assert np.array_equal(none, np.isneginf(z[r])) and (a[r][none] == 0).all(), b
        assert np.isnan(z[r][nan]).all() and np.isnan(a[r][nan]).all() and np.isnan(want[nan]).all(), b
        fine = ~(none | nan)
        bound = attention_bound(U16 if dtype == "float16" else UB16, want, spread, products)[fine]
        err = np.abs(a[r] - want)[fine]
        bad = ~((err <= bound) | (np.isnan(a[r][fine]) & np.isnan(want[fine])))
        assert not bad.any(), (b, err[bad].max(), bound[bad].min())
        assert (np.abs(z[r][fine] - wlse[fine]) <= lse_bound(wlse, products)[fine]).all(), b


class Groups:
    """Sequences that share the first pages of their group.  `groups`: (tokens of the prompt, [(rows, tokens behind the prompt)]).
    max_tokens: what the call is told of its longest sequence: by it the library decides whether a plan is worth its while (LONG: it is)."""

    LONG = 60000

    def __init__(self, groups, fmt, dim, heads, group, dtype, seed, apart=8, change=None, spare=2, max_tokens=LONG, slots=True):
        torch, S = modules()
        rng = np.random.default_rng(5000 + seed)
        self.torch, self.S, self.fmt, self.dtype, self.apart = torch, S, fmt, dtype, apart
        entries = [(p, n, t) for p, members in groups for n, t in members]
        self.counts = [n for _, n, _ in entries]
        lengths = [p + t for p, _, t in entries]
        n = len(entries)
        used = sum(p // PAGE for p, _ in groups) + sum(pages_of(p + t) - p // PAGE for p, _, t in entries)
        pages = used + 3
        self.pool = make_pool(rng, 2, pages, heads, dim, fmt)
        self.order = rng.permutation(n + spare)[:n] if slots else np.arange(n)
        table = np.full((n + spare, max(1, max(pages_of(t) for t in lengths)) + 1), -1, dtype=np.int32)
        refs = np.zeros(pages, dtype=np.int32)
        free = rng.permutation(pages).tolist()
        b = 0
        for p, members in groups:
            common = [free.pop() for _ in range(p // PAGE)]
            for _, t in members:
                mine = common + [free.pop() for _ in range(pages_of(p + t) - p // PAGE)]
                table[self.order[b], :len(mine)] = mine
                refs[mine] += 1
                b += 1
        by_slot = np.zeros(n + spare, dtype=np.int32)
        by_slot[self.order] = lengths
        self.tables = dict(table=table, lengths=by_slot, refs=refs)
        stale_slots(self.pool, self.tables, fmt, dim)
        if change:
            change(self.pool, self.tables, self.order)
        self.cache, self.dt = upload(S, self.pool, self.tables, fmt)
        self.start = starts(self.counts)
        self.group_start = starts([len(m) for _, m in groups])
        self.rows, self.q_heads, self.dim = int(self.start[-1]), heads * group, dim
        self.Q, self.q = activations(torch, rng, self.rows, self.q_heads, dim, dtype, apart)
        out = torch.full((self.rows, self.q_heads * dim + apart), math.nan, dtype=getattr(torch, dtype), device=DEV)
        self.out, self.got = out, out[:, :self.q_heads * dim].view(self.rows, self.q_heads, dim)
        self.lse = torch.full((self.rows, self.q_heads), math.nan, dtype=torch.float32, device=DEV)
        self.max_rows, self.max_tokens = max(self.counts), max_tokens or max(1, max(lengths))
        self.slots = dev(torch, self.order.astype(np.int32)) if slots else None
        ragged = any(c != 1 for c in self.counts)
        self.row_start = dev(torch, self.start) if ragged or not slots else None
        self.starts = dev(torch, self.group_start)
        self.prefix = torch.full((len(groups),), -7, dtype=torch.int32, device=DEV)
        sizes = (self.cache.layout, n, self.rows, len(groups), self.q_heads, self.max_rows, self.max_tokens)
        # (neither may depend on what it held)
        self.plan = torch.full((S.sfmp_kv_share_plan(*sizes),), 0xFF, dtype=torch.uint8, device=DEV)
        self.workspace = torch.full((S.sfmp_kv_attention_shared_workspace(*sizes),), 0xFF, dtype=torch.uint8, device=DEV)
        self.scale = 1.0 / math.sqrt(dim)

    def share(self, window=0, sinks=0, stream=None):
        self.S.sfmp_kv_share(self.cache, self.dt, self.slots, self.row_start, self.starts, self.rows, self.q_heads, self.max_rows,
                             self.max_tokens, self.plan, window, sinks, self.prefix, stream)

    def attend(self, window=0, sinks=0, layer=1, stream=None):
        self.S.sfmp_kv_attention_shared(self.cache, layer, self.dt, self.slots, self.row_start, self.starts, self.Q, self.got, self.max_rows,
                                        self.max_tokens, self.scale, self.plan, self.workspace, window, sinks, self.lse, stream)

    def check(self, window=0, sinks=0, layer=1):
        self.torch.cuda.synchronize()
        assert self.apart == 0 or self.torch.isnan(self.out[:, self.q_heads * self.dim:]).all()
        compare(self.pool, self.tables, self.order, self.start, self.q, self.got, self.lse, self.fmt, self.dtype, self.scale, window, sinks, layer)

    def planned(self, window=0, sinks=0):
        """Whether the call with these numbers uses a plan (else it needs none of more than its head)."""
        whole, self.plan = self.plan, self.plan[:256].clone()
        try:
            self.attend(window, sinks)
            return False
        except self.S.SfmpError as e:
            assert e.code == -5
            return True
        finally:
            self.plan = whole

    def common_tokens(self):
        """What the sequences of each group share, from the tables."""
        found = []
        for g in range(len(self.group_start) - 1):
            slots = self.order[self.group_start[g]:self.group_start[g + 1]]
            n = 0
            while len(slots) and all((n + 1) * PAGE <= self.tables["lengths"][s] and self.tables["table"][s, n] == self.tables["table"][slots[0], n]
                                     for s in slots):
                n += 1
            found.append(n * PAGE)
        return found
