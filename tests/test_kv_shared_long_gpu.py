"""Attention over shared pages of long contexts on the GPU: tables that several workgroups compare, parts of many pages, rows whose results are added
up in several turns.  Against 64 bits in torch on the same device."""
import math

import numpy as np
import pytest

from kv_many_util import DEV, Groups, activations, dev, modules, starts
from kv_util import PAGE, U16, UB16, attention_bound, lse_bound, make_pool, pages_of

pytestmark = pytest.mark.gpu


class Long(Groups):
    """As Groups, with tables of long prompts over a pool of few pages: full pages are drawn from it again and again, last ones are a sequence's own.
    change: (tables, pages of each prompt, number of the first sequence of each group) before they are uploaded."""

    def __init__(self, groups, fmt, dim, heads, group, dtype, seed, distinct=160, change=None):
        torch, S = modules()
        rng = np.random.default_rng(7000 + seed)
        self.torch, self.S, self.fmt, self.dtype, self.apart = torch, S, fmt, dtype, 8
        entries = [(g, p, n, t) for g, (p, members) in enumerate(groups) for n, t in members]
        lengths = np.array([p + t for _, p, _, t in entries], dtype=np.int32)
        self.counts = [n for _, _, n, _ in entries]
        n = len(entries)
        self.order = rng.permutation(n + 1)[:n]
        pages = distinct + n
        self.pool = make_pool(rng, 2, pages, heads, dim, fmt)
        table = np.full((n + 1, int(max(pages_of(t) for t in lengths)) + 1), -1, dtype=np.int32)
        prompts = [rng.integers(0, distinct, p // PAGE) for p, _ in groups]
        for b, (g, p, _, t) in enumerate(entries):
            k = pages_of(p + t)
            row = np.concatenate([prompts[g], rng.integers(0, distinct, k - len(prompts[g]))])
            if lengths[b] % PAGE:
                row[-1] = distinct + b
                bad, written = 0x7F if fmt == "fp8" else 0xFF, lengths[b] % PAGE
                codes = self.pool["codes"][:, distinct + b]
                codes[:, :, 0].reshape(2, heads, PAGE, dim)[:, :, written:] = bad
                codes[:, :, 1].reshape(2, heads, dim, PAGE)[:, :, :, written:] = bad
            table[self.order[b], :k] = row
        by_slot = np.zeros(n + 1, dtype=np.int32)
        by_slot[self.order] = lengths
        self.group_start = starts([len(m) for _, m in groups])
        self.tables = dict(table=table, lengths=by_slot)
        if change:
            change(self)
        layout = S.sfmp_kv_query(pages, heads, dim, fmt, 2)
        self.cache = S.DeviceKvCache(layout, dev(torch, self.pool["codes"]), dev(torch, self.pool["scales"].astype(np.float32)))
        self.dt = S.DeviceKvTables(dev(torch, table), dev(torch, by_slot), torch.ones(pages, dtype=torch.int32, device=DEV))
        self.start = starts(self.counts)
        self.rows, self.q_heads, self.dim = int(self.start[-1]), heads * group, dim
        self.Q, self.q = activations(torch, rng, self.rows, self.q_heads, dim, dtype, self.apart)
        self.max_rows, self.max_tokens = max(self.counts), int(lengths.max())
        self.slots, self.starts = dev(torch, self.order.astype(np.int32)), dev(torch, self.group_start)
        self.row_start = dev(torch, self.start) if any(c != 1 for c in self.counts) else None
        self.scale = 1.0 / math.sqrt(dim)
        self.buffers(len(groups))

    def buffers(self, groups, guard=4096):
        """Results, plan and workspace, each of exactly its size, in front of `guard` bytes that nobody may write."""
        torch, S = self.torch, self.S
        sizes = (self.cache.layout, len(self.order), self.rows, groups, self.q_heads, self.max_rows, self.max_tokens)
        self.guarded = []

        def make(shape, dtype, fill):
            n = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
            whole = torch.full((n + guard,), 0xA5, dtype=torch.uint8, device=DEV)
            whole[:n] = fill
            self.guarded.append(whole[n:])
            return whole[:n].view(dtype).view(shape)
        self.out = make((self.rows, self.q_heads * self.dim + self.apart), getattr(torch, self.dtype), 0xFF)  # (NaN)
        self.got = self.out[:, :self.q_heads * self.dim].view(self.rows, self.q_heads, self.dim)
        self.lse = make((self.rows, self.q_heads), torch.float32, 0xFF)
        self.prefix = make((groups,), torch.int32, 0xFF)
        self.plan = make((S.sfmp_kv_share_plan(*sizes),), torch.uint8, 0xFF)
        self.workspace = make((S.sfmp_kv_attention_shared_workspace(*sizes),), torch.uint8, 0xFF)

    def unharmed(self):
        self.torch.cuda.synchronize()
        return all((g == 0xA5).all() for g in self.guarded) and self.torch.isnan(self.out[:, self.q_heads * self.dim:]).all()

    def head(self):
        """(whether the plan is one to use, workgroups of shared pages, pages of a part of shared ones, of own ones)."""
        return self.plan[64:80].view(self.torch.int32).tolist()

    def check(self, window=0, sinks=0, layer=1, entries=None):
        torch = self.torch
        assert self.unharmed()
        heads, dim = self.cache.layout.kv_heads, self.dim
        group = self.q_heads // heads
        codes, scales = self.cache.codes[layer], self.cache.scales[layer].double()
        numbers = codes.view(torch.float8_e4m3fn).float().double() if self.fmt == "fp8" else codes.double() - 128.0
        numbers = numbers * scales[..., None]
        keys = numbers[:, :, 0].view(-1, heads, PAGE, dim)
        values = numbers[:, :, 1].view(-1, heads, dim, PAGE).transpose(2, 3).contiguous()
        for b in range(len(self.order)) if entries is None else entries:
            r = slice(int(self.start[b]), int(self.start[b + 1]))
            n, t = r.stop - r.start, int(self.tables["lengths"][self.order[b]])
            if n == 0:
                continue
            places = torch.from_numpy(self.tables["table"][self.order[b], :pages_of(t)].astype(np.int64)).to(DEV)
            at = torch.arange(t - n, t, device=DEV).repeat_interleave(group)[:, None]
            token = torch.arange(t, device=DEV)
            seen = (token <= at) & ((token > at - window) | (token < sinks)) if window else token <= at
            for h in range(heads):
                K, V = (x[places, h].reshape(-1, dim)[:t] for x in (keys, values))
                rows = slice(h * group, (h + 1) * group)
                q = self.Q[r, rows].reshape(-1, dim).double()
                z = (self.scale * (q @ K.t().contiguous())).masked_fill(~seen, -math.inf)
                lse = torch.logsumexp(z, 1)
                w = torch.exp(z - lse[:, None])
                want, spread = w @ V, w @ V.abs()
                products = (self.scale * (q.abs() @ K.abs().t().contiguous())).masked_fill(~seen, 0.0).amax(1)
                host = lambda x: x.double().cpu().numpy()  # noqa: E731
                want, spread, products, lse = (host(x) for x in (want, spread, products, lse))
                got, got_lse = host(self.got[r, rows].reshape(-1, dim)), host(self.lse[r, rows].reshape(-1))
                bound = attention_bound(U16 if self.dtype == "float16" else UB16, want, spread, products)
                assert (np.abs(got - want) <= bound).all(), (b, h, np.abs(got - want).max())  # (a NaN is not)
                assert (np.abs(got_lse - lse) <= lse_bound(lse, products)).all(), (b, h)


def _run(g, window=0, sinks=0):
    g.share(window, sinks)
    g.attend(window, sinks)
    g.check(window, sinks)
    assert g.prefix.tolist() == g.common_tokens()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_results_of_few_rows_added_up_in_several_turns(fmt, dim):
    # four wavefronts for each of 16 rows and heads, more than 64 partial results for each of them
    g = Long([(128000, [(1, 30), (1, 200)])], fmt, dim, 2, 4, "float16", dim)
    assert g.planned()
    _run(g)
    usable, _, of_group, _ = g.head()
    assert usable and 2000 // of_group > 4 * 64


@pytest.mark.parametrize("tokens,groups,members,heads,group,least", [
    (128000, 1, 20, 2, 16, 64),    # tiles of 128 rows
    (44800, 12, 11, 1, 4, 64)])    # tiles of 32
def test_results_of_many_rows_added_up_in_several_turns(tokens, groups, members, heads, group, least):
    g = Long([(tokens, [(1, 1 + 13 * i) for i in range(members)])] * groups, "int8", 64, heads, group, "bfloat16", groups)
    assert g.planned() and g.rows * g.q_heads > 512  # (one wavefront for each)
    _run(g)
    usable, _, of_group, _ = g.head()
    assert usable and (tokens // PAGE - 1) // of_group >= least


@pytest.mark.parametrize("dim,tokens,groups,members,heads,group", [
    (64, 134400, 1, 32, 4, 16), (128, 134400, 1, 64, 2, 16),   # tiles of 128 rows, a part for each of 512 workgroups
    (128, 8640, 64, 2, 8, 4), (256, 5440, 100, 2, 8, 4)])      # tiles of 32 and 16 rows, one for each of 1024 wavefronts
def test_parts_of_more_pages_than_are_held(dim, tokens, groups, members, heads, group):
    g = Long([(tokens, [(1, 1 + 70 * i) for i in range(members)])] * groups, "int8", dim, heads, group, "float16", dim, distinct=40)
    assert g.planned()
    _run(g)
    usable, _, of_group, _ = g.head()
    assert usable and of_group > 64


@pytest.mark.parametrize("groups,pages", [(1, 130), (1, 300), (1, 2300), (3, 1000), (40, 600), (150, 900), (300, 400), (600, 130)])
def test_tables_that_several_workgroups_compare(groups, pages):
    # (1024 / (groups + 1) workgroups for a group, at most 64 and one for 64 places: 3, 5, 36, 16, 10, 6, 3, 1; the sequences of some groups differ
    # somewhere, in some of them at several places, at the last place of all or at none)
    rng = np.random.default_rng(groups)
    first_other = {}

    def change(g):
        table = g.tables["table"]
        for i in range(groups):
            begin, end = int(g.group_start[i]), int(g.group_start[i + 1])
            for _ in range(int(rng.integers(0, 4))):
                b = int(rng.integers(begin, end))
                place = int(rng.integers(0, pages)) if rng.random() < 0.8 else pages - 1
                table[g.order[b], place] = (table[g.order[b], place] + 1) % 50
                first_other[i] = True
    sizes = [3] * groups if groups > 1 else [70]
    g = Long([(pages * PAGE, [(1, int(rng.integers(1, 100))) for _ in range(sizes[i])]) for i in range(groups)], "int8", 64, 1, 2, "float16", pages,
             distinct=50, change=change)
    assert g.planned() and (groups < 40 or len(first_other) > groups // 2)
    _run(g)


@pytest.mark.parametrize("window,sinks", [(20000, 0), (20000, 130), (9000, 12000), (40, 30000)])
def test_long_windows_and_first_tokens(window, sinks):
    groups = [(60000, [(3, 40 + 500 * i) for i in range(12)]), (30000, [(1, 9000), (2, 25000), (3, 3)]), (0, [(2, 40000), (1, 1)])]
    g = Long(groups, "fp8", 128, 2, 4, "bfloat16", window)
    assert g.planned(window, sinks)
    _run(g, window, sinks)


def test_groups_of_very_different_size_and_sequences_of_none():
    g = Long([(50000, [(1, 11 * i) for i in range(1, 40)]), (7000, [(1, 5000)]), (90000, [(1, 70), (1, 3)]), (3000, [(1, 40 * i) for i in range(1, 9)])],
             "int8", 128, 2, 4, "float16", 1)
    # the entries 38 and 39, behind different prompts, are a group that shares nothing, one group is empty, and the last three entries are in none
    g.group_start = np.array([0, 38, 38, 40, 42, 47], dtype=np.int32)
    g.starts = dev(g.torch, g.group_start)
    g.buffers(5)
    assert g.planned()
    _run(g)


@pytest.mark.parametrize("begin", [[5, 9, 7, 12], [3, 20, 1, 18, -5, 17, 7], [2, 2, 2], [30, 4, 50, -1], [9, 8, 7, 6, 5, 4, 3, 2, 1], [0, 24] * 6])
def test_group_starts_that_do_not_ascend_write_nothing_else(begin):
    """Entries in several groups have unspecified results; nothing is written behind any buffer, and the entries in front of all groups and behind
    them have their results, or, where such starts leave more to do than the workspace holds, no entry has."""
    g = Long([(9000, [(1, 11 * i) for i in range(12)]), (20000, [(1, 5 + i) for i in range(12)])], "int8", 128, 2, 4, "float16", 2)
    g.starts = dev(g.torch, np.array(begin, dtype=np.int32))
    g.buffers(len(begin) - 1)
    assert g.planned()
    g.share()
    g.attend()
    assert g.unharmed()
    usable = g.head()[0]
    start = np.clip(begin, 0, 24)
    held = {b for i in range(len(start) - 1) for b in range(start[i], start[i + 1])}
    alone = [b for b in range(24) if (b < start[0] or b >= start[-1]) and b not in held]
    if usable:
        g.check(entries=alone)
    else:
        assert g.torch.isnan(g.got).all() and g.torch.isnan(g.lse).all()
