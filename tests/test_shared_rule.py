"""Which calls of attention over shared pages are worth a plan, as the library decides on the host: a call that is not needs no more of the plan than its
head, and sfmp_kv_share launches nothing for it where no prefix is asked for (no GPU needed, nothing is launched)."""
import pytest

from test_many_host import WORKSPACE, call
import paper_2602_01027_amd as S


def _planned(batch, groups, tokens, heads, group, dim, max_rows=1, window=0, sinks=0):
    code = call("kv_share", L=S.sfmp_kv_query(16, heads, dim, "int8", 1), batch=batch, rows=batch * max_rows, max_rows=max_rows, groups=groups,
                q_heads=heads * group, max_tokens=tokens, window=window, sinks=sinks, sequences=batch, table_pages=tokens // 64 + 1, prefix=None, plan_bytes=256)
    assert code in (0, WORKSPACE)
    return code == WORKSPACE


LAYOUTS = [(8, 4, 128), (8, 4, 64), (4, 4, 256), (2, 8, 128)]


@pytest.mark.parametrize("heads,group,dim", LAYOUTS)
def test_nearly_as_many_groups_as_sequences_are_not_worth_a_plan(heads, group, dim):
    # us a layer, shared all but a page, planned against alone (heads and layouts in the order above): 64 of 3000 tokens in 63 groups 94 / 73, 40 / 32,
    # 84 / 73, 27 / 27; 96 of 3000 in 95 131 / 106, 58 / 47, 116 / 117, 34 / 25; of 8000 in 84 1.05 to 1.34 times
    for batch, groups, tokens in ((64, 63, 3000), (96, 95, 3000), (64, 63, 8000), (96, 95, 8000), (96, 84, 8000), (64, 56, 8000)):
        assert not _planned(batch, groups, tokens, heads, group, dim), (batch, groups, tokens)


@pytest.mark.parametrize("heads,group,dim", LAYOUTS)
def test_groups_of_many_sequences_are(heads, group, dim):
    # 96 of 8000 tokens in one group 0.25 to 0.58 times, in 24 0.46 to 0.66; 64 in 8 0.26 to 0.65
    for batch, groups, tokens in ((96, 1, 8000), (96, 24, 8000), (64, 8, 8000), (64, 16, 8000)):
        assert _planned(batch, groups, tokens, heads, group, dim), (batch, groups, tokens)


def test_few_sequences():
    # 2 of 3000 tokens 11.7 us against 14.7, 2 of 16000 18 and 26, 4 of 8000 in 2 groups 15.4 and 21.9; one for each group is never worth it
    assert _planned(2, 1, 3000, 8, 4, 128) and _planned(2, 1, 16000, 8, 4, 128) and _planned(4, 2, 8000, 8, 4, 128)
    assert not _planned(4, 4, 8000, 8, 4, 128) and not _planned(64, 64, 60000, 8, 4, 128) and not _planned(1, 0, 8000, 8, 4, 128)


def test_more_groups_are_never_worth_more():
    for heads, group, dim in LAYOUTS:
        for batch in (2, 5, 16, 33, 96, 500):
            for tokens in (500, 1500, 3000, 9000, 60000):
                # (tiles of 128 rows start later than smaller ones: among the groups of each kind)
                of_kind = {}
                for groups in range(1, batch, max(batch // 24, 1)):
                    of_kind.setdefault(-(-batch * group // groups) <= 64, []).append(_planned(batch, groups, tokens, heads, group, dim))
                for worth in of_kind.values():
                    assert worth == sorted(worth, reverse=True), (heads, dim, batch, tokens, worth)
