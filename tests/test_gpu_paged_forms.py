"""Attention over pages in every form of its kernels: tiles of 16 to 128 rows at both head sizes, masks, absent pages and values that are not finite in each, wide
groups of query heads, tables wider than they are used, costs that are counted in more than single keys, sequences alone and in batches."""
import copy

import pytest
import torch

from tests.paged_helpers import Paged, attend, check_attention, spd_mod
from tests.test_gpu_paged_attention import KINDS, check, queries, tree

pytestmark = pytest.mark.gpu

# packed rows a sequence: up to 16, 32 and 64 in tiles of as many; more: tiles of 64 or 128
MEANS = [([3, 2], 4), ([8, 8], 4), ([5, 3], 7), ([16, 13], 4), ([9], 7), ([30, 41], 3)]


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,group", MEANS)
@pytest.mark.parametrize("lens", [[40, 131], [1700, 2100]])           # (the longer ones' tiles are shared by workgroups)
def test_tiles(dtype, is_e4m3, dim, new, group, lens):
    check(Paged(71, new, lens[: len(new)], 2, dim, 16, is_e4m3), 2 * group, dtype)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("new,lens", [([1, 5], [200, 31]), ([7, 6], [90, 300]), ([12, 16], [70, 20]), ([1, 5, 90], [200, 31, 60])])
@pytest.mark.parametrize("window", [1, 17, 64, 100])
def test_windows(dtype, is_e4m3, new, lens, window):
    check(Paged(window + 1, new, lens, 2, 128, 16, is_e4m3), 6, dtype, window=window)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("new,lens,group", [([1], [0], 2), ([13, 9], [300, 0], 1), ([13, 9], [300, 0], 2), ([16, 13], [50, 1500], 4), ([64, 1, 33], [10, 40, 500], 2)])
def test_trees(dtype, is_e4m3, new, lens, group):
    p = Paged(72, new, lens, 2, 128, 32, is_e4m3)
    check(p, 2 * group, dtype, seen=tree(p.g, new))


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,heads", [([1, 7, 4], 2), ([1, 7, 4], 8), ([1, 7, 30], 8), ([1, 7, 80], 6)])
def test_pages_that_are_not_there(dtype, is_e4m3, dim, new, heads):
    p = Paged(73, new, [300, 90, 40], 2, dim, 16, is_e4m3, extra_columns=3)
    p.table[0, 3:9], p.table[1, 0], p.table[2, 1], p.table[2, 6] = -1, 1 << 30, p.n_pages, -(1 << 31)
    check(p, heads, dtype)
    check(p, heads, dtype, window=40)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,lens,group", [([6], [40], 2), ([7], [60], 4), ([13], [21], 4), ([90], [37], 2)])
def test_values_of_later_rows_that_are_not_finite(dtype, is_e4m3, dim, new, lens, group):
    """A row's key or value that is NaN or infinite concerns the rows that see it, and no other."""
    at, heads = new[0] - 3, 2 * group
    plain = torch.full((2, dim), 0.25)

    def held(k, v):
        p = Paged(74, new, lens, 2, dim, 16, is_e4m3)
        p.put(0, lens[0] + at, k, v)
        return p
    p = held(plain, plain)
    q = queries(p, heads, dtype)
    good, good_lse = attend(p, q)
    check_attention(p, q, good, good_lse)
    for what in ("nan",) if is_e4m3 else ("nan", "inf", "-inf"):
        bad = plain.clone()
        bad[0, 5] = float(what)
        got, lse = attend(held(plain, bad), q)
        assert torch.equal(got[:at], good[:at]) and torch.equal(lse, good_lse)
        assert torch.equal(got[at:, group:], good[at:, group:])                 # the other key head
        same = torch.ones(dim, dtype=torch.bool)
        same[5] = False
        assert torch.equal(got[at:, :group][..., same], good[at:, :group][..., same])
        assert not got[at:, :group, 5].isfinite().any()
        got, lse = attend(held(bad, plain), q)
        assert torch.equal(got[:at], good[:at]) and torch.equal(got[at:, group:], good[at:, group:])
        if what == "nan":
            assert got[at:, :group].isnan().all() and lse[at:, :group].isnan().all()


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [32, 64, 160])
@pytest.mark.parametrize("new,lens,window", [([1], [70], 0), ([1], [1900], 0), ([1, 0, 1, 1], [300, 5, 0, 33], 17), ([3], [200], 0), ([20, 7], [40, 150], 0), ([20, 7], [40, 150], 17)])
def test_wide_groups(dtype, is_e4m3, dim, group, new, lens, window):
    """Tiles that lie within one row, and begin and end inside rows."""
    check(Paged(75, new, lens, 1, dim, 16, is_e4m3), group, dtype, window=window)


def test_as_many_heads_as_there_may_be():
    check(Paged(76, [1, 2], [30, 0], 1, 64, 16), 1024, torch.bfloat16)
    check(Paged(76, [2, 1], [30, 0], 512, 64, 16), 1024, torch.float32)


@pytest.mark.parametrize("dtype,is_e4m3", [(torch.float32, False), (torch.bfloat16, True)])
@pytest.mark.parametrize("new,lens,kv_heads,heads,page,columns,window", [
    ([1, 2], [3000, 40], 2, 8, 256, 1 << 22, 0),           # 2^30 positions: as many as a table may reach
    ([70, 66], [900, 1700], 2, 4, 256, 1 << 22, 0),
    ([70, 66], [900, 1700], 2, 4, 256, 1 << 22, 300),
    ([3, 290, 1], [2500, 20, 7], 4, 8, 32, 1 << 22, 0),    # few and many rows
])
def test_tables_that_reach_far(dtype, is_e4m3, new, lens, kv_heads, heads, page, columns, window):
    """Costs that single keys would take beyond 31 bits are counted in more keys: shares differ, results do not."""
    check(Paged(77, new, lens, kv_heads, 64, page, is_e4m3, extra_columns=columns - max((a + b + page - 1) // page for a, b in zip(new, lens))), heads, dtype, window=window)


def test_many_sequences_with_tables_that_reach_far():
    g = torch.Generator().manual_seed(78)
    lens = torch.randint(0, 60, (1024,), generator=g).tolist()
    lens[500] = 5000
    check(Paged(78, [1] * 1024, lens, 8, 64, 16, False, extra_columns=16384 - 313), 8, torch.bfloat16)


@pytest.mark.parametrize("new", [[2, 3], [90, 70]])
def test_tables_whose_rows_are_apart(new):
    """A part of the columns of a wider table; what is beside it is not looked at."""
    spd = spd_mod()
    p = Paged(79, new, [33, 200], 2, 64, 16)
    q = queries(p, 4, torch.bfloat16)
    want, want_lse = attend(p, q)
    cache, batch = p.device()
    wide = torch.full((2, p.table.shape[1] + 5), 1 << 30, dtype=torch.int32)
    wide[:, 2:-3] = p.table
    apart = spd.PagedBatch(wide.cuda()[:, 2:-3], batch.lens, batch.n_rows, batch.row_start)
    out, lse = torch.empty_like(want), torch.empty_like(want_lse)
    spd.spd_paged_attention(cache, apart, q.cuda(), out, lse_out=lse)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    k = torch.randn((sum(new), 2, 64), generator=p.g).cuda()
    results = []
    for b in (batch, apart):
        cache, _ = p.device()
        spd.spd_paged_append(cache, b, k, k + 1)
        results.append((cache.k, cache.v))
    assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(*results))


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,lens", [([1] * 5, [5, 1900, 33, 0, 450]), ([4, 1, 0, 80, 9], [300, 1500, 20, 64, 0])])
def test_sequences_alone(dtype, is_e4m3, dim, new, lens):
    """A sequence's rows in a batch, and in a call of their own: either within its roundings of 64 bits."""
    spd = spd_mod()
    p = Paged(80, new, lens, 2, dim, 16, is_e4m3)
    q = queries(p, 8, dtype)
    out, lse = attend(p, q)
    cache, batch = p.device()
    for s in range(len(new)):
        if not new[s]:
            continue
        one = copy.copy(p)
        one.new, one.lens, one.table, one.row_start = [new[s]], [lens[s]], p.table[s : s + 1], torch.tensor([0, new[s]], dtype=torch.int32)
        mine = slice(int(p.row_start[s]), int(p.row_start[s + 1]))
        check_attention(one, q[mine], out[mine], lse[mine])
        alone, alone_lse = torch.empty_like(out[mine]), torch.empty_like(lse[mine])
        spd.spd_paged_attention(cache, spd.PagedBatch(batch.page_table[s : s + 1], batch.lens[s : s + 1], new[s]), q[mine].cuda(), alone, lse_out=alone_lse)
        check_attention(one, q[mine], alone, alone_lse)
