"""Attention over a paged cache against 64 bits: lengths, layouts, masks, pages that are not there, values that are not finite."""
import numpy as np
import pytest
import torch

from oracle import paged as op
from tests.paged_helpers import Paged, attend, check_attention, f64, spd_mod

pytestmark = pytest.mark.gpu

KINDS = [(torch.float32, False), (torch.bfloat16, False), (torch.float32, True), (torch.bfloat16, True)]


def queries(p, heads, dtype, size=2.0):
    return (size * torch.randn((int(p.row_start[-1]), heads, p.dim), generator=p.g)).to(dtype)


def check(p, heads, dtype, **kw):
    q = queries(p, heads, dtype)
    rows = kw.pop("with_row_start", True)
    out, lse = attend(p, q, with_row_start=rows, **kw)
    check_attention(p, q, out, lse, **kw)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page", [
    ([1], [0], 1, 1, 64, 16),                              # one key
    ([1], [1], 2, 1, 128, 16),
    ([1], [640], 4, 4, 128, 16),                           # a token of a conversation
    ([5], [333], 4, 4, 128, 32),                           # a verify block
    ([1, 1, 1, 1, 1], [0, 31, 32, 500, 77], 8, 2, 128, 16),        # a ragged batch
    ([3, 1, 0, 7], [15, 63, 9, 200], 14, 2, 64, 64),       # seven queries a key head, a sequence without rows
    ([40, 1], [5, 300], 12, 4, 64, 16),
    ([2], [1100], 8, 1, 128, 256),
    ([70], [0], 2, 2, 64, 32),                             # a short prompt
    ([150, 33], [20, 0], 6, 3, 128, 16),
    ([257], [130], 2, 1, 64, 128),
])
def test_against_64_bits(dtype, is_e4m3, new, lens, heads, kv_heads, dim, page):
    check(Paged(sum(new) + sum(lens) + dim, new, lens, kv_heads, dim, page, is_e4m3), heads, dtype)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page", [
    ([1], [5000], 4, 1, 128, 16),                          # one head's keys over many workgroups
    ([2, 1], [1, 4100], 2, 2, 64, 64),
    ([3, 1, 0, 2], [2000, 40, 7, 900], 20, 2, 64, 256),    # several tiles a head
    ([100], [1700], 4, 2, 64, 16),                         # many rows, keys shared by workgroups
    ([66, 70], [900, 1500], 1, 1, 128, 128),
    ([5, 300], [1200, 90], 3, 1, 64, 32),                  # few and many rows in a batch
    ([1] * 9 + [290], [33] * 9 + [20], 2, 2, 64, 32),      # one that the mean does not tell of
])
def test_long_caches(dtype, is_e4m3, new, lens, heads, kv_heads, dim, page):
    check(Paged(sum(new) + sum(lens) + dim, new, lens, kv_heads, dim, page, is_e4m3), heads, dtype)


@pytest.mark.parametrize("dtype,is_e4m3", [(torch.float32, False), (torch.bfloat16, True)])
@pytest.mark.parametrize("seqs,most_new,most_len,kv_heads", [(65, 1, 300, 1), (100, 2, 900, 4), (130, 1, 3, 2), (70, 40, 60, 1), (1300, 1, 5, 1)])
def test_many_sequences(dtype, is_e4m3, seqs, most_new, most_len, kv_heads):
    g = torch.Generator().manual_seed(seqs)
    new = torch.randint(0, most_new + 1, (seqs,), generator=g).tolist()
    new[-1] = most_new
    lens = torch.randint(0, most_len + 1, (seqs,), generator=g).tolist()
    check(Paged(seqs, new, lens, kv_heads, 64, 16, is_e4m3), kv_heads, dtype)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("window", [1, 2, 17, 64, 1000])
def test_windows(dtype, is_e4m3, window):
    check(Paged(window, [1, 5, 90], [200, 31, 60], 2, 64, 16, is_e4m3), 6, dtype, window=window)


def tree(g, new):
    """Every row sees itself, the row that it continues, and what that one sees."""
    words = []
    for n in new:
        seen = []
        for j in range(n):
            parent = int(torch.randint(0, j + 1, (1,), generator=g)) - 1
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << j)
        words += seen
    return words


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("new,lens", [([1], [0]), ([13, 9], [300, 0]), ([64, 1, 33], [10, 40, 500])])
def test_trees(dtype, is_e4m3, new, lens):
    p = Paged(9, new, lens, 2, 64, 32, is_e4m3)
    check(p, 4, dtype, seen=tree(p.g, new))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_trees_of_more_rows_than_bits(dtype):
    """Rows from the 65th on are seen by nobody, and see what their bits say."""
    p = Paged(10, [100, 3], [20, 8], 1, 64, 16)
    words = tree(p.g, [64]) + [(1 << 64) - 1] * 18 + [0] * 18 + [0, 7, 0xffff]
    check(p, 2, dtype, seen=words)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
def test_rows_that_see_nothing(dtype, is_e4m3):
    """A tree's word of 0 over an empty cache; a window over pages that were given up."""
    p = Paged(11, [4, 2], [0, 5], 2, 64, 16, is_e4m3)
    check(p, 4, dtype, seen=[0, 1, 0, 15, 0, 0])
    p = Paged(12, [2, 3], [64, 100], 1, 128, 16, is_e4m3)
    p.table[0, 4] = -1                                     # positions 64 .. 79: the first sequence's own rows, and all that their window covers
    p.table[1, :3] = p.n_pages + 5
    check(p, 2, dtype, window=1)
    check(p, 2, dtype, window=70)
    p.table[:] = -1
    check(p, 2, dtype)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
def test_pages_that_are_not_there(dtype, is_e4m3):
    p = Paged(13, [1, 7, 80], [300, 90, 40], 2, 64, 16, is_e4m3)
    p.table[0, 3:9], p.table[1, 0], p.table[2, 1], p.table[2, 6] = -1, 1 << 30, p.n_pages, -(1 << 31)
    check(p, 6, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_lengths_out_of_range(dtype):
    """Below 0: as 0.  Beyond the table: as its end; rows beyond it see what the table has."""
    p = Paged(14, [3, 2, 70], [30, 30, 20], 1, 64, 16, fill=0.5)
    p.lens = [-7, 1 << 30, 95]
    q = queries(p, 2, dtype)
    out, lse = attend(p, q)
    k, v = p.held()
    check_attention(p, q, out, lse)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("each", [1, 4, 40])
def test_equal_numbers_of_rows_without_row_start(dtype, is_e4m3, each):
    check(Paged(15, [each] * 3, [50, 0, 129], 2, 64, 32, is_e4m3), 4, dtype, with_row_start=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1.5])
def test_scales(dtype, scale):
    check(Paged(16, [6, 70], [40, 3], 2, 64, 16), 4, dtype, scale=scale)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("new,lens", [([6], [40]), ([90], [37])])
def test_values_of_later_rows_that_are_not_finite(dtype, is_e4m3, new, lens):
    """A row's key or value that is NaN or infinite concerns the rows that see it, and no other."""
    clean = Paged(17, new, lens, 2, 64, 16, is_e4m3)
    q = queries(clean, 4, dtype)
    want, want_lse = attend(clean, q)
    for what in ("nan", "inf"):
        dirty = Paged(17, new, lens, 2, 64, 16, is_e4m3)
        at = new[0] - 3
        bad = torch.full((2, 64), 0.25)
        bad[0, 5] = float(what)
        dirty.put(0, lens[0] + at, torch.full((2, 64), 0.25), bad)
        other = Paged(17, new, lens, 2, 64, 16, is_e4m3)
        other.put(0, lens[0] + at, torch.full((2, 64), 0.25), torch.full((2, 64), 0.25))
        if is_e4m3 and what == "inf":
            continue                                       # the type has none
        good, good_lse = attend(other, q)
        got, lse = attend(dirty, q)
        assert torch.equal(got[:at], good[:at]) and torch.equal(lse, good_lse)
        assert torch.equal(got[at:, 2:], good[at:, 2:])                    # the other key head
        same = torch.ones(64, dtype=torch.bool)
        same[5] = False
        assert torch.equal(got[at:, :2][..., same], good[at:, :2][..., same])
        assert not got[at:, :2, 5].isfinite().any()
        # a key that is NaN: the whole rows of its head
        dirty.put(0, lens[0] + at, bad, torch.full((2, 64), 0.25))
        got, lse = attend(dirty, q)
        assert torch.equal(got[:at], good[:at]) and torch.equal(got[at:, 2:], good[at:, 2:])
        if what == "nan":
            assert got[at:, :2].isnan().all() and lse[at:, :2].isnan().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_scores_of_minus_infinity_weigh_nothing(dtype):
    """A product beyond float32's range, downwards: as if the key were not there; a row of nothing else sees nothing."""
    p = Paged(18, [3], [20], 1, 64, 16)
    q = queries(p, 2, dtype)
    low = torch.randn((1, 64), generator=p.g)
    q[..., 0] = 1e20
    low[0, 0] = -1e20
    for at in range(23):                                   # the others have nothing there
        p.k[op.place(p.table.numpy(), p.n_pages, 16, 0, at)[0], 0, 0, at % 16, 0] = 0.0
    p.put(0, 7, low, torch.ones((1, 64)))
    out, lse = attend(p, q)
    k, v = p.held()                                        # 64 bits hold the score of -1.25e39: its weight is 0 there
    # sum |q k| of a score below 400
    want, want_lse, _, spread, _ = op.attention(f64(q), f64(k), f64(v), p.table.numpy(), p.lens, p.row_start.tolist(), 0.125)
    tol = spread * (2 * 88 * 2.0 ** -24 * 400 + 2.0 ** -17 + (2.0 ** -8 if dtype == torch.bfloat16 else 0)) + 2.0 ** -8 * np.abs(want) * (dtype == torch.bfloat16)
    assert (np.abs(f64(out) - want) <= tol).all() and np.abs(f64(lse) - want_lse).max() <= 88 * 2.0 ** -24 * 400 + 2.0 ** -17
    p = Paged(19, [1], [0], 1, 64, 16)
    p.put(0, 0, low, torch.ones((1, 64)))
    out, lse = attend(p, q[:1])
    assert (out == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [1, 8])
@pytest.mark.parametrize("new", [[3, 2], [70, 9]])
def test_strides_and_rows_behind_the_last_sequence(dtype, pad, new):
    spd = spd_mod()
    p = Paged(20, new, [33, 100], 2, 64, 16)
    rows, heads, dim = sum(new), 4, 64
    q = queries(p, heads, dtype)
    want, want_lse = attend(p, q)
    cache, batch = p.device()
    batch = spd.PagedBatch(batch.page_table, batch.lens, rows + 5, batch.row_start)
    wide = torch.full((heads, rows + 5, dim + pad), 2.0, dtype=dtype, device="cuda")
    view = wide.permute(1, 0, 2)[..., :dim]
    view[:rows] = q.cuda()
    buffer = torch.full((rows + 5, heads * dim + pad), 5.0, dtype=dtype, device="cuda")
    out = buffer[:, : heads * dim].unflatten(1, (heads, dim))
    lse = torch.full((rows + 5, heads), 5.0, device="cuda")
    spd.spd_paged_attention(cache, batch, view, out, lse_out=lse)
    assert torch.equal(lse[:rows], want_lse) and (lse[rows:] == 5.0).all()
    assert torch.equal(out[:rows], want) and (buffer[rows:] == 5.0).all() and (buffer[:, heads * dim :] == 5.0).all()


def test_one_sequence_s_result_does_not_depend_on_the_others():
    """Values: the same within the tolerance; the call itself gives the same bits every time."""
    p = Paged(21, [1] * 9, [5, 900, 33, 64, 200, 1, 0, 450, 129], 2, 128, 16)
    q = queries(p, 8, torch.bfloat16)
    a, la = attend(p, q)
    for _ in range(5):
        b, lb = attend(p, q)
        assert torch.equal(a, b) and torch.equal(la, lb)
    check_attention(p, q, a, la)


def test_workspaces_hold_anything():
    spd = spd_mod()
    p = Paged(22, [1, 4], [700, 1500], 2, 128, 16)
    q = queries(p, 8, torch.float32)
    cache, batch = p.device()
    n = spd.spd_paged_attention_workspace_bytes(cache, batch, 8)
    results = []
    for fill in (0, 255, 7):
        ws = torch.full((max(n, 1),), fill, dtype=torch.uint8, device="cuda")
        for _ in range(2):
            results.append(attend(p, q, workspace=ws))
    for out, lse in results[1:]:
        assert torch.equal(out, results[0][0]) and torch.equal(lse, results[0][1])


@pytest.mark.parametrize("new", [[1, 1, 1], [40, 3, 90]])
def test_captured_with_lengths_that_move(new):
    """Two graphs on one workspace, replayed in turn with other lengths, against eager calls."""
    spd = spd_mod()
    p = Paged(23, new, [600, 20, 310], 2, 64, 16, fill=0.5)
    q = queries(p, 4, torch.bfloat16).cuda()
    cache, batch = p.device()
    n = spd.spd_paged_attention_workspace_bytes(cache, batch, 4)
    ws = torch.full((max(1, n),), 255, dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q) for _ in range(2)]
    lses = [torch.empty(q.shape[:2], device="cuda") for _ in range(2)]
    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=side):
            spd.spd_paged_attention(cache, batch, q, outs[i], window=40 if i else 0, lse_out=lses[i], workspace=ws)
    for step in range(4):
        batch.lens.sub_(19).clamp_(min=0)
        q.mul_(1.1)
        for i in (0, 1, 0) if step % 2 else (1, 0):
            outs[i].zero_(); lses[i].zero_()
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
            spd.spd_paged_attention(cache, batch, q, out, window=40 if i else 0, lse_out=lse)
            assert torch.equal(out, outs[i]) and torch.equal(lse, lses[i])


def test_on_another_stream_and_two_at_once():
    spd = spd_mod()
    p = Paged(24, [1, 3], [400, 80], 2, 64, 16)
    q = queries(p, 4, torch.float32)
    want, want_lse = attend(p, q)
    cache, batch = p.device()
    q = q.cuda()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(q) for _ in streams]
    for _ in range(10):
        for s, o in zip(streams, outs):
            with torch.cuda.stream(s):
                spd.spd_paged_attention(cache, batch, q, o)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_lse_joins_parts():
    """Attention over a cache and, apart, over its last rows only: joined by lse it is attention over both (each side within its tolerance)."""
    spd = spd_mod()
    p = Paged(25, [4], [200], 1, 64, 16)
    q = queries(p, 2, torch.float32)
    whole, whole_lse = attend(p, q)
    near, near_lse = attend(p, q, window=50)
    cut = Paged(25, [4], [200], 1, 64, 16)
    # rows see p > x - 50; the far part of row i ends at 200 + i - 50: the same cache by another sequence per row
    far = Paged(25, [4], [200], 1, 64, 16)
    far.table = far.table.repeat(4, 1)
    far.new, far.lens, far.row_start = [1] * 4, [200 + i - 50 for i in range(4)], torch.arange(5, dtype=torch.int32)
    out, lse = attend(far, q)
    w = torch.sigmoid(lse.double() - near_lse.double())[..., None]
    joined = w * out.double() + (1 - w) * near.double()
    assert (joined - whole.double()).abs().max().item() <= 64 * 2.0 ** -20
    assert (torch.logaddexp(lse.double(), near_lse.double()) - whole_lse.double()).abs().max().item() <= 2.0 ** -18
