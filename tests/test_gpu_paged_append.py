"""Appending to a paged cache: every element of the cache against 64 bits, also those that have to stay as they were."""
import numpy as np
import pytest
import torch

from oracle import paged as op
from tests.paged_helpers import HALF, Paged, U, e4m3, f64, spd_mod

pytestmark = pytest.mark.gpu


def bits(t):
    return t.view(torch.uint8 if t.dtype == torch.float8_e4m3fn else torch.int16).cpu()


def expected(paged, k, v, freq, m, interleaved, positions):
    """Pages after the append as the values in 64 bits that are rounded, and which elements are written."""
    k0, v0 = paged.held()
    want_k, want_v = f64(k0), f64(v0)
    wrote_k, wrote_v = np.zeros(want_k.shape, bool), np.zeros(want_v.shape, bool)
    size = np.zeros(want_k.shape)
    G, table = want_k.shape[-1], paged.table.numpy()
    capacity = table.shape[1] * paged.page_size
    ks = 1.0 if paged.k_scale is None else f64(paged.k_scale)[:, None]
    own = np.zeros(k.shape[0], np.int64)
    for s in range(len(paged.new)):
        for i in range(paged.new[s]):
            r = int(paged.row_start[s]) + i
            own[r] = min(max(paged.lens[s], 0), capacity) + i
    at = own if positions is None else positions
    turned = f64(k) if freq is None else op.turned(f64(k), at, freq, m, interleaved)
    # |a| + |b| of each element's pair
    pair = np.abs(f64(k)).copy()
    if freq is not None:
        n = len(freq)
        a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
        pair[..., a] = pair[..., b] = np.abs(f64(k))[..., a] + np.abs(f64(k))[..., b]
    for s in range(len(paged.new)):
        for i in range(paged.new[s]):
            r = int(paged.row_start[s]) + i
            where = op.place(table, paged.n_pages, paged.page_size, s, int(own[r]))
            if where is None:
                continue
            page, slot = where
            want_k[page, :, :, slot, :] = (turned[r] / ks).reshape(paged.kv_heads, -1, G)
            size[page, :, :, slot, :] = (pair[r] / ks).reshape(paged.kv_heads, -1, G)
            wrote_k[page, :, :, slot, :] = True
            # values: one division in float32 (exact in its rounding) and the rounding to the cache's type
            x = v[r].float() if paged.v_scale is None else v[r].float() / paged.v_scale[:, None]
            want_v[page, :, slot // G, :, slot % G] = f64(e4m3(x) if paged.is_e4m3 else x.bfloat16())
            wrote_v[page, :, slot // G, :, slot % G] = True
    return want_k, want_v, wrote_k, wrote_v, size, turned, at


def check(paged, heads, dtype, R=0, interleaved=False, positions=None, with_row_start=True, behind=0, pad=0, size=1.0, same_q=False):
    spd = spd_mod()
    rows, dim, HK = int(paged.row_start[-1]) + behind, paged.dim, paged.kv_heads
    qkv = size * torch.randn((rows, heads + 2 * HK, dim + pad), generator=paged.g).to(dtype)
    q, k, v = qkv[..., :dim].split([heads, HK, HK], 1)
    rope = freq = None
    if R:
        rope, freq = spd.Rope(R, interleaved=interleaved, theta=20000.0, magnitude=1.25), op.frequencies(R, 20000.0)
    k0, v0 = paged.held()
    cache, batch = paged.device(with_row_start)
    batch = spd.PagedBatch(batch.page_table, batch.lens, rows, batch.row_start)
    on = qkv.cuda()
    qd, kd, vd = on[..., :dim].split([heads, HK, HK], 1)
    out = (qd if same_q else torch.full((rows, heads, dim), 3.0, dtype=dtype, device="cuda")) if R else None
    where = None if positions is None else torch.tensor(positions, dtype=torch.int32).cuda()
    spd.spd_paged_append(cache, batch, kd, vd, rope=rope, positions=where, q=qd if R else None, q_out=out)
    torch.cuda.synchronize()
    want_k, want_v, wrote_k, wrote_v, pair, _, at = expected(paged, k, v, freq, 1.25, interleaved, None if positions is None else np.asarray(positions))
    got_k, got_v = f64(cache.k), f64(cache.v)
    # not written: the same bits
    keep_k, keep_v = torch.from_numpy(~wrote_k), torch.from_numpy(~wrote_v)
    assert torch.equal(bits(cache.k)[keep_k], bits(k0)[keep_k]) and torch.equal(bits(cache.v)[keep_v], bits(v0)[keep_v])
    assert np.array_equal(got_v[wrote_v], want_v[wrote_v])
    want = want_k[wrote_k]
    m = 1.25 if R else 1.0
    # before the rounding to the cache's type: the turn (8 units, as spd_rope_apply), and in e4m3 one division
    near = pair[wrote_k] * m * 10 * U
    if paged.is_e4m3:
        tol = near + np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) * (1 + 2.0 ** -8)       # half a step of e4m3, of its smallest values 2^-10
        want = np.clip(want, -448, 448)
    else:
        tol = near + 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8)
    off = np.abs(got_k[wrote_k] - want)
    assert (off <= tol).all(), f"{(off / np.maximum(tol, 1e-300)).max()} of the tolerance"
    if R:
        mine = int(paged.row_start[-1])
        full = np.zeros(rows, np.int64)
        full[: len(at)] = at
        want_q = op.turned(f64(q), full, freq, 1.25, interleaved)
        wide = f64(q)
        n = R // 2
        a, b = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, n), slice(n, R))
        tol = np.zeros_like(wide)
        tol[..., a] = tol[..., b] = (np.abs(wide[..., a]) + np.abs(wide[..., b])) * 1.25 * 8 * U
        if dtype == torch.bfloat16:
            tol[..., :R] += 2.0 ** -8 * np.abs(want_q[..., :R]) * (1 + 2.0 ** -8)
        assert (np.abs(f64(out) - want_q)[:mine] <= tol[:mine]).all()
        assert torch.equal(out[mine:].cpu(), q[mine:] if same_q else torch.full_like(q[mine:], 3.0))


KINDS = [(torch.float32, False), (torch.bfloat16, False), (torch.float32, True), (torch.bfloat16, True)]


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page,R,interleaved", [
    ([1], [0], 1, 1, 64, 16, 0, False), ([1], [16], 4, 2, 128, 16, 128, False), ([5], [13], 8, 8, 128, 16, 128, False), ([1, 1, 1], [15, 16, 33], 6, 3, 64, 32, 64, True),
    ([40, 1, 0, 17], [3, 100, 5, 0], 6, 2, 64, 16, 32, True), ([130], [7], 3, 1, 128, 64, 66, False), ([64, 64], [0, 64], 4, 4, 64, 256, 64, False),
    ([300, 2], [1, 250], 2, 1, 64, 128, 10, True)])
def test_against_64_bits(dtype, is_e4m3, new, lens, heads, kv_heads, dim, page, R, interleaved):
    check(Paged(sum(new) + dim, new, lens, kv_heads, dim, page, is_e4m3, fill=0.5), heads, dtype, R, interleaved)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
def test_rows_of_equal_numbers_without_row_start(dtype, is_e4m3):
    check(Paged(3, [5] * 7, [0, 11, 16, 31, 32, 100, 63], 2, 64, 32, is_e4m3, fill=0.5), 4, dtype, 64, with_row_start=False)


@pytest.mark.parametrize("dtype,is_e4m3", [(torch.float32, False), (torch.bfloat16, True)])
@pytest.mark.parametrize("seqs", [65, 1024, 1025, 1500])
def test_many_sequences(dtype, is_e4m3, seqs):
    g = torch.Generator().manual_seed(seqs)
    new = torch.randint(0, 4, (seqs,), generator=g).tolist()
    check(Paged(seqs, new, torch.randint(0, 20, (seqs,), generator=g).tolist(), 1, 64, 16, is_e4m3, fill=0.5), 1, dtype, 64)


@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_behind_the_last_sequence_and_queries_in_place(dtype, pad):
    check(Paged(4, [3, 9], [5, 0], 2, 64, 16, fill=0.5), 4, dtype, 32, behind=6, pad=pad, same_q=True)


def test_positions_of_their_own():
    positions = [900, 901, 901, 902, 5, 0, 123456]
    check(Paged(5, [4, 3], [20, 7], 2, 64, 16, fill=0.5), 2, torch.float32, 64, positions=positions)


@pytest.mark.parametrize("is_e4m3", [False, True])
def test_no_place(is_e4m3):
    """Entries that name no page, positions beyond the table, lengths out of range: dropped, everything else appended."""
    p = Paged(6, [20, 20, 5, 3], [10, 40, 30, 0], 1, 64, 16, is_e4m3, fill=0.5)
    p.table[0, 1], p.table[1, 3] = -1, p.n_pages            # positions 16..31 of the first, 48..63 of the second
    p.lens[2], p.lens[3] = 1000, -4                          # beyond the table's 64 positions; counts as 0
    check(p, 2, torch.float32, 64)


@pytest.mark.parametrize("is_e4m3", [False, True])
def test_values_beyond_the_type_and_nan(is_e4m3):
    spd = spd_mod()
    p = Paged(7, [3], [0], 1, 64, 16, is_e4m3, fill=0.5)
    k = torch.randn((3, 1, 64), generator=p.g)
    k[0, 0, :5] = torch.tensor([1e30, -1e30, float("inf"), -float("inf"), float("nan")])
    cache, batch = p.device()
    spd.spd_paged_append(cache, batch, k.cuda(), k.cuda())
    for pages, scale in ((cache.k[p.table[0, 0]].cpu().float()[0, :, 0], p.k_scale), (cache.v[p.table[0, 0]].cpu().float()[0, 0, :, 0], p.v_scale)):
        got = pages.reshape(-1)[:5]
        want = torch.tensor([448.0, -448.0, 448.0, -448.0]) if is_e4m3 else k[0, 0, :4].bfloat16().float()
        assert torch.equal(got[:4], want) and got[4].isnan()


def test_captured_with_lengths_that_move():
    spd = spd_mod()
    p = Paged(8, [2, 2], [20, 3], 2, 64, 16, fill=0.5, extra_columns=0)
    cache, batch = p.device(False)
    k = torch.randn((4, 2, 64), generator=p.g).cuda()
    rope = spd.Rope(64)
    before = cache.k.clone(), cache.v.clone()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        spd.spd_paged_append(cache, batch, k, k, rope=rope)
    for step in range(3):
        cache.k.copy_(before[0]); cache.v.copy_(before[1])
        batch.lens.sub_(1)
        k.add_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = cache.k.clone(), cache.v.clone()
        cache.k.copy_(before[0]); cache.v.copy_(before[1])
        spd.spd_paged_append(cache, batch, k, k, rope=rope)
        torch.cuda.synchronize()
        assert torch.equal(got[0], cache.k) and torch.equal(got[1], cache.v) and not torch.equal(got[0], before[0])
