"""Attention over pages with bfloat16 rows: what the rounding of the softmax's weights may do to a result.

Many packed rows a sequence: the weights of the product with v are rounded to bfloat16 (a relative error of up to 2^-8 each, r_i = w_i (1 + e_i)), and the result is
divided by the sum of the rounded ones:  sum r_i v_i / sum r_i - o = sum p_i e_i (v_i - o) / sum p_i (1 + e_i),  at most 2^-8 / (1 - 2^-8) of sum p_i |v_i - o|.  So what all
keys of a row agree on, or one key outweighs, is exact to float32's roundings, those of check_attention.  Few: two terms of bfloat16, 2^-16 of each weight."""
import numpy as np
import pytest
import torch

from oracle import paged as op
from tests.paged_helpers import Paged, U, attend, e4m3, f64

pytestmark = pytest.mark.gpu

# few and many packed rows; alone and shared by workgroups
SIZES = [([1], [40], 1), ([3, 2], [300, 31], 4), ([1, 2], [5000, 700], 8), ([9], [64], 4), ([90, 5], [37, 200], 2), ([100], [1900], 2)]


def exact(p, q, scale, window=0):
    """out, lse, |v| and |v - out| averaged by the weights, the largest sum |q k| scale of a row's scores, and the keys that it sees, in 64 bits."""
    k_pages, v_pages = (f64(t) for t in p.held())
    table, rows, heads = p.table.numpy(), q.shape[0], q.shape[1]
    out, spread, apart = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
    lse, work, count = np.zeros((rows, heads)), np.zeros((rows, heads)), np.zeros(rows)
    x = f64(q)
    for s, (n, old) in enumerate(zip(p.new, p.lens)):
        places = [op.place(table, p.n_pages, p.page_size, s, at) for at in range(old + n)]
        for h in range(heads):
            g = h // (heads // p.kv_heads)
            k = np.stack([op.key_at(k_pages, page, g, t) for page, t in places]) * (1.0 if p.k_scale is None else float(p.k_scale[g]))
            v = np.stack([op.value_at(v_pages, page, g, t) for page, t in places]) * (1.0 if p.v_scale is None else float(p.v_scale[g]))
            for i in range(n):
                r, lo, hi = int(p.row_start[s]) + i, max(0, old + i - window + 1) if window else 0, old + i + 1
                z = k[lo:hi] @ x[r, h] * scale
                e = np.exp(z - z.max())
                w = e / e.sum()
                out[r, h] = w @ v[lo:hi]
                spread[r, h], apart[r, h] = w @ np.abs(v[lo:hi]), w @ np.abs(v[lo:hi] - out[r, h])
                lse[r, h], work[r, h], count[r] = z.max() + np.log(e.sum()), (np.abs(k[lo:hi]) @ np.abs(x[r, h])).max() * scale, hi - lo
    return out, lse, spread, apart, work, count


def check(p, q, window=0):
    scale = p.dim ** -0.5
    out, lse = attend(p, q, window=window)
    want, want_lse, spread, apart, work, count = exact(p, q, scale, window)
    d = (p.dim + 24) * U * work
    sums = (count[:, None] / 16 + 100) * U
    many = -(-q.shape[0] // len(p.new)) * (q.shape[1] // p.kv_heads) > 32
    # before the result's own rounding, which keeps an order
    wide = spread * (2 * d + 2 * sums)[..., None] + (apart * 2.0 ** -8 * (1 + 2.0 ** -7) if many else spread * 2.0 ** -16)
    low, high = (f64(torch.from_numpy(t).float().bfloat16()) for t in (want - wide, want + wide))
    got = f64(out)
    wrong = (got < low) | (got > high)
    assert not wrong.any(), f"{wrong.sum()} of {wrong.size}: {got[wrong][:4]} not in {low[wrong][:4]} .. {high[wrong][:4]}"
    assert (np.abs(f64(lse) - want_lse) <= d + sums + 2 * U * np.abs(want_lse)).all()
    return got, want


def elements(p, x):
    """Four elements of the cache's type that add up to x in each head."""
    rest, parts = (x / p.k_scale if p.is_e4m3 else torch.full((p.kv_heads,), x)), []
    for _ in range(4):
        parts.append(e4m3(rest).float() if p.is_e4m3 else rest.bfloat16().float())
        rest = rest - parts[-1]
    return torch.stack(parts, 1)


def set_score(p, s, at, score):
    """The key at a position so that queries of 16 in the first four elements have the score."""
    page, slot = op.place(p.table.numpy(), p.n_pages, 16, s, at)
    p.k[page, :, 0, slot, :4] = elements(p, score * p.dim ** 0.5 / 16.0)


def set_value(p, s, at, value):
    """The values [kv_heads, dim] (or one for all) at a position, as the cache holds them."""
    page, slot = op.place(p.table.numpy(), p.n_pages, 16, s, at)
    p.v[page, :, slot // p.v.shape[-1], :, slot % p.v.shape[-1]] = value


def sixteens(p, heads):
    q = torch.zeros((sum(p.new), heads, p.dim))
    q[..., :4] = 16.0
    return q.bfloat16()


@pytest.mark.parametrize("is_e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,lens,group", SIZES)
def test_values_that_are_the_same_at_every_key(is_e4m3, dim, new, lens, group):
    """Weights of all sizes, one value: the result is that value, which bfloat16 holds."""
    p = Paged(41 + dim, new, lens, 2, dim, 16, is_e4m3)
    if is_e4m3:
        p.v_scale = torch.tensor([2.0 ** -6, 2.0 ** -5])
    value = torch.where(torch.rand((2, dim), generator=p.g) < 0.5, -1.0, 1.0) * (1.875 if is_e4m3 else 1.9921875)
    for s in range(len(new)):
        for at in range(new[s] + lens[s]):
            set_value(p, s, at, value)
    got, want = check(p, (2 * torch.randn((sum(new), 2 * group, dim), generator=p.g)).bfloat16())
    assert np.array_equal(got, want.astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("is_e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,lens,group", SIZES)
def test_one_key_outweighs_the_others(is_e4m3, dim, new, lens, group):
    """Behind a start of scores of 0 a key of a score of 2 to 6, below the sums at which a reference is set anew, or of 30, beyond them."""
    for score in (2.0, 2.7, 4.1, 6.3, 30.0):
        p = Paged(43 + dim, new, lens, 2, dim, 16, is_e4m3)
        for s in range(len(new)):
            for at in range(new[s] + lens[s]):
                set_score(p, s, at, score if at == (new[s] + lens[s]) * 3 // 4 else 0.0)
        check(p, sixteens(p, 2 * group))


@pytest.mark.parametrize("is_e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,lens,group", SIZES)
@pytest.mark.parametrize("power", [1, 4])
def test_equal_scores_below_a_higher_one(is_e4m3, dim, new, lens, group, power):
    """Behind a first key of score 0 all weights are the same, and so are their roundings: 2^-power (1 + 2^-8 31 / 32), nearly half a step off.  All values but the first key's are alike."""
    p = Paged(47 + dim, new, lens, 2, dim, 16, is_e4m3)
    score = float((np.log2(1 + 2.0 ** -8 * 31 / 32) - power) * np.log(2.0))
    for s in range(len(new)):
        for at in range(new[s] + lens[s]):
            set_score(p, s, at, score if at else 0.0)
            if at:
                set_value(p, s, at, 1.875)
    check(p, sixteens(p, 2 * group))


@pytest.mark.parametrize("is_e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,lens,group", SIZES)
@pytest.mark.parametrize("window", [0, 70])
def test_random_scores(is_e4m3, dim, new, lens, group, window):
    p = Paged(53 + dim, new, lens, 2, dim, 16, is_e4m3)
    check(p, (3 * torch.randn((sum(new), 2 * group, dim), generator=p.g)).bfloat16(), window)
