"""Inputs of the paged cache's tests and the calls on them (not collected by pytest)."""
import numpy as np
import torch

from oracle import paged as op

U = 2.0 ** -24                       # half a step of float32; bf16 2^-8, e4m3 2^-4
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def spd_mod():
    from paper_2404_08856_amd import spd
    return spd


def f64(t):
    return t.detach().cpu().float().numpy().astype(np.float64)


def e4m3(t):
    return t.clamp(-448, 448).to(torch.float8_e4m3fn)


class Paged:
    """Pages in a shuffled order, cached rows of random values, everything else NaN; on the CPU until device()."""

    def __init__(self, seed, new, lens, kv_heads, dim, page_size, is_e4m3=False, fill=float("nan"), spare=2, extra_columns=0, values=None):
        g = torch.Generator().manual_seed(seed)
        self.g, self.new, self.lens, self.kv_heads, self.dim, self.page_size, self.is_e4m3 = g, list(new), list(lens), kv_heads, dim, page_size, is_e4m3
        spd = spd_mod()
        each = [(a + b + page_size - 1) // page_size for a, b in zip(new, lens)]
        self.n_pages = sum(each) + spare
        order = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((len(new), max(1, max(each)) + extra_columns), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(each):
            self.table[s, :n] = order[at : at + n].int()
            at += n
        self.row_start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
        ks, vs = spd.paged_cache_shapes(self.n_pages, page_size, kv_heads, dim, is_e4m3)
        self.k, self.v = torch.full(ks, fill), torch.full(vs, fill)
        self.k_scale = 0.005 + 0.02 * torch.rand((kv_heads,), generator=g) if is_e4m3 else None
        self.v_scale = 0.005 + 0.02 * torch.rand((kv_heads,), generator=g) if is_e4m3 else None
        for s in range(len(new)):
            for p in range(lens[s] + new[s]):
                self.put(s, p, torch.randn((kv_heads, dim), generator=g), torch.randn((kv_heads, dim), generator=g))

    def put(self, s, p, k, v):
        """Key and value [kv_heads, dim] at position p of sequence s (in e4m3: of magnitudes that its scale keeps)."""
        page, slot = op.place(self.table.numpy(), self.n_pages, self.page_size, s, p)
        G = self.k.shape[-1]
        if self.is_e4m3:
            k, v = k / self.k_scale[:, None], v / self.v_scale[:, None]
        self.k[page, :, :, slot, :] = k.reshape(self.kv_heads, -1, G)
        self.v[page, :, slot // G, :, slot % G] = v

    def held(self):
        """The pages as the cache holds them."""
        return (e4m3(self.k), e4m3(self.v)) if self.is_e4m3 else (self.k.bfloat16(), self.v.bfloat16())

    def device(self, with_row_start=True):
        spd = spd_mod()
        k, v = self.held()
        k, v = (t.view(torch.uint8).cuda().view(t.dtype) if self.is_e4m3 else t.cuda() for t in (k, v))
        cache = spd.PagedCache(k, v, *([self.k_scale.cuda(), self.v_scale.cuda()] if self.is_e4m3 else []))
        batch = spd.PagedBatch(self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(), int(self.row_start[-1]), self.row_start.cuda() if with_row_start else None)
        return cache, batch

    def attention(self, q, scale, window=0, seen=None):
        k, v = self.held()
        return op.attention(f64(q), f64(k), f64(v), self.table.numpy(), self.lens, self.row_start.tolist(), scale, window, seen,
                            None if self.k_scale is None else f64(self.k_scale), None if self.v_scale is None else f64(self.v_scale))


def check_attention(paged, q, out, lse, scale=None, window=0, seen=None):
    """Against 64 bits.  A score: float32 rows are products of 24 bits and, in a chain or a tree, no more than dim + 8 additions of
    magnitudes up to sum |q k| scale, the factor's roundings 4 units of the score, and the exponent's argument 4 more: d = (dim + 16) U work
    + 8 U work.  A weight and the sum that divides it are off by d each, and sums over n positions, in runs of at least 16 and 64 joined ones,
    by n / 16 + 100 units of their terms' magnitudes.  bfloat16 rows: the weights' rounding (2^-8 of the terms), and the output's."""
    scale = paged.dim ** -0.5 if scale is None else scale
    want, want_lse, work, spread, count = paged.attention(q, scale, window, seen)
    d = (paged.dim + 24) * U * work
    sums = (count[:, None] / 16 + 100) * U
    rel = 2 * d + sums
    if q.dtype == torch.bfloat16:
        rel = rel + 2.0 ** -8
    tol = spread * rel[..., None] * (1 + 2.0 ** -8) + HALF[q.dtype] * np.abs(want) + 2.0 ** -126
    got, got_lse = f64(out), f64(lse)
    assert np.isfinite(got).all(), "not finite"
    empty = want_lse == -np.inf
    assert (got[empty] == 0).all() and (got_lse[empty] == -np.inf).all()
    off = np.abs(got - want) / tol
    assert off.max(initial=0) <= 1, f"out: {off.max():.2f} of the tolerance at {np.unravel_index(off.argmax(), off.shape)}"
    lse_tol = (d + sums + 2 * U * np.abs(np.where(empty, 0, want_lse)))
    off = np.abs(got_lse[~empty] - want_lse[~empty]) / lse_tol[~empty]
    assert off.max(initial=0) <= 1, f"lse: {off.max():.2f} of the tolerance"


def attend(paged, q, scale=None, window=0, seen=None, with_row_start=True, workspace=None):
    """out and lse of the call, behind guard rows that have to stay as they were."""
    spd = spd_mod()
    cache, batch = paged.device(with_row_start)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    words = None if seen is None else torch.tensor([w - (1 << 64) if w >> 63 else w for w in seen], dtype=torch.int64, device="cuda")
    spd.spd_paged_attention(cache, batch, q.cuda(), out, scale, window, words, lse, workspace)
    torch.cuda.synchronize()
    return out, lse
