"""Log probabilities, entropy, rank and alternatives against 64 bits: whole numbers equal, the rest within float32's roundings."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def spd_mod():
    from paper_2404_08856_amd import spd
    return spd


def reference(rows, tokens, temperature, probs, top):
    """Values and how far float32 may be from them.  z: one rounding each for the difference, 1 / T and the product.  A sum of
    V terms, however it is nested over at most 2^8 terms a level, is off by less than 2^8 * 2^-24 of its terms' magnitudes; a term's
    exponential by 4 |z - max| + 4 units of 2^-24."""
    n, V = rows.shape
    eps = 2.0 ** -24
    p = rows.astype(np.float64)
    out = {"lp": np.empty(n), "h": np.empty(n), "rank": np.empty(n, np.int64), "ids": np.full((n, top), -1), "ilp": np.full((n, top), -np.inf)}
    tol = {k: np.zeros_like(out[k], dtype=np.float64) for k in ("lp", "h", "ilp")}
    for r in range(n):
        v, t = p[r], int(tokens[r])
        known = 0 <= t < V
        bad = np.isnan(v).any() or (v == np.inf).any() or (probs and (v < 0).any())
        if bad:
            out["lp"][r] = out["h"][r] = np.nan
            out["rank"][r] = -1
            out["ilp"][r] = np.nan
            continue
        live = v > (0.0 if probs else -np.inf)
        lp, e = np.full(V, -np.inf), np.full(V, 0.0)
        if live.any():
            if probs:
                lp[live] = np.log(v[live])
                e[live] = 4 * eps * (1 + np.abs(lp[live]))
                h_tol = eps * np.sum(v[live] * (260 * np.abs(lp[live]) + 8))
            else:
                d = (v - v.max()) / temperature
                w = np.exp(d)
                total = w.sum()
                lp[live] = d[live] - np.log(total)
                m = w[live] / total
                mean = np.sum(m * np.abs(d[live]))
                log_tol = eps * (264 + 4 * mean + 4 * np.log(total))
                e[live] = 4 * eps * np.abs(d[live]) + log_tol + 2 * eps * np.abs(lp[live])
                h_tol = log_tol + eps * np.sum(m * np.abs(d[live]) * (540 + 8 * np.abs(d[live]) + 4 * mean))
            q = np.exp(lp[live])
            out["h"][r] = -np.sum(q * lp[live])
            tol["h"][r] = h_tol
        else:
            out["h"][r] = 0.0
        out["lp"][r] = lp[t] if known else -np.inf
        tol["lp"][r] = e[t] if known else 0.0
        order = np.argsort(-v, kind="stable")
        out["rank"][r] = int(np.nonzero(order == t)[0][0]) if known else V
        best = order[:top][live[order[:top]]]
        out["ids"][r, : len(best)] = best
        out["ilp"][r, : len(best)], tol["ilp"][r, : len(best)] = lp[best], e[best]
    return out, tol


def call(rows, tokens, temperature, probs, top, pad=0):
    spd = spd_mod()
    n, V = rows.shape
    wide = torch.full((n, V + pad), float("nan"), device="cuda")
    wide[:, :V] = torch.from_numpy(rows).cuda()
    new = lambda s, t: torch.full(s, -7, dtype=t, device="cuda")
    lp, h, rank = new((n,), torch.float32), new((n,), torch.float32), new((n,), torch.int32)
    ids, ilp = new((n, top), torch.int32), new((n, top), torch.float32)
    spd.spd_token_logprobs(wide[:, :V], torch.from_numpy(np.asarray(tokens, np.int32)).cuda(), temperature, spd.SPD_ROWS_ARE_PROBS if probs else 0, lp, h, rank, ids, ilp)
    return {k: v.cpu().numpy() for k, v in (("lp", lp), ("h", h), ("rank", rank), ("ids", ids), ("ilp", ilp))}


def check(rows, tokens, temperature=1.0, probs=False, top=5, pad=0):
    rows = np.ascontiguousarray(rows, dtype=np.float32)
    got = call(rows, tokens, temperature, probs, top, pad)
    want, tol = reference(rows, tokens, float(np.float32(temperature)), probs, top)
    assert np.array_equal(got["rank"], want["rank"]) and np.array_equal(got["ids"], want["ids"])
    for k in ("lp", "h", "ilp"):
        fine = np.isfinite(want[k])
        assert np.array_equal(got[k][~fine], want[k][~fine].astype(np.float32), equal_nan=True), k
        assert np.all(np.abs(got[k][fine] - want[k][fine]) <= tol[k][fine]), (k, np.max(np.abs(got[k][fine] - want[k][fine]) - tol[k][fine]))


def logits(n, V, seed, scale=2.0):
    rng = np.random.default_rng(seed)
    x = scale * rng.standard_normal((n, V))
    x[np.arange(n), rng.integers(0, V, n)] += 6
    return x.astype(np.float32), rng.integers(0, V, n)


@pytest.mark.parametrize("V", [1, 2, 3, 31, 64, 100, 1000, 1024, 4095, 8192, 12289, 32000, 32003, 32768, 32769, 65536, 100003, 131072])
@pytest.mark.parametrize("n,top", [(1, 5), (3, 32), (2, 0), (3, 1)])
def test_vocabularies_of_any_size(V, n, top):
    x, t = logits(n, V, V + n)
    check(x, t, 1.0, False, top)


@pytest.mark.parametrize("V", [77, 32000, 40001])
@pytest.mark.parametrize("temperature", [0.05, 0.7, 3.0])
@pytest.mark.parametrize("pad", [0, 1, 4])
def test_temperatures_and_strided_rows(V, temperature, pad):
    x, t = logits(6, V, V)
    check(x, t, temperature, False, 7, pad)


@pytest.mark.parametrize("V", [50, 5000, 32000, 70000])
def test_probability_rows(V):
    x, t = logits(5, V, V)
    p = torch.softmax(torch.from_numpy(x).double(), -1).float().numpy()
    p[1] = 0
    p[1, V // 2] = 1                                       # what a draft step leaves at temperature 0
    p[2, ::2] = 0
    p[3] = 0                                               # nothing
    check(p, t, 0.0, True, 6)


@pytest.mark.parametrize("V", [40, 1000, 32000, 33000])
@pytest.mark.parametrize("top", [4, 32])
def test_equal_entries_go_by_index(V, top):
    rng = np.random.default_rng(V)
    x = np.stack([np.zeros(V), np.where(np.arange(V) % 2, 0.0, -0.0), rng.integers(0, 3, V), rng.integers(0, 60, V), np.arange(V) // 7, -(np.arange(V) // 5)]).astype(np.float32)
    check(x, [V - 1, V // 2, 3, V // 3, 0, V - 2], 1.0, False, top)


@pytest.mark.parametrize("V", [64, 4096, 32000, 36001])
def test_entries_that_gather_in_one_place(V):
    """Descending, ascending and comb-like rows: whatever part of the row a thread or a wave holds, the first ones may all sit there."""
    i = np.arange(V)
    rows = [-i * 0.01, i * 0.01, np.where(i % 64 == 5, 9.0 + i * 1e-4, 0.0), np.where(i % 256 < 4, 9.0 + i * 1e-4, 0.0), np.where(i % 4096 < 4, 9.0 - i * 1e-4, -1.0),
            np.where(i >= V - 40, 9.0 + i * 1e-3, i * 1e-5), np.where(i < 600, 9.0 + (i % 7), 0.0)]
    check(np.stack(rows), [0, V - 1, V // 2, 1, 2, 3, V - 1][: len(rows)], 1.0, False, 32)


@pytest.mark.parametrize("V", [30, 32000, 50000])
def test_masked_empty_and_invalid_rows(V):
    x, t = logits(12, V, V)
    x[0] = -np.inf                                         # nothing left
    x[1] = -np.inf
    x[1, V - 3] = -5.0                                     # one entry
    x[2, : V // 2] = -np.inf
    x[3] = np.finfo(np.float32).min                        # masked by the type's lowest value
    x[3, 7] = 1.0
    x[4, V // 3] = np.nan
    x[5, V // 3] = np.inf
    x[6, :] = np.finfo(np.float32).min
    t[2], t[7], t[8] = 0, -1, V                            # a masked token, two that are none
    x[9, :] = 3.0e38
    x[9, 5] = -3.0e38
    x[10] = -np.inf
    x[10, [1, V - 1]] = 2.5
    x[11, : V - 2] = -np.inf
    check(x, t, 1.0, False, 6)


def test_probabilities_that_are_none():
    V = 1000
    p = np.full((4, V), 1.0 / V, dtype=np.float32)
    p[0, 3], p[1, 999], p[2, 0] = -1e-30, np.nan, np.inf
    check(p, [1, 2, 3, 4], 1.0, True, 3)


@pytest.mark.parametrize("V", [12, 32000, 40000])
def test_probabilities_below_the_normal_range(V):
    rng = np.random.default_rng(V)
    p = np.full((3, V), 1.0 / V, dtype=np.float32)
    p[0, 5], p[0, 7] = 1e-45, 1e-39
    p[1] = np.exp2(-rng.integers(100, 148, V).astype(np.float64))
    p[2] = 0
    p[2, [1, 4]] = 1e-41, 1.0
    check(p, [5, 3, 1], 1.0, True, 4)


def test_optional_outputs_and_many_rows():
    spd = spd_mod()
    x, t = logits(300, 1111, 3)
    want, tol = reference(x, t, 1.0, False, 2)
    dx, dt = torch.from_numpy(x).cuda(), torch.from_numpy(t.astype(np.int32)).cuda()
    h = torch.empty(300, device="cuda")
    spd.spd_token_logprobs(dx, None, 1.0, 0, entropy_out=h)
    assert np.all(np.abs(h.cpu().numpy() - want["h"]) <= tol["h"])
    lp = torch.empty(300, device="cuda")
    spd.spd_token_logprobs(dx, dt, 1.0, 0, logprob_out=lp)
    assert np.all(np.abs(lp.cpu().numpy() - want["lp"]) <= tol["lp"])
    rank = torch.empty(300, dtype=torch.int32, device="cuda")
    spd.spd_token_logprobs(dx, dt, 1.0, 0, rank_out=rank)
    assert np.array_equal(rank.cpu().numpy(), want["rank"])
    ids, ilp = torch.empty((300, 2), dtype=torch.int32, device="cuda"), torch.empty((300, 2), device="cuda")
    spd.spd_token_logprobs(dx, None, 1.0, 0, top_tokens_out=ids, top_logprobs_out=ilp)
    assert np.array_equal(ids.cpu().numpy(), want["ids"])
    spd.spd_token_logprobs(dx, None, 1.0, 0)


@pytest.mark.parametrize("n,V", [(4, 32000), (3, 90001)])
def test_calls_on_two_streams_and_a_captured_call(n, V):
    spd = spd_mod()
    outs = []
    for i in range(2):
        x, t = logits(n, V, 50 + i)
        dx, dt = torch.from_numpy(x).cuda(), torch.from_numpy(t.astype(np.int32)).cuda()
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            ids, ilp = torch.empty((n, 9), dtype=torch.int32, device="cuda"), torch.empty((n, 9), device="cuda")
            lp = torch.empty(n, device="cuda")
            for _ in range(3):
                spd.spd_token_logprobs(dx, dt, 1.0, 0, lp, None, None, ids, ilp)
        outs.append((x, t, dx, dt, lp, ids))
    torch.cuda.synchronize()
    for x, t, _, _, lp, ids in outs:
        want, tol = reference(x, t, 1.0, False, 9)
        assert np.array_equal(ids.cpu().numpy(), want["ids"]) and np.all(np.abs(lp.cpu().numpy() - want["lp"]) <= tol["lp"])
    x, t, dx, dt = outs[0][:4]
    ws = torch.empty(max(1, spd.spd_logprobs_workspace_bytes(n, V, 9)), dtype=torch.uint8, device="cuda")
    ids, ilp, lp = torch.empty((n, 9), dtype=torch.int32, device="cuda"), torch.empty((n, 9), device="cuda"), torch.empty(n, device="cuda")
    spd.spd_token_logprobs(dx, dt, 1.0, 0, lp, None, None, ids, ilp, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spd.spd_token_logprobs(dx, dt, 1.0, 0, lp, None, None, ids, ilp, ws)
    for i in range(3):
        x, t = logits(n, V, 70 + i)
        dx.copy_(torch.from_numpy(x))
        dt.copy_(torch.from_numpy(t.astype(np.int32)))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        want, tol = reference(x, t, 1.0, False, 9)
        assert np.array_equal(ids.cpu().numpy(), want["ids"]) and np.all(np.abs(lp.cpu().numpy() - want["lp"]) <= tol["lp"])
        again = torch.empty_like(lp)
        spd.spd_token_logprobs(dx, dt, 1.0, 0, again)
        torch.cuda.synchronize()
        assert math.isfinite(float(again.sum()))
