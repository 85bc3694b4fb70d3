"""The paged cache as a program uses it: appended to and read by turns, and by whole models."""
import numpy as np
import pytest
import torch

from oracle import decoder as dec
from oracle import paged as op
from paper_2404_08856_amd import synth
from tests.helpers import check_logits, oracle_cfg, randomize_gains, to_device
from tests.paged_helpers import HALF, U, f64, spd_mod
from tests.test_gpu_q4_model import q4_model

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,is_e4m3", [(torch.float32, False), (torch.bfloat16, False), (torch.bfloat16, True)])
def test_prompts_then_tokens(dtype, is_e4m3):
    """Prompts in pieces, then blocks with a step back after each, four queries a key head, stretched positions: every output against 64 bits on what the
    pages hold, every page against the keys and values that went in."""
    spd = spd_mod()
    g = torch.Generator().manual_seed(31)
    seqs, H, HK, D, P, capacity = 3, 8, 2, 64, 16, 160
    ks, vs = spd.paged_cache_shapes(seqs * capacity // P + 1, P, HK, D, is_e4m3)
    t8 = lambda s: torch.zeros(s, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    cache = spd.PagedCache(t8(ks), t8(vs), torch.full((HK,), 0.02).cuda(), torch.full((HK,), 0.015).cuda()) if is_e4m3 else \
        spd.PagedCache(torch.zeros(ks, dtype=torch.bfloat16, device="cuda"), torch.zeros(vs, dtype=torch.bfloat16, device="cuda"))
    scales = ([f64(cache.k_scale), f64(cache.v_scale)] if is_e4m3 else [np.ones(HK), np.ones(HK)])
    table = torch.randperm(seqs * capacity // P, generator=g).int().view(seqs, -1)
    rope = spd.Rope(D, scaling=spd.SPD_ROPE_RAMP, factor=4.0, low=1.0, high=4.0, original_positions=64.0)
    freq = op.frequencies(D, 10000.0, "ramp", 4.0, 1.0, 4.0, 64.0)
    lens = [0] * seqs
    keys = [np.zeros((capacity, HK, D)) for _ in range(seqs)]
    values = [np.zeros((capacity, HK, D)) for _ in range(seqs)]
    dl = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    for new, back in [([70, 5, 33], 0), ([20, 40, 0], 0), ([1, 1, 1], 0), ([5, 5, 5], 3), ([5, 5, 5], 1), ([1, 1, 1], 0)]:
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        rows = int(start[-1])
        qkv = torch.randn((rows, H + 2 * HK, D), generator=g).to(dtype)
        on = qkv.cuda()
        q, k, v = on.split([H, HK, HK], 1)
        batch = spd.PagedBatch(table.cuda(), dl, rows, torch.from_numpy(start).cuda())
        spd.spd_paged_append(cache, batch, k, v, rope=rope, q=q, q_out=q)
        out, lse = torch.empty((rows, H, D), dtype=dtype, device="cuda"), torch.empty((rows, H), device="cuda")
        spd.spd_paged_attention(cache, batch, q, out, lse_out=lse)
        torch.cuda.synchronize()
        for s in range(seqs):
            for i in range(new[s]):
                r = start[s] + i
                keys[s][lens[s] + i] = op.turned(f64(qkv[r : r + 1, H : H + HK]), [lens[s] + i], freq)[0] / scales[0][:, None]
                values[s][lens[s] + i] = f64(qkv[r, H + HK :]) / scales[1][:, None]
        held_k, held_v = f64(cache.k), f64(cache.v)
        half, least = (2.0 ** -4, 2.0 ** -10) if is_e4m3 else (2.0 ** -8, 0.0)
        for s in range(seqs):
            for p in range(lens[s] + new[s]):
                page, slot = op.place(table.numpy(), cache.n_pages, P, s, p)
                for h in range(HK):
                    # the turn's 8 units of two elements (of at most 5.5, over the scale), the quotient's and the type's rounding
                    got, want = op.key_at(held_k, page, h, slot), np.clip(keys[s][p][h], -448, 448)
                    assert (np.abs(got - want) <= np.maximum(half * np.abs(want), least) * 1.01 + 11 * 10 * U / scales[0][h]).all()
                    got, want = op.value_at(held_v, page, h, slot), np.clip(values[s][p][h], -448, 448)
                    assert (np.abs(got - want) <= np.maximum(half * np.abs(want), least) * 1.01 + 1e-6 * np.abs(want)).all()
        want, want_lse, work, spread, count = op.attention(f64(q), held_k, held_v, table.numpy(), lens, start.tolist(), D ** -0.5, 0, None, *(scales if is_e4m3 else (None, None)))
        d = (D + 24) * U * work
        rel = 2 * d + (count[:, None] / 16 + 100) * U + (2.0 ** -8 if dtype == torch.bfloat16 else 0)
        assert (np.abs(f64(out) - want) <= spread * rel[..., None] * 1.01 + HALF[dtype] * np.abs(want)).all()
        assert (np.abs(f64(lse) - want_lse) <= d + (count[:, None] / 16 + 100) * U + 2 * U * np.abs(want_lse)).all()
        lens = [a + b - (back if b else 0) for a, b in zip(lens, new)]
        dl.copy_(torch.tensor(lens, dtype=torch.int32))


def pages_of(spd, shape, seqs, capacity, page_size=16, is_e4m3=False):
    ks, vs = spd.paged_cache_shapes(seqs * capacity // page_size + 1, page_size, shape.n_heads, shape.head_dim, is_e4m3)
    if is_e4m3:
        one = lambda s: torch.zeros(s, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        scale = torch.full((shape.n_heads,), 0.02, device="cuda")
        layers = [spd.PagedCache(one(ks), one(vs), scale, scale) for _ in range(shape.n_layers)]
    else:
        one = lambda s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
        layers = [spd.PagedCache(one(ks), one(vs)) for _ in range(shape.n_layers)]
    table = torch.randperm(seqs * capacity // page_size, generator=torch.Generator().manual_seed(5)).int().view(seqs, -1).cuda()
    return layers, table


SHAPES = [synth.SHAPES["tiny_target"], synth.ModelShape(2, 256, 2, 128, 680, 512), synth.ModelShape(2, 4096, 32, 128, 11008, 512)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("q4", [False, True])
def test_models_over_pages(shape, q4):
    """Prompts of different lengths, ragged verify blocks, blocks without row_start: logits against the oracle, sequence by sequence."""
    spd = spd_mod()
    seqs = 3
    if q4:
        model, wn = q4_model(shape, 21, 128, 1, 32)
    else:
        w = randomize_gains(synth.make_weights(shape, 21))
        wn = synth.weights_to_numpy(w)
        model = spd.Model(spd.make_config(shape, 1, 32), to_device(w))           # (the model's own cache is smaller than what the pages hold)
    cfg = oracle_cfg(shape)
    layers, table = pages_of(spd, shape, seqs, 96)
    rope = spd.Rope(shape.head_dim, theta=shape.rope_theta)
    caches, lens = [dec.KVCache(cfg, 128) for _ in range(seqs)], torch.zeros(seqs, dtype=torch.int32, device="cuda")
    seed = 0
    for new in ([38, 3, 21], [5, 0, 1], [4, 4, 4], [1, 1, 1]):
        toks = [synth.text_tokens(n, shape.vocab, seed + s) if n else np.zeros(0, np.int32) for s, n in enumerate(new)]
        seed += 10
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        uniform = len(set(new)) == 1
        extra = 0 if uniform else 2                        # rows of nobody behind the last sequence
        batch = spd.PagedBatch(table, lens, int(start[-1]) + extra, None if uniform else torch.from_numpy(start).cuda())
        tokens = torch.from_numpy(np.concatenate(toks + [np.zeros(extra, np.int32)]).astype(np.int32)).cuda()
        logits = torch.empty((batch.n_rows, shape.vocab), device="cuda")
        model.spd_verify_forward_paged(tokens, layers, batch, rope, logits)
        lens += torch.tensor(new, dtype=torch.int32, device="cuda")
        for s in range(seqs):
            if new[s]:
                check_logits(logits[start[s] : start[s + 1]].cpu().numpy(), dec.forward_tokens(cfg, wn, caches[s], toks[s]), f"sequence {s}, rows {new}")


def test_a_tree_of_drafted_tokens_is_its_branches():
    """t with two drafted continuations of two and three tokens: each branch's logits are those of that branch verified alone."""
    spd = spd_mod()
    shape = SHAPES[0]
    w = randomize_gains(synth.make_weights(shape, 22))
    wn, cfg = synth.weights_to_numpy(w), oracle_cfg(shape)
    model = spd.Model(spd.make_config(shape, 1, 32), to_device(w))
    layers, table = pages_of(spd, shape, 1, 96)
    rope = spd.Rope(shape.head_dim, theta=shape.rope_theta)
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    prompt = synth.text_tokens(20, shape.vocab, 1)
    logits = torch.empty((20, shape.vocab), device="cuda")
    model.spd_verify_forward_paged(torch.from_numpy(prompt).cuda(), layers, spd.PagedBatch(table, lens, 20), rope, logits)
    lens += 20
    t, a, b = [int(x) for x in synth.text_tokens(1, shape.vocab, 2)], [7, 11], [13, 17, 19]
    tokens = torch.tensor(t + a + b, dtype=torch.int32, device="cuda")
    seen = torch.tensor([0b1, 0b11, 0b111, 0b1001, 0b11001, 0b111001], dtype=torch.int64, device="cuda")
    positions = torch.tensor([20, 21, 22, 21, 22, 23], dtype=torch.int32, device="cuda")
    logits = torch.empty((6, shape.vocab), device="cuda")
    model.spd_verify_forward_paged(tokens, layers, spd.PagedBatch(table, lens, 6), rope, logits, positions, seen)
    for branch, rows in ((t + a, [0, 1, 2]), (t + b, [0, 3, 4, 5])):
        cache = dec.KVCache(cfg, 64)
        dec.forward_tokens(cfg, wn, cache, prompt)
        check_logits(logits[rows].cpu().numpy(), dec.forward_tokens(cfg, wn, cache, np.array(branch, np.int32)), f"branch {branch}")


def test_models_over_8_bit_pages_and_captured():
    """The step captured once and replayed with other tokens and lengths gives the eager step's bits."""
    spd = spd_mod()
    shape = SHAPES[0]
    model = spd.Model(spd.make_config(shape, 1, 32), to_device(randomize_gains(synth.make_weights(shape, 23))))
    layers, table = pages_of(spd, shape, 2, 96, is_e4m3=True)
    rope = spd.Rope(shape.head_dim, theta=shape.rope_theta)
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    batch = spd.PagedBatch(table, lens, 10)
    tokens = torch.from_numpy(synth.text_tokens(10, shape.vocab, 3)).cuda()
    ws = torch.full((1 << 26,), 255, dtype=torch.uint8, device="cuda")
    eager, captured = torch.empty((10, shape.vocab), device="cuda"), torch.empty((10, shape.vocab), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        model.spd_verify_forward_paged(tokens, layers, batch, rope, captured, workspace=ws)
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        model.spd_verify_forward_paged(tokens, layers, batch, rope, eager, workspace=ws)          # (the same places again)
        torch.cuda.synchronize()
        assert torch.equal(captured, eager) and torch.isfinite(eager).all()
        lens += 4
        tokens.add_(17).remainder_(shape.vocab)


def test_refusals_of_models_over_pages():
    spd = spd_mod()
    shape = SHAPES[0]
    model = spd.Model(spd.make_config(shape, 1, 32), to_device(synth.make_weights(shape, 24)))
    layers, table = pages_of(spd, shape, 1, 96)
    rope = spd.Rope(shape.head_dim)
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")

    def refused(code, layers=layers, rows=5, rope=rope, ws=None):
        tokens, logits = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.empty((rows, shape.vocab), device="cuda")
        with pytest.raises(spd.SpdError) as e:
            model.spd_verify_forward_paged(tokens, layers, spd.PagedBatch(table, lens, rows), rope, logits, workspace=ws)
        assert e.value.code == code
    other, _ = pages_of(spd, synth.ModelShape(2, 256, 2, 64, 688, 1024), 1, 96)
    refused(spd.SPD_ERR_SHAPE, layers=[layers[0], other[1]])
    wide, _ = pages_of(spd, shape, 1, 96, 32)
    refused(spd.SPD_ERR_SHAPE, layers=[layers[0], wide[1]])
    refused(spd.SPD_ERR_SHAPE, rows=65)
    refused(spd.SPD_ERR_SHAPE, rope=spd.Rope(shape.head_dim + 2))
    refused(spd.SPD_ERR_CAPACITY, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("new", [[1, 3], [150, 9]])
def test_offsets_beyond_32_bits(new):
    """Pages of 512 KiB behind the first 4 GiB: append and attention there give the bits that they give in the first pages."""
    spd = spd_mod()
    HK, D, P, H, n_pages = 8, 128, 256, 16, 8600
    ks, vs = spd.paged_cache_shapes(n_pages, P, HK, D)
    cache = spd.PagedCache(torch.empty(ks, dtype=torch.bfloat16, device="cuda"), torch.empty(vs, dtype=torch.bfloat16, device="cuda"))
    assert cache.k.numel() * 2 > 1 << 32
    g = torch.Generator().manual_seed(6)
    rows, lens = sum(new), torch.tensor([700, 90], dtype=torch.int32).cuda()
    start = torch.tensor([0, new[0], rows], dtype=torch.int32).cuda()
    qkv = torch.randn((rows, H + 2 * HK, D), generator=g).bfloat16().cuda()
    old = torch.randn((790, 2, HK, D), generator=g).bfloat16().cuda()
    rope, results = spd.Rope(D), []
    for first in (0, n_pages - 8):
        table = torch.arange(first, first + 8, dtype=torch.int32).view(2, 4).flip(0).contiguous().cuda()
        for s, (a, b) in enumerate(((0, 700), (700, 790))):
            spd.spd_paged_append(cache, spd.PagedBatch(table[s : s + 1], torch.zeros(1, dtype=torch.int32, device="cuda"), b - a), old[a:b, 0], old[a:b, 1])
        q, k, v = qkv.split([H, HK, HK], 1)
        turned, out, lse = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty((rows, H, D), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, H), device="cuda")
        batch = spd.PagedBatch(table, lens, rows, start)
        spd.spd_paged_append(cache, batch, k, v, rope=rope, q=q, q_out=turned)
        spd.spd_paged_attention(cache, batch, turned, out, lse_out=lse)
        results.append((turned, out, lse, cache.k[first : first + 8].clone(), cache.v[first : first + 8].clone()))
    torch.cuda.synchronize()
    for x, y in zip(*[r[:3] for r in results]):
        assert torch.equal(x, y) and torch.isfinite(x).all()
    for page in (4, 5):                                    # two that the first sequence fills
        assert torch.equal(results[0][3][page], results[1][3][page]) and torch.equal(results[0][4][page], results[1][4][page])
