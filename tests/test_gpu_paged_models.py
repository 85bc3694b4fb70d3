"""Models over pages: trees whose branches are committed, and pages in 8 bits, against the oracle."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import decoder as dec
from oracle import paged as op
from paper_2404_08856_amd import synth
from tests.helpers import LOGIT_MAX_ABS, check_logits, oracle_cfg, randomize_gains, to_device
from tests.paged_helpers import f64, spd_mod
from tests.test_gpu_paged_run import SHAPES, pages_of

pytestmark = pytest.mark.gpu


def model_of(spd, shape, seed):
    w = randomize_gains(synth.make_weights(shape, seed))
    return spd.Model(spd.make_config(shape, 1, 32), to_device(w)), synth.weights_to_numpy(w)


@pytest.mark.parametrize("second", [False, True])
def test_a_branch_of_a_tree_is_committed(second):
    """t with continuations a and b, of which one is accepted.  The first lies behind t: the length takes it.  The other's tokens go again, as the first rows of the next block."""
    spd = spd_mod()
    shape = SHAPES[0]
    model, wn = model_of(spd, shape, 25)
    cfg = oracle_cfg(shape)
    layers, table = pages_of(spd, shape, 1, 96)
    rope = spd.Rope(shape.head_dim, theta=shape.rope_theta)
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(tokens, positions=None, seen=None):
        logits = torch.empty((len(tokens), shape.vocab), device="cuda")
        on = [None if x is None else torch.tensor(x, dtype=t, device="cuda") for x, t in ((positions, torch.int32), (seen, torch.int64))]
        model.spd_verify_forward_paged(torch.tensor(tokens, dtype=torch.int32, device="cuda"), layers, spd.PagedBatch(table, lens, len(tokens)), rope, logits, *on)
        return logits.cpu().numpy()
    prompt = synth.text_tokens(20, shape.vocab, 1).tolist()
    step(prompt)
    lens += 20
    t, a, b, more = synth.text_tokens(1, shape.vocab, 2).tolist(), [7, 11], [13, 17, 19], [23, 29]
    step(t + a + b, [20, 21, 22, 21, 22, 23], [0b1, 0b11, 0b111, 0b1001, 0b11001, 0b111001])
    lens += 1 if second else 3                             # of slots 20 .. 25: t; t and a
    new = b + more if second else more
    logits = step(new)
    cache = dec.KVCache(cfg, 64)
    dec.forward_tokens(cfg, wn, cache, np.array(prompt + t + ([] if second else a), np.int32))
    check_logits(logits, dec.forward_tokens(cfg, wn, cache, np.array(new, np.int32)), f"behind branch {'b' if second else 'a'}")


def test_trees_have_positions():
    """Branches share positions, which only the caller knows."""
    spd = spd_mod()
    shape = SHAPES[0]
    model, _ = model_of(spd, shape, 26)
    layers, table = pages_of(spd, shape, 1, 96)
    batch = spd.PagedBatch(table, torch.zeros(1, dtype=torch.int32, device="cuda"), 3)
    tokens, seen = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.tensor([1, 3, 5], dtype=torch.int64, device="cuda")
    logits = torch.full((3, shape.vocab), 7.0, device="cuda")
    with pytest.raises(spd.SpdError) as e:
        model.spd_verify_forward_paged(tokens, layers, batch, spd.Rope(shape.head_dim), logits, seen=seen)
    assert e.value.code == spd.SPD_ERR_INVALID_ARG and (logits == 7.0).all() and all((c.k == 0).all() for c in layers)


class Held:
    """Keys or values of a sequence as the pages hold them, in the place of the oracle's, which it only notes."""

    def __init__(self, values):
        self.values, self.noted, self.shape = values, {}, values.shape

    def __setitem__(self, at, x):
        self.noted[at[0]] = x

    def __getitem__(self, at):
        return self.values[at]


@pytest.mark.parametrize("shape", SHAPES[:2])
def test_models_over_8_bit_pages(shape):
    """Scales of their own for each layer and head, of keys and of values.  The oracle reads the keys and values that the pages hold: logits as always; and what they hold
    is what the oracle would have put there, rounded to e4m3 (from activations that are a tenth as far off as logits may be)."""
    spd = spd_mod()
    model, wn = model_of(spd, shape, 27)
    cfg = dataclasses.replace(oracle_cfg(shape), kv_bf16=False)
    seqs, capacity, P, H = 2, 96, 16, shape.n_heads
    layers, table = pages_of(spd, shape, seqs, capacity, P, is_e4m3=True)
    for l, c in enumerate(layers):
        scales = 0.015 * (1 + l) + 0.004 * torch.arange(2 * H, dtype=torch.float32).view(2, H)
        layers[l] = spd.PagedCache(c.k, c.v, scales[0].cuda(), scales[1].cuda())
    rope = spd.Rope(shape.head_dim, theta=shape.rope_theta)
    lens, seed, slack = [0] * seqs, 0, LOGIT_MAX_ABS / 10
    on = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    for new in ([38, 21], [5, 1], [4, 4]):
        toks = [synth.text_tokens(n, shape.vocab, seed + s) for s, n in enumerate(new)]
        seed += 10
        start = torch.tensor([0, new[0], sum(new)], dtype=torch.int32)
        logits = torch.empty((sum(new), shape.vocab), device="cuda")
        model.spd_verify_forward_paged(torch.from_numpy(np.concatenate(toks)).cuda(), layers, spd.PagedBatch(table, on, sum(new), start.cuda()), rope, logits)
        k_pages, v_pages = [f64(c.k) for c in layers], [f64(c.v) for c in layers]
        k_scale, v_scale = [f64(c.k_scale)[:, None] for c in layers], [f64(c.v_scale)[:, None] for c in layers]
        for s in range(seqs):
            places = [op.place(table.cpu().numpy(), layers[0].n_pages, P, s, p) for p in range(lens[s] + new[s])]
            cache = dec.KVCache(cfg, lens[s] + new[s])
            cache.k = Held(np.stack([np.stack([np.stack([op.key_at(k, page, h, slot) for h in range(H)]) * scale for page, slot in places]) for k, scale in zip(k_pages, k_scale)]))
            cache.v = Held(np.stack([np.stack([np.stack([op.value_at(v, page, h, slot) for h in range(H)]) * scale for page, slot in places]) for v, scale in zip(v_pages, v_scale)]))
            cache.length = lens[s]
            check_logits(logits[start[s] : start[s + 1]].cpu().numpy(), dec.forward_tokens(cfg, wn, cache, toks[s]), f"sequence {s}, rows {new}")
            for held, scales in ((cache.k, k_scale), (cache.v, v_scale)):
                for l in range(shape.n_layers):
                    want, got = held.noted[l], held.values[l, lens[s] :]
                    limited = np.clip(want, -448 * scales[l], 448 * scales[l])
                    # half a step of e4m3, of its smallest values 2^-10
                    assert (np.abs(got - limited) <= np.maximum(2.0 ** -4 * (np.abs(limited) + slack), 2.0 ** -10 * scales[l]) + slack).all()
        lens = [a + b for a, b in zip(lens, new)]
        on.copy_(torch.tensor(lens, dtype=torch.int32))
