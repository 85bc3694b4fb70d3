"""Long prompts of models in 4 bits: row counts where bf16 prompts take the other tile shape (whose sums of squares come in other parts), prompts of
more than one pass with rests below and above the shortest run that the prompt kernels take, every group size.  The scales are powers of two, so the
weights' values are bf16's as well: the same prompt through a bf16 model of those values is the reference."""
import numpy as np
import pytest
import torch

from paper_2404_08856_amd import synth
from tests.helpers import check_logits
from tests.test_gpu_prefill import SHAPES, cached

pytestmark = pytest.mark.gpu

WIDE, SMALL = SHAPES["wide"], SHAPES["small"]                  # d 4096 (O and down in the large shape from 1025 rows) and 128
LAYERS_7B = synth.ModelShape(2, 4096, 32, 128, 11008, 512)


def both_models(shape, group, capacity, seed):
    """(a model in 4 bits, a bf16 model of the same values): integers of 3 standard deviations' spread, scales 2^-8 and 2^-7: 0.018 an entry."""
    from paper_2404_08856_amd import spd
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    d, hd, F, V = shape.d_model, shape.n_heads * shape.head_dim, shape.d_ffn, shape.vocab

    def matrix(n, k):
        q = torch.clamp(torch.round(3 * torch.randn((n, k + k % 2), generator=g, device="cuda")), -8, 7).to(torch.int32) & 15
        q = (q[:, 0::2] | (q[:, 1::2] << 4)).to(torch.uint8)
        scales = torch.exp2(torch.randint(-8, -6, (n, (k + group - 1) // group), generator=g, device="cuda").float()).bfloat16()
        values = torch.empty((n, k), dtype=torch.bfloat16, device="cuda")
        spd.spd_q4_dequantize(q, scales, group, values)
        return (q, scales), values

    def gain():
        return 1 + 0.3 * torch.randn(d, generator=g, device="cuda")
    shapes = {"wq": (hd, d), "wk": (hd, d), "wv": (hd, d), "wo": (d, hd), "w_gate": (F, d), "w_up": (F, d), "w_down": (d, F)}
    head, head16 = matrix(V, d)
    embed = (0.02 * torch.randn((V, d), generator=g, device="cuda")).bfloat16()
    four = {"group": group, "embed": embed, "lm_head": head, "final_norm": gain(), "layers": []}
    plain = {"embed": embed, "lm_head": head16, "final_norm": four["final_norm"], "layers": []}
    for _ in range(shape.n_layers):
        gains = {"attn_norm": gain(), "mlp_norm": gain()}
        mats = {name: matrix(*s) for name, s in shapes.items()}
        four["layers"].append({**gains, **{k: v[0] for k, v in mats.items()}})
        plain["layers"].append({**gains, **{k: v[1] for k, v in mats.items()}})
    cfg = spd.make_config(shape, 1, capacity)
    return spd.Model(cfg, four), spd.Model(cfg, plain)


def check_rows(got, want, layer):
    """K or V of both models, bf16 values of float32 sums.  Layer 0: equal or one step apart (2^-7 at most), near zero the sums' own rounding.  Layer 1: a flipped
    step of one V component (2^-8 of up to 6) reaches early rows with a weight near 1, through Wo and Wk (0.018 an entry, 4096 columns): 5e-4 against
    values above 1, 2e-3 at four sigma, and through the MLP as well, up to 3 times that: 1e-2 with room for a second one.  All in all such flips
    are some in 10^4: a norm that is off by a part of its sums would be off by percents in every row."""
    err = np.abs(got - want)
    floor = (1e-5 if layer == 0 else 1e-2) * np.sqrt(np.mean(want * want))
    assert np.all(err <= np.maximum(2.0 ** -7 * np.abs(want), floor)), (layer, err.max())
    assert np.mean(err > 0) < 0.02 or layer > 0, (layer, np.mean(err > 0))
    assert np.linalg.norm(err) <= 1e-3 * np.linalg.norm(want), (layer, np.linalg.norm(err) / np.linalg.norm(want))


@pytest.mark.parametrize("shape,group,parts", [
    (WIDE, 32, (1024,)), (WIDE, 128, (1025,)), (WIDE, 64, (2048,)), (WIDE, 64, (2048 + 55,)), (WIDE, 32, (2048 + 56,)), (WIDE, 128, (1100, 1037)),
    (SMALL, 32, (2048 + 24,)), (SMALL, 64, (2048 + 25, 70)), (SMALL, 128, (2 * 2048 + 300,)), (LAYERS_7B, 128, (2048 + 640,)), (LAYERS_7B, 32, (1280,)),
])
def test_long_prompts_against_a_bf16_model_of_the_same_values(shape, group, parts):
    n = sum(parts)
    print(f"4-bit prompt {shape.d_model} x {shape.d_ffn}, groups of {group}, {parts}", flush=True)
    models = both_models(shape, group, n + 8, 7 + n)
    rows = torch.from_numpy(synth.image_rows(n, shape.d_model, 8)).cuda()
    toks = torch.from_numpy(synth.text_tokens(5, shape.vocab, 9)).cuda()[None].contiguous()
    seen = []
    for m in models:
        logits, at = [], 0
        for part in parts:
            last = torch.empty(shape.vocab, device="cuda")
            m.spd_prefill(0, rows[at:at + part].contiguous(), last)
            logits.append(last.cpu().numpy())
            at += part
        out = torch.empty((1, 5, shape.vocab), device="cuda")
        m.spd_verify_forward(toks, out)
        logits.append(out[0].cpu().numpy())
        assert m.spd_kv_get_len(1) == [n + 5]
        seen.append((logits, [cached(m, l, n + 5, shape) for l in range(shape.n_layers)]))
        m.close()
    for i, (a, b) in enumerate(zip(seen[0][0], seen[1][0])):
        check_logits(a, b, f"part {i}")
    for layer, (a, b) in enumerate(zip(seen[0][1], seen[1][1])):
        for got, want in zip(a, b):
            check_rows(got.astype(np.float64), want.astype(np.float64), layer)
