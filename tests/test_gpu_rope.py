"""Rotary positions against 64 bits.

A sine or cosine: the place within the turn is cut to 2^-32 turns (1.5e-9), the remainder of an eighth of a turn rounded twice (2 * 0.79 units of
2^-24), the Taylor sum another unit and a half: 4 units; times the magnitude: 5.  A result: (|a| + |b|) m times those, one rounding of a product and one of
the difference: 8 units of (|a| + |b|) m.  bfloat16 outputs are rounded once more (2^-8)."""
import numpy as np
import pytest
import torch

from oracle import paged as op
from tests.paged_helpers import HALF, U, f64, spd_mod

pytestmark = pytest.mark.gpu


def make(spd, R, interleaved, scaling, theta=10000.0, magnitude=1.0, factors=None):
    kinds = {"none": 0, "linear": 1, "ramp": 2, "log_ramp": 3}
    args = {"factor": 6.5, "low": 1.0, "high": 30.0}
    rope = spd.Rope(R, theta=theta, interleaved=interleaved, scaling=kinds[scaling], original_positions=4096.0, magnitude=magnitude, factors=factors, **args)
    freq = op.frequencies(R, np.float32(theta), scaling, np.float32(6.5), 1.0, 30.0, 4096.0, None if factors is None else np.float32(factors))
    return rope, freq, float(np.float32(magnitude))


def check(x, out, positions, freq, m, interleaved, inverse):
    want = op.turned(f64(x), positions, freq, m, interleaved, inverse)
    n = len(freq)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    size = np.abs(f64(x))
    tol = np.zeros_like(want)
    # the reference's own angle: positions of up to 2^31 times a frequency in float64
    angle = np.abs(np.asarray(positions, np.float64))[:, None, None] * freq * 2.0 ** -52
    tol[..., a] = tol[..., b] = (size[..., a] + size[..., b]) * m * (8 * U + angle)
    if x.dtype == torch.bfloat16:
        tol[..., : 2 * n] += 2.0 ** -8 * np.abs(want[..., : 2 * n]) * (1 + 2.0 ** -8)
    off = np.abs(f64(out) - want)
    assert (off <= tol).all(), f"{(off / np.maximum(tol, 1e-300)).max():.2f} of the tolerance"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,heads,dim,R,interleaved,scaling,inverse", [
    (1, 1, 2, 2, False, "none", False), (1, 12, 64, 64, False, "none", False), (5, 32, 128, 128, False, "ramp", False), (3, 7, 80, 40, True, "log_ramp", True),
    (17, 3, 96, 96, False, "linear", True), (2, 5, 130, 66, True, "none", False), (9, 1, 256, 256, True, "ramp", False), (33, 2, 63, 30, False, "log_ramp", False),
    (257, 9, 128, 64, False, "none", False), (4, 2, 128, 8, True, "none", False), (4, 2, 128, 16, False, "none", False)])
def test_against_64_bits(dtype, rows, heads, dim, R, interleaved, scaling, inverse):
    spd = spd_mod()
    g = torch.Generator().manual_seed(rows * 1000 + dim)
    x = torch.randn((rows, heads, dim), generator=g).to(dtype)
    positions = torch.randint(0, 5000, (rows,), generator=g, dtype=torch.int32)
    rope, freq, m = make(spd, R, interleaved, scaling, magnitude=1.0 if R % 4 else 1.25)
    out = torch.full_like(x, 9.0, device="cuda")
    spd.spd_rope_apply(rope, x.cuda(), positions.cuda(), out, inverse=inverse)
    check(x, out, positions.tolist(), freq, m, interleaved, inverse)
    same = x.cuda()
    spd.spd_rope_apply(rope, same, positions.cuda(), same, inverse=inverse)
    assert torch.equal(same, out)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_and_negative_positions(interleaved):
    spd = spd_mod()
    positions = [0, 1, -1, 2**20 + 1, -(2**20), 2**31 - 1, -(2**31), 999983]
    x = torch.randn((len(positions), 3, 64), generator=torch.Generator().manual_seed(3))
    rope, freq, m = make(spd, 64, interleaved, "none")
    out = torch.empty_like(x, device="cuda")
    spd.spd_rope_apply(rope, x.cuda(), torch.tensor(positions, dtype=torch.int32).cuda(), out)
    check(x, out, positions, freq, m, interleaved, False)
    assert torch.equal(out[0].cpu(), x[0])


def test_factors_of_each_pair():
    spd = spd_mod()
    factors = [1.0 + 0.37 * i for i in range(16)]
    rope, freq, m = make(spd, 32, False, "linear", theta=500000.0, magnitude=0.75, factors=factors)
    x = torch.randn((6, 2, 64), generator=torch.Generator().manual_seed(4))
    positions = [3, 100, 70000, 5, 0, 12345]
    out = torch.empty_like(x, device="cuda")
    spd.spd_rope_apply(rope, x.cuda(), torch.tensor(positions, dtype=torch.int32).cuda(), out)
    check(x, out, positions, freq, m, False, False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_strided_rows_and_heads(dtype, pad):
    """Views into wider buffers, heads before rows, and nothing written beside the heads."""
    spd = spd_mod()
    g = torch.Generator().manual_seed(11 + pad)
    rows, heads, dim, R = 19, 4, 64, 32
    rope, freq, m = make(spd, R, False, "none")
    positions = torch.randint(0, 9000, (rows,), generator=g, dtype=torch.int32)
    wide = torch.randn((heads, rows, dim + pad), generator=g).to(dtype).cuda()
    x = wide.permute(1, 0, 2)[..., :dim]
    buffer = torch.full((rows, heads * dim + pad), 5.0, dtype=dtype, device="cuda")
    out = buffer[:, : heads * dim].unflatten(1, (heads, dim))
    spd.spd_rope_apply(rope, x, positions.cuda(), out)
    check(x, out, positions.tolist(), freq, m, False, False)
    assert (buffer[:, heads * dim :] == 5.0).all()
    if pad:
        before = wide[..., dim:].clone()
        spd.spd_rope_apply(rope, x, positions.cuda(), x)
        assert torch.equal(x, out) and torch.equal(wide[..., dim:], before)


def test_the_gradient_of_x_is_the_turn_back():
    """out = J x with J the turn: the inverse is J^T, by <y, J x> = <J^T y, x> in 64 bits of the float32 results, and against differences (the
    map is linear, so a difference of any width is the derivative, up to the roundings of both sides)."""
    spd = spd_mod()
    g = torch.Generator().manual_seed(5)
    rope, _, m = make(spd, 24, True, "ramp", magnitude=1.3)
    x, y, e = (torch.randn((7, 3, 40), generator=g).cuda() for _ in range(3))
    positions = torch.randint(0, 3000, (7,), generator=g, dtype=torch.int32).cuda()
    run = lambda t, back: (lambda o: (spd.spd_rope_apply(rope, t, positions, o, inverse=back), o)[1])(torch.empty_like(t))
    fwd, back = run(x, False), run(y, True)
    size = (y.double().abs().sum() * x.double().abs().max() + x.double().abs().sum() * y.double().abs().max()).item()
    assert abs((y.double() * fwd.double()).sum().item() - (back.double() * x.double()).sum().item()) <= 2 * 8 * U * m * 2 * size
    diff = (run(x + e, False).double() - fwd.double())
    # <y, J e>: x + e is rounded (U of it), both turns by 8 U of (|a| + |b|) m
    total = (y.double() * diff).sum().item()
    bound = (y.double().abs().sum() * (x.abs().max() + e.abs().max()).double() * 2 * m * 18 * U).item()
    assert abs(total - (back.double() * e.double()).sum().item()) <= bound


def test_turned_back_is_what_was():
    spd = spd_mod()
    rope, _, _ = make(spd, 128, False, "none")
    x = torch.randn((50, 8, 128), generator=torch.Generator().manual_seed(6)).cuda()
    positions = torch.arange(0, 50 * 1777, 1777, dtype=torch.int32).cuda()
    out, again = torch.empty_like(x), torch.empty_like(x)
    spd.spd_rope_apply(rope, x, positions, out)
    spd.spd_rope_apply(rope, out, positions, again, inverse=True)
    assert (again - x).abs().max().item() <= 2 * 8 * U * 4 * x.abs().max().item()


def test_values_that_are_not_finite_stay_with_their_pair():
    spd = spd_mod()
    rope, _, _ = make(spd, 32, False, "none")
    x = torch.randn((4, 2, 64), generator=torch.Generator().manual_seed(7))
    positions = torch.tensor([1, 2, 3, 4], dtype=torch.int32).cuda()
    clean, dirty = torch.empty_like(x, device="cuda"), torch.empty_like(x, device="cuda")
    spd.spd_rope_apply(rope, x.cuda(), positions, clean)
    y = x.clone()
    y[1, 0, 3], y[2, 1, 50] = float("nan"), float("inf")
    spd.spd_rope_apply(rope, y.cuda(), positions, dirty)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[1, 0, 3] = bad[1, 0, 19] = bad[2, 1, 50] = True
    assert torch.equal(dirty.cpu()[~bad], clean.cpu()[~bad])
    assert dirty[1, 0, 3].isnan() and dirty[1, 0, 19].isnan() and dirty[2, 1, 50] == float("inf")


def test_captured_and_on_another_stream():
    spd = spd_mod()
    rope, freq, m = make(spd, 64, False, "none")
    x = torch.randn((6, 5, 64), generator=torch.Generator().manual_seed(8)).cuda()
    positions = torch.arange(6, dtype=torch.int32).cuda()
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        spd.spd_rope_apply(rope, x, positions, out)
    for step in range(3):
        x.mul_(1.5)
        positions.add_(17)
        out.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        check(x, out, positions.tolist(), freq, m, False, False)
