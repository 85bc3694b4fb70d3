"""Products with 4-bit weights at the ends of their documented ranges: small and large activations together with small and large scales, in the
kernels of few and of many rows."""
import numpy as np
import pytest
import torch

from tests.test_gpu_q4 import device_matrix, spd_mod, to_bf16, values

pytestmark = pytest.mark.gpu

# every way that rows are taken: one, up to 4, 5, up to 8, 12, 16 (digits kept and made anew), and the kernel of many rows
SIZES = [(1, 33, 1000, 32), (1, 48, 11008, 128), (3, 40, 700, 64), (4, 33, 8200, 64), (5, 40, 4500, 128), (5, 4100, 130, 32), (8, 64, 2000, 64), (12, 64, 384, 64), (16, 48, 2000, 32),
         (40, 528, 4096, 128), (64, 31, 17000, 32)]


def product(q, scales, G, x):
    y = torch.full((x.shape[0], q.shape[0]), -1.0, device="cuda")
    spd_mod().spd_q4_matmul(device_matrix(q, scales, G), torch.from_numpy(x.astype(np.float32)).cuda(), y)
    return y.double().cpu().numpy()


@pytest.mark.parametrize("rows,N,K,G", SIZES)
@pytest.mark.parametrize("px,ps", [(-64, -60), (-84, -40), (-38, -86), (-86, 86), (88, -88), (60, 40), (14, 86)])
def test_integers_times_powers_of_two_on_both_sides_are_exact(rows, N, K, G, px, ps):
    """Integers up to 15 times 2^px, scales 2^ps times 1/4 to 2: every sum is a multiple of 2^(px + ps - 2) below 2^22 * 2^(px + ps)
    (15 * 8 * 2 * 17000 < 2^22), 24 bits that a normal float32 has where px + ps - 2 >= -126."""
    rng = np.random.default_rng(rows + K + px)
    x = rng.integers(-15, 16, (rows, K)) * 2.0 ** px
    q = rng.integers(-8, 8, (N, K))
    scales = np.exp2(rng.integers(-2, 2, (N, (K + G - 1) // G)) + float(ps)).astype(np.float32)
    assert np.array_equal(product(q, scales, G, x), x @ values(q, scales, G).T)


@pytest.mark.parametrize("rows,N,K,G", SIZES)
@pytest.mark.parametrize("px,ps", [(-60, -54), (-80, -34), (-34, -80), (50, 50)])
def test_small_activations_and_scales_within_their_roundings(rows, N, K, G, px, ps):
    """Against 64 bits.  Roundings: digits leave out at most 2^-29 of a row's largest magnitude or 2^-23 of an entry; a group's integer sum rounds
    four times until it is in the output's sum, which is one of groups + 20 numbers: additions of 2^-24 of a sum of magnitudes each (the
    digits' are at most those and 2^-6 of the largest).  Results that come near 2^-126 round by 2^-150 an addition."""
    rng = np.random.default_rng(3 * rows + K - px)
    x = (rng.standard_normal((rows, K)) * 2.0 ** px).astype(np.float32).astype(np.float64)
    groups = (K + G - 1) // G
    q = np.clip(np.rint(rng.standard_normal((N, K)) * 3), -8, 7).astype(np.int64)
    scales = to_bf16(2.0 ** ps * (0.5 + rng.random((N, groups))))
    w = values(q, scales, G)
    top = np.max(np.abs(x), axis=1, keepdims=True)
    mass, weight = np.abs(x) @ np.abs(w).T, np.sum(np.abs(w), axis=1)[None]
    tol = (groups + 24) * (2.0 ** -24 * (mass + 2.0 ** -6 * top * weight) + 2.0 ** -150) + 2.0 ** -29 * top * weight
    assert np.all(np.abs(product(q, scales, G, x) - x @ w.T) <= tol)


@pytest.mark.parametrize("rows,N,K,G", SIZES)
def test_integers_beside_a_column_2_29_times_as_large_are_exact(rows, N, K, G):
    """An entry counts to 2^-29 of the largest magnitude of its row: integers stay whole beside 2^29.  Its own weights are 0, so the sums are those
    of integers up to 15 (below 2^22)."""
    rng = np.random.default_rng(5 * rows + K)
    x = rng.integers(-15, 16, (rows, K)).astype(np.float64)
    q = rng.integers(-8, 8, (N, K))
    x[:, 77::128], q[:, 77::128] = 2.0 ** 29, 0
    scales = np.exp2(rng.integers(-2, 2, (N, (K + G - 1) // G))).astype(np.float32)
    assert np.array_equal(product(q, scales, G, x), x @ values(q, scales, G).T)


@pytest.mark.parametrize("rows,N,K,G", SIZES)
@pytest.mark.parametrize("px,ps", [(-26, -98), (20, -98), (-86, 99), (-30, 99), (2, 99)])
def test_scales_up_to_2_100_and_down_to_2_minus_100(rows, N, K, G, px, ps):
    """As the integers above: sums below 2^22 * 2^(px + ps), multiples of 2^(px + ps - 2) >= 2^-126."""
    test_integers_times_powers_of_two_on_both_sides_are_exact(rows, N, K, G, px, ps)
