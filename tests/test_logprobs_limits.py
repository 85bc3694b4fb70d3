"""Temperatures and sizes at the limits of the log probabilities' calls (refusals: no GPU work)."""
import ctypes

import numpy as np
import pytest

from tests.test_q4_logprobs_refusals import expect, f32, i32, lib, null, some, sz, u32


@pytest.mark.parametrize("temperature", [1e-45, 2.9e-39, 3.5e-39, 4.2e-39])
def test_temperatures_whose_exponents_have_no_factor(temperature):
    """2^((l - max) log2(e) / T): the factor is beyond float32 below T = 4.24e-39, also where 1 / T is not (2.94e-39)."""
    spd, _ = lib()
    expect(spd.SPD_ERR_INVALID_ARG, "spd_token_logprobs", some, sz(100), some, i32(2), i32(100), f32(temperature), u32(0), some, null, null, i32(0), null, null, null, sz(0), null)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [50, 32000, 40000])
@pytest.mark.parametrize("temperature", [4.3e-39, 1e-38, 1e38, 3.4e38])
def test_temperatures_next_to_the_limits(V, temperature):
    """Differences below 0.6: divided by T they stay finite."""
    from tests.test_gpu_logprobs import check
    rng = np.random.default_rng(V)
    x = (0.6 * rng.random((3, V)) - 0.3).astype(np.float32)
    x[1, [3, V - 1]] = 0.3                                     # two first ones
    check(x, [1, V - 1, V // 2], temperature, False, 4)


def test_sizes_that_the_call_refuses_have_no_workspace_either():
    spd, l = lib()
    n = ctypes.c_size_t()
    for rows, vocab in ((1, 2**24 + 1), (2**22, 5000), (2**21, 32769), (2**31 - 1, 2**24)):
        expect(spd.SPD_ERR_SHAPE, "spd_logprobs_workspace_bytes", i32(rows), i32(vocab), i32(1), ctypes.byref(n))
    for rows, vocab in ((2**22 - 1, 32768), (2**21 - 1, 32769), (1, 2**24)):
        assert l.spd_logprobs_workspace_bytes(i32(rows), i32(vocab), i32(1), ctypes.byref(n)) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("V", [40, 32000, 40000])
@pytest.mark.parametrize("temperature", [3.0, 200.0])
def test_differences_beyond_float32_that_the_temperature_brings_back(V, temperature):
    """Up to 6.8e38 below the largest entry: finite once divided by T."""
    from tests.test_gpu_logprobs import check
    x = np.zeros((2, V), dtype=np.float32)
    x[:, 5], x[:, 7:30] = 3.0e38, np.finfo(np.float32).min
    x[1, 6] = 3.0e38
    check(x, [7, 9], temperature, False, 32)
