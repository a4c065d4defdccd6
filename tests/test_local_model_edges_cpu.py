"""Host-side checks of extremes of a local step's operators (refusals before any CUDA call, with fake but well-formed pointers), and
what the 8-bit states' definition amounts to."""
import numpy as np
import pytest

import local_model_ref as ref

P = [0x10000000 * k for k in range(1, 15)]     # far apart


@pytest.fixture(scope="module")
def b():
    from paper_2507_20424_b200 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.mark.parametrize("temperature", [4e-39, 1e-39, 1e-42, 1e-45])
def test_policy_refuses_temperatures_whose_reciprocal_is_beyond_fp32(b, temperature):
    rc = b.load().dppf_policy_loss(P[0], 1, 8, 100, 104, P[1], 64, P[2], P[3], P[4], P[5], 0.2, 0.2, 0.1, temperature, P[6], P[7], P[8], 104, P[9], 1 << 27, None)
    assert rc == b.ERR_INVALID_ARG


@pytest.mark.parametrize("beta1,noise,low,high", [(0.9, 0.0, 1.7, 1.9), (0.95, 0.0, 3.2, 3.4), (0.99, 0.0, 2.5, 2.7), (0.9, 0.3, 0.97, 1.02), (0.95, 0.3, 1.05, 1.13), (0.99, 3.0, 0.95, 1.02)])
def test_first_moment_in_8_bits_lags_as_documented(beta1, noise, low, high):
    """What rounding to nearest does to a first moment whose gradients fall to 0.3: its median over the average that it stands for,
    in the sequence that the kernel reproduces bit for bit."""
    rng, n, steps = np.random.default_rng(0), 256 * 16, 200
    size = (np.exp(rng.normal(size=n)) * 1e-3).astype(np.float32)
    largest = np.zeros(n, bool)
    largest[ref.blocks_of(size).argmax(1) + 256 * np.arange(n // 256)] = True          # they keep their gradients, and so their block's scale
    codes, scales, want = [np.zeros(n, np.uint8)] * 2, [np.zeros(n // 256, np.float32)] * 2, np.zeros(n)
    for step in range(1, 2 * steps + 1):
        g = size * np.where((step > steps) & ~largest, np.float32(0.3), np.float32(1)) * (1 + noise * rng.normal(size=n)).astype(np.float32)
        mc, ms, rc, rs = ref.adamw8_states(g, codes[0], codes[1], scales[0], scales[1], beta1, 0.999, step)
        codes, scales, want = (mc, rc), (ms, rs), beta1 * want + (1 - beta1) * g
    median = np.median((ref.decode(codes[0], scales[0], n) / want)[~largest])
    assert low < median < high, median
