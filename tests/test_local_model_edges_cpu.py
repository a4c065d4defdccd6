"""Host-side checks of extremes of a local step's operators (refusals before any CUDA call; fake but well-formed pointers)."""
import pytest

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
