"""Sizes that a 32- or 64-bit integer does not hold are refused by the binding: ctypes would pass their low bits on."""
import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2507_20424_b200 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.mark.parametrize("T,H", [(8, 2 ** 32 + 8), (2 ** 64 + 8, 8), (8, 8 - 2 ** 32)])
def test_workspaces(b, T, H):
    with pytest.raises(ValueError):
        b.alloc_layer_norm_workspace(T, H, device="cpu")
    with pytest.raises(ValueError):
        b.alloc_attention_workspace(T, H, device="cpu")


@pytest.mark.parametrize("bad", [dict(turned=2 ** 32 + 8), dict(turned=-2 ** 32 + 8), dict(scaling="by parts", factor=2.0, original_length=2 ** 64 + 4096)])
def test_rotary_frequencies(b, bad):
    with pytest.raises(ValueError):
        b.rotary_frequencies(**{"turned": 64, "device": "cpu", **bad})


def test_windows(b):
    """One that is longer than any batch is passed on as the longest; a negative one stays negative, for the C entry to refuse."""
    assert [b._window(n) for n in (0, 5, 2 ** 31 - 1, 2 ** 31, 2 ** 32 + 5, 2 ** 80)] == [0, 5] + [2 ** 31 - 1] * 4
    assert all(b._window(n) < 0 for n in (-1, -2 ** 31, 5 - 2 ** 32, -2 ** 80))
