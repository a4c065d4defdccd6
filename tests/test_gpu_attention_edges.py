"""Attention on the GPU where values are not finite, large, or beyond 32 bits, and where a kernel gives up.

Tolerances are those of test_gpu_attention, and for the part of the exponentials that is a polynomial (2.9e-6 of the value at most, with the
roundings of its six operations 3.3e-6, where the others have 2 ulp): 3.3e-6 more for lse, and a hundredth more of the others, whose 2^-8
of each probability is above 500 times that.
"""
import math

import pytest
import torch

from gpu_util import require_gpu
from test_gpu_attention import BF16, inputs, randn, reference, same_bits, starts_of, within as within_half_steps

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def b():
    return require_gpu()[1]


def within(got, want, tol, what=""):
    within_half_steps(got, want, tol + 3.3e-6 if what == "lse" else tol * 1.01, what)


def rows_below(T, first):
    """[T, len(first)]: whether a row comes before first[h]."""
    return torch.arange(T, device="cuda")[:, None] < first


def check_rows(got, clean, spoiled, what):
    """Rows of got[T, heads, ...] are NaN throughout where spoiled[T, heads], and have clean's bits elsewhere."""
    assert torch.isnan(got[spoiled].float()).all(), what
    assert same_bits(got[~spoiled], clean[~spoiled]), what


# ---------------------------------------------------------------- NaN, one at a time in each place of a tile

def one_nan_a_head(t, first):
    """t[T, heads, D] with a NaN in one element of row first + h of head h."""
    t = t.clone()
    h = torch.arange(t.shape[1], device="cuda")
    t[first + h, h, 5] = NAN
    return t


@pytest.mark.parametrize("D", [32, 64, 88, 128])
@pytest.mark.parametrize("share", [1, 2])
@pytest.mark.parametrize("first", [0, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_a_nan_key_in_each_place_of_a_tile(b, D, share, first, causal):
    T, kv = 260, 128
    q, k, v = inputs(T, kv * share, kv, D, seed=1)
    plan = b.AttentionPlan(starts_of([T]), T)
    clean = b.dppf_attention(q, k, v, plan, causal=causal)
    grad_out = randn(q.shape, 2)
    bad = one_nan_a_head(k, first)
    got = b.dppf_attention(q, bad, v, plan, causal=causal)
    sees = ~rows_below(T, first + torch.arange(kv, device="cuda").repeat_interleave(share))
    if not causal:
        sees = torch.ones_like(sees)
    check_rows(got.out, clean.out, sees, "out")
    check_rows(got.lse.t(), clean.lse.t(), sees, "lse")
    own = b.dppf_attention_grad(grad_out, q, bad, v, got.out, got.lse, plan, causal=causal)
    assert torch.isnan(own.q[sees].float()).all()
    assert torch.isnan(own.k.float()).all() and torch.isnan(own.v.float()).all()       # the last query sees every key, and has no probabilities
    given = b.dppf_attention_grad(grad_out, q, bad, v, clean.out, clean.lse, plan, causal=causal)      # statistics that do not tell of it
    assert torch.isnan(given.q[sees].float()).all()


@pytest.mark.parametrize("D", [32, 64, 88, 128])
@pytest.mark.parametrize("share", [1, 2])
@pytest.mark.parametrize("first", [0, 128])
def test_a_nan_query_in_each_place_of_a_tile(b, D, share, first):
    T, heads = 260, 128
    q, k, v = inputs(T, heads, heads // share, D, seed=3)
    plan = b.AttentionPlan(starts_of([T]), T)
    clean = b.dppf_attention(q, k, v, plan)
    grad_out = randn(q.shape, 4)
    want = b.dppf_attention_grad(grad_out, q, k, v, clean.out, clean.lse, plan)
    bad = one_nan_a_head(q, first)
    own = torch.isnan(bad.float()).any(2)
    got = b.dppf_attention(bad, k, v, plan)
    check_rows(got.out, clean.out, own, "out")
    check_rows(got.lse.t(), clean.lse.t(), own, "lse")
    grads = b.dppf_attention_grad(grad_out, bad, k, v, clean.out, clean.lse, plan)
    check_rows(grads.q, want.q, own, "grad_q")
    seen = rows_below(T, first + torch.arange(heads, device="cuda").view(-1, share).amax(1) + 1)      # by the last of the heads' queries
    check_rows(grads.v, want.v, seen, "grad_v")
    assert torch.isnan(grads.k[seen].float()).all()


# ---------------------------------------------------------------- waits that give up in one kernel

@pytest.mark.parametrize("heads,kv_heads,D", [(4, 2, 128), (2, 2, 64), (8, 1, 72)])
def test_only_the_first_kernel_of_the_gradient_gives_up(b, heads, kv_heads, D):
    """It forms D_i as well as grad_q: what is made of the D that it did not form must not look like a gradient."""
    starts = starts_of([300, 20])
    T = 330                                                                     # the last ten of no sequence
    q, k, v = inputs(T, heads, kv_heads, D, seed=5)
    plan = b.AttentionPlan(starts, T)
    f = b.dppf_attention(q, k, v, plan)
    want = b.dppf_attention_grad(q, q, k, v, f.out, f.lse, plan)
    try:
        b.debug_set_poll_limits(-1, 0)
        got = b.dppf_attention_grad(q, q, k, v, f.out, f.lse, plan)
        assert b.dppf_device_status(plan.buffer) == b.ERR_TIMEOUT
    finally:
        b.debug_set_poll_limits(-1, -1)
    assert torch.isnan(got.q[:320].float()).all() and torch.isnan(got.k[:320].float()).all()
    assert same_bits(got.v, want.v) and not got.q[320:].any() and not got.k[320:].any()
    plan.renew(starts)
    again = b.dppf_attention_grad(q, q, k, v, f.out, f.lse, plan)
    assert all(same_bits(x, y) for x, y in zip(again, want)) and b.dppf_device_status(plan.buffer) == b.OK


# ---------------------------------------------------------------- large values under scores that rise

@pytest.mark.parametrize("heads,kv_heads,D", [(4, 2, 64), (3, 3, 128)])
@pytest.mark.parametrize("jump", [9.0, 16.0, 20.0, 41.0])                       # 13 to 59 powers of two
@pytest.mark.parametrize("offset", [0, 64])                                     # from tile to tile, or from half to half
@pytest.mark.parametrize("causal", [True, False])
def test_large_values_under_growing_scores(b, heads, kv_heads, D, jump, offset, causal):
    """Sums are kept relative to an older maximum for a while; what that multiplies the values by has to leave them finite.  700 keys: up to 2^98."""
    T = 700
    starts = starts_of([T])
    q, k, v = (x.clone() for x in inputs(T, heads, kv_heads, D, seed=7, std=0.3))
    q[..., 0] = 8.0
    k[..., 0] = ((torch.arange(T, device="cuda") + offset) // 128 * jump)[:, None].to(BF16)
    v = (v.float() * 2.0 ** 95).to(BF16)                                        # 0.3 * 2^95, and 1.6 * 2^95 = 2^95.7 the largest
    got = b.dppf_attention(q, k, v, b.AttentionPlan(starts, T), causal=causal, scale=0.125)
    want = reference(q, k, v, starts, causal, 0, 0.125)
    within(got.lse, *want["lse"], "lse")
    within(got.out, *want["out"], "out")
