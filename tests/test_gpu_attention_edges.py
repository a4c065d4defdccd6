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


# ---------------------------------------------------------------- how far a row that is not finite reaches

MASKS = [(True, 0), (False, 0), (True, 1), (True, 100), (True, 300)]


def reach(T, at, causal, window):
    """Two masks over a sequence's rows: those that see key `at`, and those whose tile of 128 holds one that sees a key of `at`'s tile."""
    i = torch.arange(T, device="cuda")
    gap = i[:, None] - i
    seen = torch.ones(T, T, dtype=torch.bool, device="cuda")
    if causal:
        seen &= gap >= 0
    if window:
        seen &= gap < window
    tiles = torch.zeros(T, T, dtype=torch.bool, device="cuda")
    for r in range(0, T, 128):
        for c in range(0, T, 128):
            tiles[r:r + 128, c:c + 128] = seen[r:r + 128, c:c + 128].any()
    return seen, tiles


def placed(mask, lead, T):
    """mask as one over the T rows of a batch, its first row being row `lead`."""
    out = torch.zeros(T, dtype=torch.bool, device="cuda")
    out[lead:lead + len(mask)] = mask
    return out


def check_reach(got, clean, sure, may, what):
    """[T, heads, D]: NaN in `sure` rows (of column 5 alone where only that can be), clean's bits outside of `may`."""
    assert torch.isnan(got[sure][..., 5].float()).all(), what
    assert same_bits(got[~may], clean[~may]), what


@pytest.mark.parametrize("causal,window", MASKS)
@pytest.mark.parametrize("heads,kv_heads,D", [(4, 2, 64), (2, 1, 128), (3, 3, 72)])
@pytest.mark.parametrize("at", [0, 130, 200, 255, 256, 599])
@pytest.mark.parametrize("value", [NAN, float("inf")])
def test_how_far_rows_that_are_not_finite_reach(b, causal, window, heads, kv_heads, D, at, value):
    lead, n, T = 77, 600, 750
    starts = starts_of([70, n, 0, 3], lead=7)
    q, k, v = inputs(T, heads, kv_heads, D, seed=9)
    grad_out = randn((T, heads, D), 10)
    plan = b.AttentionPlan(starts, T)
    kw = dict(causal=causal, window=window)
    f = b.dppf_attention(q, k, v, plan, **kw)
    g = b.dppf_attention_grad(grad_out, q, k, v, f.out, f.lse, plan, **kw)
    seen, tiles = reach(n, at, causal, window)
    queries, near_queries = placed(seen[:, at], lead, T), placed(tiles[:, at], lead, T)      # that see it as a key
    keys, near_keys = placed(seen[at], lead, T), placed(tiles[at], lead, T)                  # that it sees as a query
    none, own = torch.zeros_like(queries), placed(torch.arange(n, device="cuda") == at, lead, T)

    def spoiled(t):
        t = t.clone()
        t[lead + at, :, 5] = value
        return t

    # forward: a value reaches the tiles, a key those that see it, a query itself (an infinite score may be of no weight)
    bad = b.dppf_attention(q, k, spoiled(v), plan, **kw)
    assert same_bits(bad.lse, f.lse)
    others = torch.arange(D, device="cuda") != 5
    assert same_bits(bad.out[..., others], f.out[..., others])
    assert not torch.isfinite(bad.out[queries][..., 5].float()).any()
    assert same_bits(bad.out[~near_queries], f.out[~near_queries])
    bad = b.dppf_attention(q, spoiled(k), v, plan, **kw)
    check_reach(bad.out, f.out, queries if value != value else none, queries, "key, out")
    assert same_bits(bad.lse[:, ~queries], f.lse[:, ~queries])
    bad = b.dppf_attention(spoiled(q), k, v, plan, **kw)
    check_reach(bad.out, f.out, own if value != value else none, own, "query, out")

    # the gradient, from the statistics of finite rows
    bad = b.dppf_attention_grad(spoiled(grad_out), q, k, v, f.out, f.lse, plan, **kw)
    check_reach(bad.q, g.q, own if value != value else none, own, "grad_out, grad_q")
    check_reach(bad.k, g.k, keys if value != value else none, keys, "grad_out, grad_k")
    check_reach(bad.v, g.v, none, near_keys, "grad_out, grad_v")
    assert not torch.isfinite(bad.v[keys][..., 5].float()).any() and same_bits(bad.v[..., others], g.v[..., others])
    bad = b.dppf_attention_grad(grad_out, q, spoiled(k), v, f.out, f.lse, plan, **kw)
    check_reach(bad.q, g.q, queries if value != value else none, near_queries, "key, grad_q")
    check_reach(bad.k, g.k, own if value != value else none, own, "key, grad_k")
    check_reach(bad.v, g.v, own if value != value else none, own, "key, grad_v")
    bad = b.dppf_attention_grad(grad_out, q, k, spoiled(v), f.out, f.lse, plan, **kw)
    check_reach(bad.q, g.q, queries if value != value else none, queries, "value, grad_q")
    check_reach(bad.k, g.k, own if value != value else none, own, "value, grad_k")
    assert same_bits(bad.v, g.v)
    bad = b.dppf_attention_grad(grad_out, spoiled(q), k, v, f.out, f.lse, plan, **kw)
    check_reach(bad.q, g.q, own if value != value else none, own, "query, grad_q")
    check_reach(bad.k, g.k, keys if value != value else none, near_keys, "query, grad_k")
    check_reach(bad.v, g.v, keys if value != value else none, keys, "query, grad_v")


# ---------------------------------------------------------------- numbers beyond 32 bits

@pytest.mark.parametrize("more", [2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 70 + 1])
def test_windows_beyond_32_bits_are_none(b, more):
    T = 300
    q, k, v = inputs(T, 2, 2, 64, seed=11)
    plan = b.AttentionPlan(starts_of([T]), T)
    f = b.dppf_attention(q, k, v, plan)
    got = b.dppf_attention(q, k, v, plan, window=more)
    assert same_bits(got.out, f.out) and same_bits(got.lse, f.lse)
    want = b.dppf_attention_grad(q, q, k, v, f.out, f.lse, plan)
    assert all(same_bits(x, y) for x, y in zip(want, b.dppf_attention_grad(q, q, k, v, f.out, f.lse, plan, window=more)))
    for call in (lambda w: b.dppf_attention(q, k, v, plan, window=w), lambda w: b.dppf_attention_grad(q, q, k, v, f.out, f.lse, plan, window=w)):
        with pytest.raises(b.DppfError) as err:
            call(-more)
        assert err.value.status == b.ERR_INVALID_ARG


def test_sizes_beyond_32_bits_are_refused(b):
    H = 2 ** 32 + 8                                                             # 8 to a 32-bit integer
    x = torch.empty(1, H, dtype=BF16, device="cuda")
    for rows in (x, x[0]):
        with pytest.raises(ValueError):
            b.dppf_layer_norm(rows, x[0])
    stat = torch.ones(1, device="cuda")
    with pytest.raises(ValueError):
        b.dppf_layer_norm_grad(x, x, stat, stat, x[0], x[0], grad_x=x)
    with pytest.raises(ValueError):
        b.dppf_embedding(x, torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        b.dppf_rotary(x.view(1, 1, H), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.ones(1, dtype=torch.float64, device="cuda"), out=x.view(1, 1, H))
    with pytest.raises(ValueError):
        b.AttentionPlan(torch.zeros(2, dtype=torch.int32, device="cuda"), 2 ** 64 + 5)


# ---------------------------------------------------------------- many sequences

@pytest.mark.parametrize("causal,window", [(False, 0), (True, 0), (True, 3)])
def test_gradients_of_many_sequences(b, causal, window):
    """More sequences than the plan's kernel has threads, against the formulas; sequences of no rows among them."""
    lens = torch.randint(0, 9, (3000,), generator=torch.Generator().manual_seed(5)).tolist()
    lens[1030], lens[2040] = 300, 129                                           # and some that do not fit a tile, past the first thousand
    lead, tail = 5, 140
    starts = starts_of(lens, lead)
    T = int(starts[-1]) + tail
    q, k, v = inputs(T, 2, 1, 32, seed=12)
    grad_out = randn((T, 2, 32), 13)
    plan = b.AttentionPlan(starts, T)
    kw = dict(causal=causal, window=window)
    f = b.dppf_attention(q, k, v, plan, **kw)
    want = reference(q, k, v, starts, causal, window, 32 ** -0.5)
    within(f.lse, *want["lse"], "lse")
    within(f.out, *want["out"], "out")
    got = b.dppf_attention_grad(grad_out, q, k, v, f.out, f.lse, plan, **kw)
    want = reference(q, k, v, starts, causal, window, 32 ** -0.5, (grad_out, f.out, f.lse))
    for name in "qkv":
        within(getattr(got, name), *want[name], name)
    for t in (f.out, *got):
        assert not t[:lead].any() and not t[T - tail:].any()
    for rows in (slice(0, lead), slice(T - tail, T)):
        assert (f.lse[:, rows] == -math.inf).all()                              # minus infinity, not plus
