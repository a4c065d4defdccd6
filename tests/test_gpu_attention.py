"""Attention within packed sequences on the GPU, forward and backward, against plain implementations in 64 bits.

Tolerances.  Half a step of bf16 is 2^-8, of fp32 2^-24.  A score is a sum of D products in fp32: off by at most 2^-20 A, A = the
sum of their magnitudes times scale.  A sum of exponentials (2 ulp each) adds at most 64 in a thread and then a term a block of
128 keys: below 7e-6 for up to 40 blocks.  So
  lse      7e-6 + 2^-20 A =: e
  out      every probability is rounded to bf16: (2^-8 + 2 e) sum p |v|, and 2^-8 |out| for the result
  grads    p is e off (the given lse), dP is off by 2^-20 of its magnitudes' sum and D_t likewise, dS = p (dP - D_t) is rounded to
           bf16: (2^-8 + 2 e) |dS| + p 2^-19 (sum |do v| + sum |do o|) for each, times |k| or |q|, summed;  dv as out; 2^-8 of the result
"""
import math

import pytest
import torch

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
BF16, F64 = torch.bfloat16, torch.float64
HALF = 2.0 ** -8


@pytest.fixture(scope="module")
def b():
    return require_gpu()[1]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(shape, seed, std=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * std).to(BF16)


def same_bits(x, y):
    k = {4: torch.int32, 2: torch.int16}[x.element_size()]
    return x.shape == y.shape and torch.equal(x.contiguous().view(k), y.contiguous().view(k))


def starts_of(lens, lead=0):
    at = [lead]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def within(got, want, tol, what=""):
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    fine = torch.isfinite(want)
    off = (got.double() - want)[fine].abs() - tol[fine]
    assert not off.numel() or float(off.max()) <= 0, (what, float(off.max()), float(tol[fine].max()))


def reference(q, k, v, starts, causal, window, scale, grad=None):
    """{name: (value, tolerance)} by the formulas in fp64; grad: (grad_out, out, lse) as given to the gradient."""
    T, heads, D = q.shape
    share = heads // k.shape[1]
    zero = lambda n: [torch.zeros(T, n, D, dtype=F64, device="cuda") for _ in range(2)]  # noqa: E731
    out, dq, dk, dv = zero(heads), zero(heads), zero(k.shape[1]), zero(k.shape[1])
    lse = [torch.full((heads, T), -math.inf, dtype=F64, device="cuda"), torch.zeros(heads, T, dtype=F64, device="cuda")]
    at = starts.tolist()
    for a, e in zip(at, at[1:]):
        n = e - a
        if n <= 0:
            continue
        i = torch.arange(n, device="cuda")
        gap = i[:, None] - i
        seen = torch.ones(n, n, dtype=torch.bool, device="cuda")
        if causal:
            seen &= gap >= 0
        if window:
            seen &= gap < window
        for h in range(heads):
            j = h // share
            qq, kk, vv = q[a:e, h].double(), k[a:e, j].double(), v[a:e, j].double()
            s = (qq @ kk.t() * scale).masked_fill(~seen, -math.inf)
            size = (qq.abs() @ kk.abs().t() * scale).masked_fill(~seen, 0).amax(1)
            err = 7e-6 + 2.0 ** -20 * size
            if grad is None:
                l = torch.logsumexp(s, 1)
                p = torch.exp(s - l[:, None])
                lse[0][h, a:e], lse[1][h, a:e] = l, err
                out[0][a:e, h] = p @ vv
                out[1][a:e, h] = (HALF + 2 * err[:, None]) * (p @ vv.abs()) + HALF * (p @ vv).abs()
                continue
            do, o, l = grad[0][a:e, h].double(), grad[1][a:e, h].double(), grad[2][h, a:e].double()
            p = torch.exp(s - l[:, None])
            ds = p * (do @ vv.t() - (do * o).sum(1, keepdim=True))
            off = (HALF + 2 * err[:, None]) * ds.abs() + p * 2.0 ** -19 * (do.abs() @ vv.abs().t() + (do * o).abs().sum(1, keepdim=True))
            dq[0][a:e, h], dq[1][a:e, h] = ds @ kk * scale, off @ kk.abs() * scale
            dk[0][a:e, j] += ds.t() @ qq * scale
            dk[1][a:e, j] += off.t() @ qq.abs() * scale
            dv[0][a:e, j] += p.t() @ do
            dv[1][a:e, j] += (p * (HALF + 2 * err[:, None])).t() @ do.abs()
    if grad is None:
        return {"out": tuple(out), "lse": tuple(lse)}
    return {name: (x, tol + HALF * x.abs()) for name, (x, tol) in (("q", dq), ("k", dk), ("v", dv))}


LENGTHS = [[1], [2], [127], [128], [129], [255], [256], [257], [700], [5, 0, 1, 300, 130, 0], [1] * 40, [384, 384], [33, 129, 640]]
HEADS = [(1, 1, 64), (2, 1, 128), (4, 4, 128), (3, 1, 64), (8, 2, 72), (6, 2, 32), (2, 2, 8), (4, 1, 120)]


def inputs(T, heads, kv_heads, D, seed=1, std=1.0):
    rows = randn((T, heads + 2 * kv_heads, D), seed, std)
    return rows[:, :heads], rows[:, heads:heads + kv_heads], rows[:, heads + kv_heads:]


MASKS = [(True, 0), (False, 0), (True, 1), (True, 100), (True, 200)]


@pytest.mark.parametrize("lens", LENGTHS, ids=str)
@pytest.mark.parametrize("heads,kv_heads,D", [(2, 1, 128), (3, 3, 64)])
@pytest.mark.parametrize("causal,window", MASKS)
def test_forward_lengths(b, lens, heads, kv_heads, D, causal, window):
    starts = starts_of(lens)
    T = int(starts[-1])
    q, k, v = inputs(T, heads, kv_heads, D)
    plan = b.AttentionPlan(starts, T)
    got = b.dppf_attention(q, k, v, plan, causal=causal, window=window)
    want = reference(q, k, v, starts, causal, window, D ** -0.5)
    assert b.dppf_device_status(plan.buffer) == b.OK
    within(got.lse, *want["lse"], "lse")
    within(got.out, *want["out"], "out")


@pytest.mark.parametrize("heads,kv_heads,D", HEADS)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 77)])
def test_forward_heads(b, heads, kv_heads, D, causal, window):
    starts = starts_of([150, 1, 333], lead=7)
    T = int(starts[-1]) + 131                                                  # rows of no sequence at both ends
    q, k, v = inputs(T, heads, kv_heads, D, seed=2, std=2.0)
    plan = b.AttentionPlan(starts.long(), T)
    got = b.dppf_attention(q, k, v, plan, causal=causal, window=window, scale=0.11)
    want = reference(q, k, v, starts, causal, window, 0.11)
    within(got.lse, *want["lse"], "lse")
    within(got.out, *want["out"], "out")
    assert not got.out[:7].any() and not got.out[-131:].any() and torch.isinf(got.lse[:, -131:]).all()
    again = b.dppf_attention(q, k, v, plan, causal=causal, window=window, scale=0.11)
    assert same_bits(again.out, got.out) and same_bits(again.lse, got.lse)


def check_grads(b, lens, heads, kv_heads, D, causal, window, scale=None, lead=0, tail=0, seed=3):
    starts = starts_of(lens, lead)
    T = int(starts[-1]) + tail
    q, k, v = inputs(T, heads, kv_heads, D, seed)
    scale = D ** -0.5 if scale is None else scale
    plan = b.AttentionPlan(starts, T)
    fwd = b.dppf_attention(q, k, v, plan, causal=causal, window=window, scale=scale)
    grad_out = randn((T, heads, D), seed + 1, 0.5)
    got = b.dppf_attention_grad(grad_out, q, k, v, fwd.out, fwd.lse, plan, causal=causal, window=window, scale=scale)
    assert b.dppf_device_status(plan.buffer) == b.OK
    want = reference(q, k, v, starts, causal, window, scale, (grad_out, fwd.out, fwd.lse))
    for name in ("v", "q", "k"):
        within(getattr(got, name), *want[name], name)
        x = getattr(got, name)
        assert not x[:lead].any() and not x[T - tail:].any()
    again = b.dppf_attention_grad(grad_out, q, k, v, fwd.out, fwd.lse, plan, causal=causal, window=window, scale=scale)
    assert all(same_bits(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("lens", LENGTHS, ids=str)
@pytest.mark.parametrize("heads,kv_heads,D", [(2, 1, 128), (3, 3, 64)])
@pytest.mark.parametrize("causal,window", MASKS)
def test_backward_lengths(b, lens, heads, kv_heads, D, causal, window):
    check_grads(b, lens, heads, kv_heads, D, causal, window)


@pytest.mark.parametrize("heads,kv_heads,D", HEADS)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 77)])
def test_backward_heads(b, heads, kv_heads, D, causal, window):
    check_grads(b, [150, 1, 333], heads, kv_heads, D, causal, window, scale=0.11, lead=7, tail=131)
