"""Attention within packed sequences on the GPU, forward and backward, against plain implementations in 64 bits.

Tolerances.  Half a step of bf16 is 2^-8, of fp32 2^-24.  A score is a sum of D products in fp32: off by at most 2^-20 A, A = the
sum of their magnitudes times scale.  A sum of exponentials (2 ulp each) adds at most 64 in a thread and then a term a block of
128 keys: below 7e-6 for up to 40 blocks.  So
  lse      7e-6 + 2^-20 A =: e
  out      every probability is rounded to bf16: (2^-8 + 2 e) sum p |v|, and 2^-8 |out| for the result
  grads    p is e off (the given lse), dP is off by 2^-20 of its magnitudes' sum and D_t likewise, dS = p (dP - D_t) is rounded to
           bf16: (2^-8 + 2 e) |dS| + p 2^-19 (sum |do v| + sum |do o|) for each, times |k| or |q|, summed;  dv as out; 2^-8 of the result
  all      exponentials below 2^-126 are 0; times factors of up to 2^16 and summed over up to 2^10 keys that is below 2^-100
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
    off = (got.double() - want)[fine].abs() - tol[fine] - 2.0 ** -100
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


def test_gradient_is_the_slope(b):
    """Against differences of the formula in 64 bits: the loss is sum c out."""
    starts = starts_of([5, 40, 131])
    T, heads, kv, D = int(starts[-1]), 4, 2, 32
    q, k, v = inputs(T, heads, kv, D, seed=5, std=0.5)
    c = randn((T, heads, D), 6)
    plan = b.AttentionPlan(starts, T)
    fwd = b.dppf_attention(q, k, v, plan)
    grads = b.dppf_attention_grad(c, q, k, v, fwd.out, fwd.lse, plan)

    def loss(q, k, v):
        out = reference_out(q, k, v, starts)
        return (c.double() * out).sum()

    at, step = [x.double() for x in (q, k, v)], 1e-5
    for i in range(3):
        for seed in range(2):
            d = torch.randn(at[i].shape, generator=gen(30 + seed), device="cuda", dtype=F64)
            up, down = ([x + sign * step * d if n == i else x for n, x in enumerate(at)] for sign in (1, -1))
            slope = float((loss(*up) - loss(*down)) / (2 * step))
            got = float((grads[i].double() * d).sum())
            # the gradient's roundings, 2^-8 each of P, dS and the result, add up like random ones: 4 * 2^-8 of the root of the sum of squares
            assert abs(got - slope) < 4 * HALF * float((grads[i].double() * d).square().sum().sqrt()) + 1e-4, (i, got, slope)


def reference_out(q, k, v, starts):
    out = torch.zeros(q.shape, dtype=F64, device="cuda")
    at = starts.tolist()
    share = q.shape[1] // k.shape[1]
    for a, e in zip(at, at[1:]):
        for h in range(q.shape[1]):
            s = q[a:e, h] @ k[a:e, h // share].t() * q.shape[2] ** -0.5
            s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), -math.inf)
            out[a:e, h] = torch.softmax(s, 1) @ v[a:e, h // share]
    return out


@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (3, 3)])
@pytest.mark.parametrize("jump", [20.0, 300.0, -300.0])
@pytest.mark.parametrize("causal", [True, False])
def test_scores_that_grow_from_tile_to_tile(b, heads, kv_heads, jump, causal):
    """Keys whose scores rise (or fall) by `jump` from tile to tile: sums have to be taken relative to a new maximum, or most keys vanish."""
    T, D = 700, 64
    starts = starts_of([T])
    q, k, v = (x.clone() for x in inputs(T, heads, kv_heads, D, seed=7, std=0.3))
    q[..., 0] = 8.0
    k[..., 0] = (torch.arange(T, device="cuda") // 128 * jump)[:, None].to(BF16)
    plan = b.AttentionPlan(starts, T)
    got = b.dppf_attention(q, k, v, plan, causal=causal)
    want = reference(q, k, v, starts, causal, 0, D ** -0.5)
    within(got.lse, *want["lse"], "lse")
    within(got.out, *want["out"], "out")
    grad_out = randn((T, heads, D), 8)
    grads = b.dppf_attention_grad(grad_out, q, k, v, got.out, got.lse, plan, causal=causal)
    want = reference(q, k, v, starts, causal, 0, D ** -0.5, (grad_out, got.out, got.lse))
    for name in ("q", "k", "v"):
        within(getattr(grads, name), *want[name], name)


@pytest.mark.parametrize("heads,kv_heads,D", [(4, 2, 128), (2, 2, 56)])
@pytest.mark.parametrize("causal", [True, False])
def test_other_rows_do_not_matter(b, heads, kv_heads, D, causal):
    """What stands in rows of other sequences, or of none, NaN and infinities included, changes no bit of a sequence's results."""
    lens, at = [60, 200, 77], 1
    starts = starts_of(lens, lead=9)
    T = int(starts[-1]) + 50
    a, e = int(starts[at]), int(starts[at + 1])
    q, k, v = (x.clone() for x in inputs(T, heads, kv_heads, D, seed=9))
    grad_out = randn((T, heads, D), 10)
    plan = b.AttentionPlan(starts, T)

    def run():
        f = b.dppf_attention(q, k, v, plan, causal=causal)
        return f, b.dppf_attention_grad(grad_out, q, k, v, f.out, f.lse, plan, causal=causal)

    f0, g0 = run()
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device="cuda").to(BF16)
    for t in (q, k, v, grad_out):
        for rows in (slice(0, a), slice(e, T)):
            t[rows] = bad[torch.randint(0, 4, t[rows].shape, generator=gen(11), device="cuda")]
    f1, g1 = run()
    assert same_bits(f0.out[a:e], f1.out[a:e]) and same_bits(f0.lse[:, a:e], f1.lse[:, a:e])
    assert all(same_bits(x[a:e], y[a:e]) for x, y in zip(g0, g1))
    for t in (f1.out, *g1):
        assert not t[:9].any() and not t[-50:].any()


def test_values_that_are_not_finite_spoil_their_queries(b):
    starts = starts_of([300])
    q, k, v = (x.clone() for x in inputs(300, 2, 1, 64, seed=12))
    k[200, 0, 5] = float("nan")
    out = b.dppf_attention(q, k, v, b.AttentionPlan(starts, 300))
    assert torch.isnan(out.out[200:].float()).all() and torch.isfinite(out.out[:128].float()).all()


def test_layouts(b):
    """Heads in blocks of their own, padded rows, gradients beside one another; nothing beside them is written."""
    T, heads, kv, D = 333, 4, 2, 40
    starts = starts_of([100, 233])
    base = inputs(T, heads, kv, D, seed=13)
    grad_out = randn((T, heads, D), 14)
    plan = b.AttentionPlan(starts, T)
    f = b.dppf_attention(*base, plan)
    g = b.dppf_attention_grad(grad_out, *base, f.out, f.lse, plan)

    def by_head(n, pad=8):
        whole = torch.full((n, T, D + pad), float("nan"), dtype=BF16, device="cuda")
        return whole, whole[:, :, :D].transpose(0, 1)

    copies = []
    for t in (*base, grad_out):
        _, view = by_head(t.shape[1])
        view.copy_(t)
        copies.append(view)
    whole, out = by_head(heads)
    lse = torch.full((heads, T), float("nan"), device="cuda")
    b.dppf_attention(*copies[:3], plan, out=out, lse=lse)
    assert same_bits(out, f.out) and same_bits(lse, f.lse) and torch.isnan(whole[:, :, D:].float()).all()
    rows = torch.full((T, (heads + 2 * kv) * D + 24), float("nan"), dtype=BF16, device="cuda")
    cut = lambda n, first: rows[:, first:first + n * D].unflatten(1, (n, D))  # noqa: E731
    dq, dk, dv = cut(heads, 8), cut(kv, 8 + heads * D), cut(kv, 8 + (heads + kv) * D)
    got = b.dppf_attention_grad(copies[3], *copies[:3], out, lse, plan, grad_q=dq, grad_k=dk, grad_v=dv)
    assert got.q is dq and same_bits(dq, g.q) and same_bits(dk, g.k) and same_bits(dv, g.v)
    assert torch.isnan(rows[:, :8].float()).all() and torch.isnan(rows[:, 8 + (heads + 2 * kv) * D:].float()).all()


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_starts_that_are_out_of_order(b, dtype):
    T = 500
    q, k, v = inputs(T, 2, 1, 64, seed=15)
    starts = torch.tensor([-7, 100, 60, 250, 250, 9999, 400], device="cuda").to(dtype)
    kept = torch.tensor([0, 100, 100, 250, 250, 500, 500], dtype=torch.int32, device="cuda")
    got = b.dppf_attention(q, k, v, b.AttentionPlan(starts, T))
    want = b.dppf_attention(q, k, v, b.AttentionPlan(kept, T))
    assert same_bits(got.out, want.out) and same_bits(got.lse, want.lse)
    if dtype is torch.int64:
        far = b.AttentionPlan(torch.tensor([-2 ** 62, 2 ** 40], device="cuda"), T)
        assert same_bits(b.dppf_attention(q, k, v, far).out, b.dppf_attention(q, k, v, b.AttentionPlan(starts_of([T]), T)).out)


def test_many_sequences(b):
    lens = torch.randint(0, 9, (5000,), generator=torch.Generator().manual_seed(3)).tolist()
    starts = starts_of(lens)
    T = int(starts[-1]) + 3
    q, k, v = inputs(T, 2, 1, 32, seed=16)
    plan = b.AttentionPlan(starts, T)
    got = b.dppf_attention(q, k, v, plan, causal=False)
    # block diagonal scores, some thousands of rows at a time
    seq = torch.bucketize(torch.arange(T, device="cuda"), starts[1:].long(), right=True)
    want = torch.zeros(T, 2, 32, dtype=F64, device="cuda")
    for a in range(0, T - 3, 4000):
        e = min(T - 3, a + 4000)
        lo, hi = max(0, a - 16), min(T - 3, e + 16)
        for h in range(2):
            s = q[a:e, h].double() @ k[lo:hi, 0].double().t() * 32 ** -0.5
            want[a:e, h] = torch.softmax(s.masked_fill(seq[a:e, None] != seq[None, lo:hi], -math.inf), 1) @ v[lo:hi, 0].double()
    within(got.out, want, (HALF + 1e-4) * 6.0 + HALF * want.abs())              # sum p |v| <= max |v| < 6
    grads = b.dppf_attention_grad(q, q, k, v, got.out, got.lse, plan, causal=False)
    assert all(torch.isfinite(x.float()).all() for x in grads) and b.dppf_device_status(plan.buffer) == b.OK


def test_far_rows(b):
    T, heads, D = 300_000, 64, 128                                              # 2.5e9 elements
    n = 300
    starts = starts_of([n], lead=T - n)
    q = torch.empty(T, heads, D, dtype=BF16, device="cuda")
    k, v = torch.empty(T, 2, D, dtype=BF16, device="cuda"), torch.empty(T, 2, D, dtype=BF16, device="cuda")
    q[-n:], k[-n:], v[-n:] = (x for x in (randn((n, heads, D), 17), randn((n, 2, D), 18), randn((n, 2, D), 19)))
    far, near = b.AttentionPlan(starts, T), b.AttentionPlan(starts_of([n]), n)
    f, g = b.dppf_attention(q, k, v, far), b.dppf_attention(q[-n:], k[-n:], v[-n:], near)
    assert same_bits(f.out[-n:], g.out) and same_bits(f.lse[:, -n:], g.lse) and not f.out[:-n].any()
    df = b.dppf_attention_grad(q, q, k, v, f.out, f.lse, far)
    # the heads that share a key head may be summed in other parts where there are few rows: against the formulas
    want = reference(q[-n:], k[-n:], v[-n:], starts_of([n]), True, 0, D ** -0.5, (q[-n:], g.out, g.lse))
    for name, x in zip("qkv", df):
        within(x[-n:], *want[name], name)
        assert not x[:-n].any()


def test_streams_graphs_and_a_shared_plan(b):
    lens, other = [130, 1, 200], [31, 200, 100]
    starts = starts_of(lens)
    T = int(starts[-1])
    q, k, v = (x.clone() for x in inputs(T, 4, 2, 64, seed=20))
    grad_out = randn((T, 4, 64), 21)
    plan, ws = b.AttentionPlan(starts, T), b.alloc_attention_workspace(T, 4)

    def step(ws=ws):
        f = b.dppf_attention(q, k, v, plan)
        return (*f, *b.dppf_attention_grad(grad_out, q, k, v, f.out, f.lse, plan, ws=ws))

    want = step()
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in sides:                                                             # side by side on one plan, each its own workspace
        with torch.cuda.stream(s):
            got.append([step(b.alloc_attention_workspace(T, 4)) for _ in range(4)])
    torch.cuda.synchronize()
    assert all(same_bits(x, y) for runs in got for r in runs for x, y in zip(r, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.renew(starts)
        captured = step()
    starts.copy_(starts_of(other))
    q.copy_(randn(q.shape, 22))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    plan = b.AttentionPlan(starts_of(other), T)
    assert all(same_bits(x, y) for x, y in zip(captured, step()))


def test_waits_that_give_up(b):
    """With no polls allowed every wait gives up at once: the rows are NaN and the status says so; the next calls are well."""
    starts = starts_of([300, 20])
    T = 320
    q, k, v = inputs(T, 4, 2, 128, seed=23)
    plan = b.AttentionPlan(starts, T)
    want = b.dppf_attention(q, k, v, plan)
    grads = b.dppf_attention_grad(q, q, k, v, want.out, want.lse, plan)
    try:
        b.debug_set_poll_limits(0, -1)
        got = b.dppf_attention(q, k, v, plan)
        status = b.dppf_device_status(plan.buffer)
        assert status == b.ERR_TIMEOUT and torch.isnan(got.out.float()).all() and torch.isnan(got.lse).all()
        plan.renew(starts)
        assert b.dppf_device_status(plan.buffer) == b.OK
        bad = b.dppf_attention_grad(q, q, k, v, want.out, want.lse, plan)
        assert b.dppf_device_status(plan.buffer) == b.ERR_TIMEOUT and all(torch.isnan(x.float()).all() for x in bad)
    finally:
        b.debug_set_poll_limits(-1, -1)
    plan.renew(starts)
    again = b.dppf_attention(q, k, v, plan)
    assert same_bits(again.out, want.out) and all(same_bits(x, y) for x, y in zip(grads, b.dppf_attention_grad(q, q, k, v, again.out, again.lse, plan)))
    assert b.dppf_device_status(plan.buffer) == b.OK


def test_a_plan_of_other_sequences_writes_nothing(b):
    """The lists of a plan lie where its numbers of rows and sequences put them: another number is told from the plan itself."""
    T = 900
    q, k, v = inputs(T, 2, 1, 64, seed=26)
    plan = b.AttentionPlan(starts_of([300, 300, 300]), T)
    plan.sequences = 600                                                        # as a C caller may get it wrong
    plan.buffer = torch.cat([plan.buffer, torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")])
    out, lse = torch.full_like(q, 7.0), torch.full((2, T), 7.0, device="cuda")
    b.dppf_attention(q, k, v, plan, out=out, lse=lse)
    assert b.dppf_device_status(plan.buffer) == b.ERR_WORKSPACE and (out == 7).all() and (lse == 7).all()
    got = b.dppf_attention_grad(q, q, k, v, out, lse, plan, grad_q=torch.full_like(q, 7.0), grad_k=torch.full_like(k, 7.0), grad_v=torch.full_like(v, 7.0))
    assert all((x == 7).all() for x in got)


@pytest.mark.parametrize("window", [500, 501, 2 ** 31 - 1])
def test_windows_as_long_as_the_batch(b, window):
    T = 500
    q, k, v = inputs(T, 3, 3, 64, seed=27)
    plan = b.AttentionPlan(starts_of([T]), T)
    f, g = b.dppf_attention(q, k, v, plan), b.dppf_attention(q, k, v, plan, window=window)
    assert same_bits(f.out, g.out) and same_bits(f.lse, g.lse)
    assert all(same_bits(x, y) for x, y in zip(b.dppf_attention_grad(q, q, k, v, f.out, f.lse, plan), b.dppf_attention_grad(q, q, k, v, f.out, f.lse, plan, window=window)))


def test_a_plan_of_other_rows_writes_nothing(b):
    plan = b.AttentionPlan(starts_of([64]), 64)
    q, k, v = inputs(64, 1, 1, 64, seed=24)
    plan.buffer[:4096].zero_()
    out, lse = torch.full_like(q, 7.0), torch.full((1, 64), 7.0, device="cuda")
    b.dppf_attention(q, k, v, plan, out=out, lse=lse)
    assert b.dppf_device_status(plan.buffer) == b.ERR_WORKSPACE and (out == 7).all() and (lse == 7).all()
    got = b.dppf_attention_grad(q, q, k, v, out, lse, plan, grad_q=torch.full_like(q, 7.0), grad_k=torch.full_like(k, 7.0), grad_v=torch.full_like(v, 7.0))
    assert all((x == 7).all() for x in got)


def test_no_tokens_and_refusals(b):
    plan = b.AttentionPlan(torch.zeros(3, dtype=torch.int32, device="cuda"), 0)
    empty = torch.empty(0, 4, 64, dtype=BF16, device="cuda")
    f = b.dppf_attention(empty, empty[:, :2], empty[:, :2], plan)
    assert f.out.shape == (0, 4, 64) and f.lse.shape == (4, 0)
    assert b.dppf_attention_grad(empty, empty, empty[:, :2], empty[:, :2], f.out, f.lse, plan).k.shape == (0, 2, 64)
    T = 20
    q, k, v = inputs(T, 4, 2, 64, seed=25)
    plan = b.AttentionPlan(starts_of([T]), T)
    for bad in (dict(q=q.float()), dict(k=k[:, :1]), dict(v=v[:10]), dict(q=q[..., :32]), dict(out=q[:, :2]), dict(q=q[0]), dict(lse=torch.empty(3, T, device="cuda")), dict(q=q.half())):
        a = {"q": q, "k": k, "v": v, "out": None, "lse": None, **bad}
        with pytest.raises(ValueError):
            b.dppf_attention(a["q"], a["k"], a["v"], plan, out=a["out"], lse=a["lse"])
    q3 = torch.cat([q, q], 1)[:, :7]
    odd = torch.zeros(T, 4, 72, dtype=BF16, device="cuda")
    for args, kw, status in (((q3, k, v), {}, b.ERR_INVALID_ARG), ((q, k, v), dict(window=5, causal=False), b.ERR_INVALID_ARG), ((q, k, v), dict(window=-1), b.ERR_INVALID_ARG),
                             ((q, k, v), dict(scale=0.0), b.ERR_INVALID_ARG), ((q, k, v), dict(scale=float("nan")), b.ERR_INVALID_ARG), ((q, k, v), dict(out=q), b.ERR_INVALID_ARG),
                             ((odd[..., 1:65], k, v), {}, b.ERR_ALIGNMENT), ((odd[..., :60], odd[:, :2, :60], odd[:, :2, :60]), {}, b.ERR_INVALID_ARG)):
        with pytest.raises(b.DppfError) as err:
            b.dppf_attention(*args, plan, **kw)
        assert err.value.status == status
    f = b.dppf_attention(q, k, v, plan)
    with pytest.raises(b.DppfError):
        b.dppf_attention_grad(q, q, k, v, f.out, f.lse, plan, grad_q=f.out)
    with pytest.raises(ValueError):
        b.dppf_attention_grad(q, q, k, v, f.out, f.lse[:2], plan)
    with pytest.raises(ValueError):
        b.dppf_attention_grad(q[:, :2], q, k, v, f.out, f.lse, plan)
    with pytest.raises(ValueError):
        b.AttentionPlan(torch.zeros(1, dtype=torch.int32, device="cuda"), 5)
    with pytest.raises(ValueError):
        b.AttentionPlan(torch.zeros(2, device="cuda"), 5)
    with pytest.raises(ValueError):
        plan.renew(torch.zeros(5, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("seed", range(10))
def test_random_batches(b, seed):
    """Batches of more tiles than SMs, so that blocks stay for several: heads, widths, masks and lengths at random, rows of no sequence in between."""
    import random
    rng = random.Random(1000 + seed)
    kv_heads = rng.choice([1, 2, 3, 5, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4] if kv_heads > 3 else [4, 6, 7, 8, 12])
    D = 8 * rng.randrange(1, 17)
    lens = [rng.choice([0, 1, rng.randrange(2, 130), rng.randrange(100, 700), rng.randrange(600, 1500)]) for _ in range(rng.randrange(4, 12))]
    lead, tail = rng.choice([0, rng.randrange(1, 300)]), rng.choice([0, rng.randrange(1, 300)])
    causal = rng.random() < 0.7
    window = rng.choice([0, rng.randrange(1, 900)]) if causal else 0
    starts = starts_of(lens, lead)
    T = int(starts[-1]) + tail
    q, k, v = inputs(T, heads, kv_heads, D, seed=seed)
    scale = rng.uniform(0.02, 0.3)
    plan = b.AttentionPlan(starts, T)
    got = b.dppf_attention(q, k, v, plan, causal=causal, window=window, scale=scale)
    want = reference(q, k, v, starts, causal, window, scale)
    within(got.lse, *want["lse"], "lse")
    within(got.out, *want["out"], "out")
    again = b.dppf_attention(q, k, v, plan, causal=causal, window=window, scale=scale)
    assert same_bits(again.out, got.out) and same_bits(again.lse, got.lse)
    check_grads(b, lens, heads, kv_heads, D, causal, window, scale=scale, lead=lead, tail=tail, seed=seed)


def test_the_stride_of_a_single_head_says_nothing(b):
    """0 or any other multiple of 8 at the C entries, where the binding gives the width."""
    T, D = 150, 64
    q, k, v = (t.contiguous() for t in inputs(T, 1, 1, D, seed=31))
    plan = b.AttentionPlan(starts_of([100, 50]), T)
    want = b.dppf_attention(q, k, v, plan)
    grads = b.dppf_attention_grad(q, q, k, v, want.out, want.lse, plan)
    ws, lib, stream = b.alloc_attention_workspace(T, 1), b.load(), torch.cuda.current_stream().cuda_stream
    at = (plan.buffer.data_ptr(), plan.buffer.nbytes)
    for head in (0, 8, 4096):
        out, lse, got = torch.empty_like(q), torch.empty_like(want.lse), [torch.empty_like(q) for _ in range(3)]
        rows = lambda t: (t.data_ptr(), D, head)  # noqa: E731
        assert lib.dppf_attention(*rows(q), *rows(k), *rows(v), T, 2, 1, 1, D, 1, 0, D ** -0.5, *rows(out), lse.data_ptr(), *at, stream) == 0
        assert lib.dppf_attention_grad(*rows(q), *rows(q), *rows(k), *rows(v), *rows(want.out), want.lse.data_ptr(), T, 2, 1, 1, D, 1, 0, D ** -0.5,
                                       *[x for t in got for x in rows(t)], *at, ws.data_ptr(), ws.nbytes, stream) == 0
        assert same_bits(out, want.out) and same_bits(lse, want.lse) and all(same_bits(x, y) for x, y in zip(got, grads))


def test_heads_of_no_width_are_refused(b):
    none = torch.empty(5, 2, 0, dtype=BF16, device="cuda")
    with pytest.raises(b.DppfError) as err:
        b.dppf_attention(none, none, none, b.AttentionPlan(starts_of([5]), 5))
    assert err.value.status == b.ERR_INVALID_ARG
