"""Layer norm and rotary positions on the GPU against plain implementations in 64 bits.

Tolerances (eps = 2^-24; a result in bf16 is off by up to 2^-8 of itself more, HALF):
  layer norm   a thread adds 16 elements (rows above 16,384: up to 128), a tree of ten joins them: C eps with C = 60 (200) covers the
               mean's and the variance's sums and the products; the mean's error is relative to mean|h|:
               C eps (|xh w| + r mean|h| |w|) + 2 eps |b|
  gradient     mean and rstd are inputs, so xh is 2 eps off: C eps r (|u| + mean|u| + |xh| mean|u xh|) + 2 eps |dsum|;
               a column's sum adds at most T / 32 rows in a thread and 160 partial sums: (T / 32 + 180) eps sum|terms|
  rotary       the fraction of a turn is rounded to fp32 (half a turn at most: 1.9e-7 rad), cosine and sine are 1.2e-7 off, two
               products and a sum are rounded: 6e-7 (|x1| + |x2|) |scale|
"""
import math

import pytest
import torch

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def b():
    return require_gpu()[1]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(shape, seed, dtype=F32, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * std + mean).to(dtype)


def strided(rows, cols, stride, offset, dtype):
    """[rows, cols] view with a row stride and a start `offset` elements into its storage; gaps hold NaN."""
    return torch.full((offset + rows * stride,), float("nan"), dtype=dtype, device="cuda")[offset:].view(rows, stride)[:, :cols]


def storage_of(t):
    return torch.empty(0, dtype=t.dtype, device=t.device).set_(t.untyped_storage())


def same_bits(x, y):
    k = {4: torch.int32, 2: torch.int16}[x.element_size()]
    return x.shape == y.shape and torch.equal(x.contiguous().view(k), y.contiguous().view(k))


def within(got, want, tol):
    off = (got.double() - want).abs()
    assert bool((off <= tol + HALF[got.dtype] * want.abs()).all()), float((off - tol - HALF[got.dtype] * want.abs()).max())


# ---------------------------------------------------------------- layer norm

def check_norm(got, h, w, bias, eps):
    H = h.shape[-1]
    C = 60 if H <= 16384 else 200
    hd, wd = h.double(), w.double()
    mean = hd.mean(-1, keepdim=True)
    rstd = ((hd - mean).square().mean(-1, keepdim=True) + eps) ** -0.5
    size = hd.abs().mean(-1, keepdim=True)
    xh = (hd - mean) * rstd
    want = xh * wd + (0 if bias is None else bias.double())
    tol = C * EPS * ((xh * wd).abs() + rstd * size * wd.abs()) + (0 if bias is None else 2 * EPS * bias.double().abs())
    within(got.out, want, tol)
    within(got.mean, mean[..., 0], C * EPS * size[..., 0])
    within(got.rstd, rstd[..., 0], C * EPS * (rstd + rstd ** 2 * size)[..., 0])


SIZES = [(1, 1), (1, 7), (3, 64), (9, 257), (17, 512), (5, 513), (4, 1000), (2, 1022), (3, 4096), (2, 8192), (2, 9999), (2, 16384), (1, 16386), (3, 65536)]


@pytest.mark.parametrize("T,H", SIZES)
@pytest.mark.parametrize("xt,bt,ot,wt", [(F32, None, F32, F32), (F32, BF16, BF16, F32), (BF16, None, BF16, BF16), (BF16, F32, F32, F32), (BF16, BF16, BF16, F32), (F32, F32, BF16, BF16)])
def test_norm(b, T, H, xt, bt, ot, wt):
    x, w, bias = randn((T, H), 1, xt, 2.0, 0.5), randn(H, 2, wt, 0.2, 1.0), randn(H, 3, wt, 0.3)
    branch = None if bt is None else randn((T, H), 4, bt)
    x0 = x.clone()
    got = b.dppf_layer_norm(x, w, bias, eps=1e-5, branch=branch, out_dtype=ot)
    assert got.out.dtype == ot and same_bits(x, x0)
    h = x if branch is None else (x.float() + branch.float()).to(xt)
    assert same_bits(got.sum, h)
    check_norm(got, h, w, bias, 1e-5)
    plain = b.dppf_layer_norm(h, w, out_dtype=ot)                               # no bias, no branch
    check_norm(plain, h, w, None, 1e-5)
    if branch is not None:                                                      # the sum in the place of x, the same bits
        again = b.dppf_layer_norm(x, w, bias, eps=1e-5, branch=branch, sum_out=x, out_dtype=ot)
        assert same_bits(again.out, got.out) and same_bits(x, h) and same_bits(again.mean, got.mean)


@pytest.mark.parametrize("H,stride,off", [(32, 40, 0), (32, 37, 1), (32, 34, 2), (600, 601, 3), (640, 648, 8)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_strides(b, H, stride, off, dtype):
    T = 13
    x, branch, sum_out, out = (strided(T, H, stride, off, dtype) for _ in range(4))
    x.copy_(randn((T, H), 5))
    branch.copy_(randn((T, H), 6))
    w = randn(H + off, 7, dtype)[off:]
    got = b.dppf_layer_norm(x, w, branch=branch, sum_out=sum_out, out=out)
    h = (x.float() + branch.float()).to(dtype)
    assert same_bits(sum_out.contiguous(), h)
    check_norm(got, h, w, None, 1e-5)
    for t in (out, sum_out):
        t.fill_(float("nan"))
        assert torch.isnan(storage_of(t)).all()                                # nothing outside was written


def test_norm_of_hard_rows(b):
    H = 1000
    x = randn((6, H), 8)
    x[0] = 3.0                                                                  # equal values: variance 0
    x[1] += 1e4                                                                 # a mean far above the deviations
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    x[4] *= 1e-20                                                               # variance below eps
    w, bias = randn(H, 9), randn(H, 10)
    got = b.dppf_layer_norm(x, w, bias)
    keep = [0, 1, 4, 5]
    check_norm(b.LayerNorm(got.out[keep], x[keep], got.mean[keep], got.rstd[keep]), x[keep], w, bias, 1e-5)
    assert torch.equal(got.out[0], bias)
    assert torch.isnan(got.out[2]).all() and torch.isnan(got.out[3]).all()
    assert torch.isnan(b.dppf_layer_norm(x[:1], w, eps=0.0).out).all()


def norm_grads(dy, x, mean, rstd, w, dsum):
    dy, x, w, r = dy.double(), x.double(), w.double(), rstd.double()[:, None]
    xh, u = (x - mean.double()[:, None]) * r, dy * w
    mu, mx = u.mean(1, keepdim=True), (u * xh).mean(1, keepdim=True)
    dx = r * (u - mu - xh * mx) + (0 if dsum is None else dsum.double())
    C = 60 if x.shape[1] <= 16384 else 200
    tol = C * EPS * r * (u.abs() + u.abs().mean(1, keepdim=True) + xh.abs() * (u * xh).abs().mean(1, keepdim=True)) + (0 if dsum is None else 2 * EPS * dsum.double().abs())
    n = (x.shape[0] / 32 + 180) * EPS
    return dx, tol, (dy * xh).sum(0), n * (dy * xh).abs().sum(0), dy.sum(0), n * dy.abs().sum(0)


@pytest.mark.parametrize("T,H", [(1, 1), (3, 7), (700, 64), (333, 257), (40, 512), (3001, 200), (1, 513), (300, 1000), (150, 4096), (1300, 1022), (37, 8192), (35, 8194), (3, 65536)])
@pytest.mark.parametrize("xt,ot,wt,gt,stream,bias", [(F32, F32, F32, F32, False, True), (F32, BF16, F32, F32, True, True), (BF16, BF16, BF16, BF16, True, False), (BF16, F32, F32, BF16, False, True)])
def test_norm_grad(b, T, H, xt, ot, wt, gt, stream, bias):
    x, dy, w = randn((T, H), 11, xt, 2.0, 0.3), randn((T, H), 12, ot, 0.1), randn(H, 13, wt, 0.2, 1.0)
    dsum = randn((T, H), 14, xt, 0.1) if stream else None
    fwd = b.dppf_layer_norm(x, w)
    dw, db = torch.full((H,), float("nan"), dtype=gt, device="cuda"), torch.full((H,), float("nan"), dtype=gt, device="cuda") if bias else None
    dx = b.dppf_layer_norm_grad(dy, x, fwd.mean, fwd.rstd, w, dw, db, grad_sum=dsum)
    want, tol, want_w, tol_w, want_b, tol_b = norm_grads(dy, x, fwd.mean, fwd.rstd, w, dsum)
    within(dx, want, tol)
    within(dw, want_w, tol_w)
    if bias:
        within(db, want_b, tol_b)
    # added to what is there, from run to run the same bits, and in the place of an input
    dw2, db2 = torch.ones_like(dw), torch.ones_like(db) if bias else None
    into = dsum if stream else dy if xt == ot else None
    dx2 = b.dppf_layer_norm_grad(dy, x, fwd.mean, fwd.rstd, w, dw2, db2, grad_sum=dsum, grad_x=into, accumulate=True)
    assert same_bits(dx2, dx) and (into is None or dx2 is into)
    within(dw2, 1.0 + want_w, tol_w + 2 * EPS * (1 + want_w.abs()))
    if bias:
        within(db2, 1.0 + want_b, tol_b + 2 * EPS * (1 + want_b.abs()))


def test_norm_grad_is_the_slope(b):
    """Against differences of the formula in 64 bits: the loss is sum c y + sum s h."""
    T, H = 5, 96
    x, branch, w, bias, c, s = (randn((T, H) if k not in (2, 3) else (H,), 20 + k) for k in range(6))
    fwd = b.dppf_layer_norm(x, w, bias, branch=branch)
    dw, db = torch.empty_like(w), torch.empty_like(w)
    dx = b.dppf_layer_norm_grad(c, fwd.sum, fwd.mean, fwd.rstd, w, dw, db, grad_sum=s)

    def loss(h, w, bias):
        m = h.mean(1, keepdim=True)
        return (c.double() * ((h - m) * ((h - m).square().mean(1, keepdim=True) + 1e-5) ** -0.5 * w + bias)).sum() + (s.double() * h).sum()

    at, step = [fwd.sum.double(), w.double(), bias.double()], 1e-5
    for k, grad in enumerate((dx, dw, db)):
        for seed in range(3):
            d = torch.randn(at[k].shape, generator=gen(30 + seed), device="cuda", dtype=torch.float64)
            up, down = ([v + sign * step * d if i == k else v for i, v in enumerate(at)] for sign in (1, -1))
            slope = (loss(*up) - loss(*down)) / (2 * step)
            # cancellation of losses of size 100 leaves 1e-14 * 100 / 1e-5, the third derivative 1e-10 times a few hundred
            assert abs(float((grad.double() * d).sum() - slope)) < 1e-4 * math.sqrt(d.numel())


@pytest.mark.parametrize("H,stride,off", [(32, 37, 1), (600, 602, 2), (640, 648, 8)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_grad_strides(b, H, stride, off, dtype):
    T = 13
    x, dy, dsum, dx = (strided(T, H, stride, off, dtype) for _ in range(4))
    for k, t in enumerate((x, dy, dsum)):
        t.copy_(randn((T, H), 40 + k))
    w = randn(H, 43, dtype)
    fwd = b.dppf_layer_norm(x, w)
    dw = torch.empty(H, device="cuda")
    b.dppf_layer_norm_grad(dy, x, fwd.mean, fwd.rstd, w, dw, grad_sum=dsum, grad_x=dx)
    want, tol, want_w, tol_w, _, _ = norm_grads(dy, x, fwd.mean, fwd.rstd, w, dsum)
    within(dx, want, tol)
    within(dw, want_w, tol_w)
    dx.fill_(float("nan"))
    assert torch.isnan(storage_of(dx)).all()


def test_norm_of_no_rows_and_shapes(b):
    w = torch.ones(16, device="cuda")
    got = b.dppf_layer_norm(torch.empty(0, 16, device="cuda"), w)
    assert got.out.shape == (0, 16) and got.mean.shape == (0,)
    dw = torch.full((16,), 3.0, device="cuda")
    b.dppf_layer_norm_grad(got.out, got.sum, got.mean, got.rstd, w, dw, accumulate=True)
    assert torch.equal(dw, torch.full_like(dw, 3.0))
    b.dppf_layer_norm_grad(got.out, got.sum, got.mean, got.rstd, w, dw)
    assert torch.equal(dw, torch.zeros_like(dw))
    x = randn((3, 5, 16), 50)
    got = b.dppf_layer_norm(x, w)
    assert got.out.shape == x.shape and got.mean.shape == (3, 5)
    assert b.dppf_layer_norm_grad(x, x, got.mean, got.rstd, w, dw).shape == x.shape
    with pytest.raises(b.DppfError) as e:
        b.dppf_layer_norm(x, w, out=x)
    assert e.value.status == b.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        b.dppf_layer_norm(x, w[:8])
    with pytest.raises(ValueError):
        b.dppf_layer_norm(x, w, sum_out=x)
    with pytest.raises(ValueError):
        b.dppf_layer_norm(x, w, branch=x[:2])
    with pytest.raises(ValueError):
        b.dppf_layer_norm_grad(x, x, got.mean, got.rstd, w, dw, grad_sum=x.to(BF16))


def test_norm_past_32_bits(b):
    T, H = 70_000, 32768                                                        # 2.3e9 elements
    x = torch.zeros(T, H, dtype=BF16, device="cuda")
    x[-2:] = randn((2, H), 51, BF16)
    w = randn(H, 52)
    got = b.dppf_layer_norm(x, w)
    check_norm(b.LayerNorm(got.out[-2:], None, got.mean[-2:], got.rstd[-2:]), x[-2:], w, None, 1e-5)
    assert not got.out[:-2].any()
    dw = torch.empty(H, device="cuda")
    dy = got.out
    dy[:-2] = 1.0
    dx = b.dppf_layer_norm_grad(dy, x, got.mean, got.rstd, w, dw, grad_x=dy)
    assert torch.isfinite(dx[-2:]).all() and torch.isfinite(dw).all() and float(dx[-2:].abs().sum()) > 0


# ---------------------------------------------------------------- rotary positions

def turned(x, positions, freq, scale, interleaved, inverse):
    n = 2 * len(freq)
    a = positions.double()[:, None] * freq * (-1 if inverse else 1)
    c, s = a.cos()[:, None] * scale, a.sin()[:, None] * scale
    out = x.double().clone()
    p, q = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    out[..., p], out[..., q] = x[..., p].double() * c - x[..., q].double() * s, x[..., q].double() * c + x[..., p].double() * s
    tol = torch.zeros_like(out)
    tol[..., p] = tol[..., q] = 6e-7 * abs(scale) * (x[..., p].double().abs() + x[..., q].double().abs())
    return out, tol


@pytest.mark.parametrize("T,heads,D,n", [(1, 1, 2, 2), (5, 3, 64, 64), (1000, 4, 128, 128), (33, 40, 128, 64), (17, 2, 80, 72), (9, 5, 36, 10), (7, 3, 19, 6), (3, 2, 1024, 1024), (2, 1024, 16, 16), (301, 7, 96, 96)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved,inverse,pt", [(False, False, torch.int32), (True, False, torch.int64), (False, True, torch.int64), (True, True, torch.int32)])
def test_rotary(b, T, heads, D, n, dtype, interleaved, inverse, pt):
    x = randn((T, heads, D), 60, dtype)
    positions = torch.randint(-50, 1_000_000, (T,), generator=gen(61), device="cuda").to(pt)
    freq, scale = b.rotary_frequencies(n, scaling="by parts", factor=4.0, original_length=4096)
    want, tol = turned(x, positions, freq, scale, interleaved, inverse)
    got = b.dppf_rotary(x, positions, freq, scale, interleaved, inverse)
    within(got, want, tol)
    assert same_bits(got[..., n:], x[..., n:])
    back = b.dppf_rotary(got.float(), positions, freq, 1 / scale, interleaved, not inverse)      # the inverse undoes it
    assert float((back - got.float().new_tensor(x.double().cpu().numpy())).abs().max()) < (1e-5 if dtype == F32 else 0.04)
    assert b.dppf_rotary(x, positions, freq, scale, interleaved, inverse, out=x) is x and same_bits(x, got)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 3), (4, 8), (2, 2)])
def test_rotary_strides(b, interleaved, dtype, offset, pad):
    """Query heads of fused rows, keys of a tensor [heads, tokens, width]; what lies beside stays."""
    T, heads, D = 37, 5, 32
    freq, _ = b.rotary_frequencies(D)
    positions = torch.arange(T, device="cuda")
    rows = randn((T * (heads * D + 100 + pad) + offset,), 62, dtype)
    q = rows[offset:].view(T, -1)[:, 20:20 + heads * D].unflatten(1, (heads, D))
    before = rows.clone()
    want, tol = turned(q, positions, freq, 1.0, interleaved, False)
    out = torch.full((offset + heads * T * (D + pad),), float("nan"), dtype=dtype, device="cuda")
    view = out[offset:].view(heads, T, D + pad)[:, :, :D].transpose(0, 1)
    b.dppf_rotary(q, positions, freq, interleaved=interleaved, out=view)
    within(view, want, tol)
    assert same_bits(rows, before)
    b.dppf_rotary(q, positions, freq, interleaved=interleaved, out=q)
    assert same_bits(q.contiguous(), view.contiguous())
    q.copy_(before[offset:].view(T, -1)[:, 20:20 + heads * D].unflatten(1, (heads, D)))
    view.fill_(float("nan"))
    assert same_bits(rows, before) and torch.isnan(out).all()


def test_rotary_far_positions_and_refusals(b):
    x = randn((4, 2, 64), 63)
    freq, _ = b.rotary_frequencies(64)
    positions = torch.tensor([2 ** 31 - 1, 10 ** 9, -10 ** 9, 0], device="cuda")
    want, tol = turned(x, positions, freq, 1.0, False, False)
    within(b.dppf_rotary(x, positions, freq), want, tol + 1e-6)                  # 2e9 radians in 64 bits: 2e9 * 2^-52 = 5e-7 off on either side
    assert b.dppf_rotary(x[:0], positions[:0], freq).shape == (0, 2, 64)
    for bad in (dict(x=x[0]), dict(positions=positions[:3]), dict(positions=positions.float()), dict(freq=freq.float()), dict(x=x.half()), dict(out=x[:, :1])):
        a = {"x": x, "positions": positions, "freq": freq, "out": None, **bad}
        with pytest.raises(ValueError):
            b.dppf_rotary(a["x"], a["positions"], a["freq"], out=a["out"])
    for bad in (dict(out=x.transpose(0, 1).reshape(-1)[:512].view(2, 4, 64).transpose(0, 1)), dict(freq=torch.ones(33, dtype=torch.float64, device="cuda")), dict(x=x[:1].expand(4, 2, 64))):
        a = {"x": x, "freq": freq, "out": None, **bad}
        if "out" in bad:
            a["out"] = torch.empty(0, device="cuda").set_(x.untyped_storage(), 64, (3, 2, 64), (128, 64, 1))
            a["x"] = x[:3]
        with pytest.raises(b.DppfError) as e:
            b.dppf_rotary(a["x"], positions[:a["x"].shape[0]], a["freq"], out=a["out"])
        assert e.value.status == b.ERR_INVALID_ARG


def test_block_operators_on_a_side_stream_and_in_a_graph(b):
    T, heads, D = 257, 4, 64
    x, w, pos = randn((T, heads * D), 64, BF16), randn(heads * D, 65, BF16, 0.1, 1.0), torch.arange(T, device="cuda")
    freq, _ = b.rotary_frequencies(D)
    ws = b.alloc_layer_norm_workspace(T, heads * D)
    dw = torch.empty(heads * D, device="cuda")

    def step():
        n = b.dppf_layer_norm(x, w)
        q = b.dppf_rotary(n.out.view(T, heads, D), pos, freq)
        back = b.dppf_rotary(q, pos, freq, inverse=True)
        return q, b.dppf_layer_norm_grad(back.view(T, -1), x, n.mean, n.rstd, w, dw, ws=ws), dw.clone()

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(same_bits(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        x.copy_(randn((T, heads * D), 66, BF16))
        graph.replay()
    fresh = step()
    torch.cuda.synchronize()
    assert all(same_bits(p, q) for p, q in zip(fresh, got))
