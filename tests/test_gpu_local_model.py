"""The operators of a language-model worker's local step on the GPU against plain implementations in 64 bits.

Tolerances (eps = 2^-24, the unit roundoff of fp32; a bf16 result may be half a bf16 spacing, 2^-8 relative, off):
  lookup        one product, rounded once: equal bit for bit
  lookup grad   n products and n sums: (n + 2) eps sum|terms|, plus the rounding of the result's type
  policy        lp = (x_y - max)/T - ln S: differences and products eps each on magnitudes up to |lp| + ln V;
                S from exponentials with 2 ulp each and an argument rounding eps |x - max| log2e, summed in runs of
                at most a few hundred: 1e-6 (2 + |lp|) bounds lp.  A gradient entry inherits lp's error through the
                ratio (relative, times the slope's terms) and its own exponential: 1e-5 relative, plus 4e-6 of the
                row's coefficient, plus the rounding of the result's type
  AdamW         32 bits: a dozen operations, 2e-6 relative to the largest term
                8 bits: codes equal to those of a fixed sequence of rounded fp32 operations
"""
import math

import numpy as np
import pytest
import torch

import local_model_ref as ref
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16)}
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def b():
    return require_gpu()[1]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def strided(rows, cols, stride, offset, dtype, fill=float("nan")):
    """[rows, cols] view with a row stride and a start `offset` elements into its storage; gaps hold `fill`."""
    return torch.full((offset + rows * stride,), fill, dtype=dtype, device="cuda")[offset:].view(rows, stride)[:, :cols]


def storage_of(t):
    return torch.empty(0, dtype=t.dtype, device=t.device).set_(t.untyped_storage())


def same_bits(x, y):
    k = {4: torch.int32, 2: torch.int16, 1: torch.int8}[x.element_size()]
    return torch.equal(x.contiguous().view(k), y.contiguous().view(k))


# ---------------------------------------------------------------- embedding

def some_ids(T, V, dtype, seed, pad=0.2, alike=False):
    g = gen(seed)
    ids = (torch.exp(torch.rand(T, generator=g, device="cuda") * math.log(V + 1)) - 1).long().clamp(0, V - 1)
    if alike:
        ids[:] = V - 1
    u = torch.rand(T, generator=g, device="cuda")
    ids[u < pad / 2] = -1
    ids[(u >= pad / 2) & (u < pad)] = V          # outside on the other side
    return ids.to(dtype)


@pytest.mark.parametrize("T,V,H", [(1, 1, 1), (1, 50, 64), (7, 1000, 8), (333, 77, 257), (65, 513, 1000), (5, 3, 8192), (2000, 300_001, 24), (129, 40, 65536)])
@pytest.mark.parametrize("tt,ot,it", [(F32, F32, torch.int32), (F32, BF16, torch.int64), (BF16, F32, torch.int64), (BF16, BF16, torch.int32)])
def test_lookup_is_the_rounded_product(b, T, V, H, tt, ot, it):
    table = (torch.randn(V, H, generator=gen(1), device="cuda") * 3).to(tt)
    ids = some_ids(T, V, it, 2)
    ok = (ids >= 0) & (ids < V)
    want = torch.where(ok[:, None], table[ids.long().clamp(0, V - 1)].float() * 1.7, 0.0).to(ot)
    assert same_bits(b.dppf_embedding(table, ids, scale=1.7, out_dtype=ot), want)


@pytest.mark.parametrize("stride_t,off_t,stride_o,off_o", [(40, 0, 40, 0), (37, 1, 41, 0), (40, 3, 48, 8), (32, 8, 33, 5)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_lookup_strides_and_offsets(b, stride_t, off_t, stride_o, off_o, dtype):
    V, H, T = 19, 32, 23
    table = strided(V, H, stride_t, off_t, dtype)
    table.copy_(torch.randn(V, H, generator=gen(3), device="cuda"))
    out = strided(T, H, stride_o, off_o, dtype)
    before = storage_of(out).clone()
    ids = some_ids(T, V, torch.int64, 4, pad=0.0)
    b.dppf_embedding(table, ids, scale=0.5, out=out)
    assert same_bits(out, (table[ids].float() * 0.5).to(dtype))
    out.fill_(float("nan"))
    assert torch.isnan(storage_of(out)).all() and torch.isnan(before).all()      # nothing outside out was written


def test_lookup_shapes_and_refusals(b):
    table = torch.randn(11, 16, device="cuda")
    ids = torch.randint(0, 11, (3, 5), device="cuda")
    out = b.dppf_embedding(table, ids)
    assert out.shape == (3, 5, 16) and torch.equal(out, table[ids])
    assert b.dppf_embedding(table, ids[:0]).shape == (0, 5, 16)
    with pytest.raises(ValueError):
        b.dppf_embedding(table, ids.float())
    with pytest.raises(ValueError):
        b.dppf_embedding(table, ids[:, :-1])                 # not contiguous
    with pytest.raises(ValueError):
        b.dppf_embedding(table.half(), ids)
    with pytest.raises(ValueError):
        b.dppf_embedding(table.t(), ids)
    with pytest.raises(ValueError):
        b.dppf_embedding(table, ids, out=torch.empty(15, 17, device="cuda"))
    with pytest.raises(b.DppfError) as e:
        b.dppf_embedding(table, torch.zeros(11, dtype=torch.int64, device="cuda"), out=table)
    assert e.value.status == b.ERR_INVALID_ARG


def test_lookup_offsets_past_32_bits(b):
    V, H = 600_000, 4096                                     # 2.4e9 elements
    table = torch.empty(V, H, dtype=BF16, device="cuda")
    ids = torch.tensor([0, V - 1, 524_289, 599_998], device="cuda")
    table[ids] = torch.randn(4, H, generator=gen(5), device="cuda").to(BF16)
    assert same_bits(b.dppf_embedding(table, ids), table[ids])
    go = torch.randn(4, H, generator=gen(6), device="cuda").to(BF16)
    before = table[ids].float()
    b.dppf_embedding_grad(go, ids, table, accumulate=True)
    assert same_bits(table[ids], (before + go.float()).to(BF16))


def check_grad(b, T, V, H, gt, tt, it, add, seed, scale=0.75, alike=False, pad=0.2):
    ids = some_ids(T, V, it, seed, pad=pad, alike=alike)
    go = torch.randn(T, H, generator=gen(seed + 1), device="cuda").to(gt)
    start = torch.randn(V, H, generator=gen(seed + 2), device="cuda").to(tt) if add else torch.full((V, H), float("nan"), dtype=tt, device="cuda")
    got = start.clone()
    b.dppf_embedding_grad(go, ids, got, scale=scale, accumulate=add)
    want, mags, count = ref.embedding_grad(go, ids, (V, H), scale, start if add else None)
    err = (got.cpu().double() - want).abs()
    bound = (count[:, None] + 3) * EPS * mags + HALF[tt] * want.abs()
    assert bool((err <= bound).all()), float((err - bound).max())
    if add:
        assert same_bits(got[(count == 0).cuda()], start[(count == 0).cuda()])
    else:
        assert bool((got[(count == 0).cuda()] == 0).all())
    again = start.clone()
    b.dppf_embedding_grad(go, ids, again, scale=scale, accumulate=add)
    assert same_bits(got, again)


@pytest.mark.parametrize("T,V,H", [(1, 1, 1), (1, 100, 64), (2, 1, 8), (31, 7, 5), (32, 511, 40), (33, 512, 257), (1000, 50, 16), (2048, 5000, 24), (2049, 5000, 24),
                                   (4097, 262_143, 8), (3000, 300_000, 3), (20_011, 1009, 72)])
@pytest.mark.parametrize("gt,tt,it,add", [(F32, F32, torch.int32, False), (BF16, F32, torch.int64, True), (F32, BF16, torch.int64, False), (BF16, BF16, torch.int32, True)])
def test_lookup_gradient(b, T, V, H, gt, tt, it, add):
    check_grad(b, T, V, H, gt, tt, it, add, seed=T + V + H)


@pytest.mark.parametrize("T,V,H,alike,pad", [(70_001, 40_000, 16, False, 0.1), (70_001, 9, 8, True, 0.0), (5000, 33, 1024, True, 0.5), (400, 20, 64, False, 1.0), (9000, 2, 2056, False, 0.0)])
def test_lookup_gradient_long_alike_and_all_padding(b, T, V, H, alike, pad):
    check_grad(b, T, V, H, BF16, F32, torch.int64, False, seed=7, alike=alike, pad=pad)
    check_grad(b, T, V, H, F32, F32, torch.int32, True, seed=8, alike=alike, pad=pad)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("stride_t,off_t,stride_o,off_o", [(48, 0, 40, 0), (37, 1, 41, 0), (40, 4, 40, 4)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_lookup_gradient_strides(b, add, stride_t, off_t, stride_o, off_o, dtype):
    V, H, T = 37, 32, 150
    ids = some_ids(T, V, torch.int64, 9)
    go = strided(T, H, stride_o, off_o, dtype)
    go.copy_(torch.randn(T, H, generator=gen(10), device="cuda"))
    table = strided(V, H, stride_t, off_t, dtype)
    if add:
        table.copy_(torch.randn(V, H, generator=gen(11), device="cuda"))
    want, mags, count = ref.embedding_grad(go.clone(), ids, (V, H), 1.0, table.clone() if add else None)
    b.dppf_embedding_grad(go, ids, table, accumulate=add)
    err = (table.cpu().double() - want).abs()
    assert bool((err <= (count[:, None] + 3) * EPS * mags + HALF[dtype] * want.abs()).all())
    table.fill_(float("nan"))
    assert torch.isnan(storage_of(table)).all()               # gaps untouched


def test_lookup_gradient_of_no_tokens(b):
    t = torch.full((5, 8), 3.0, device="cuda")
    ids, go = torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, 8, device="cuda")
    assert b.dppf_embedding_grad(go, ids, t, accumulate=True) is None and bool((t == 3).all())
    b.dppf_embedding_grad(go, ids, t)
    assert bool((t == 0).all())


def test_lookup_gradient_against_differences(b):
    V, H, T = 23, 40, 200
    table = torch.randn(V, H, generator=gen(12), device="cuda")
    ids, go = some_ids(T, V, torch.int64, 13), torch.randn(T, H, generator=gen(14), device="cuda")
    grad = torch.empty_like(table)
    b.dppf_embedding_grad(go, ids, grad, scale=1.25)
    d = torch.randn(V, H, generator=gen(15), device="cuda")
    f = lambda s: (b.dppf_embedding(table + s * d, ids, scale=1.25).double() * go.double()).sum()  # noqa: E731
    # linear in the table: the difference carries the roundings of T H products of order 1
    assert abs(float((f(0.5) - f(-0.5)) - (grad.double() * d.double()).sum())) <= T * H * 4 * EPS * 30


def test_lookup_gradient_refusals_and_workspace_reuse(b):
    ids, go, t = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.ones(4, 8, device="cuda"), torch.zeros(3, 8, device="cuda")
    with pytest.raises(b.DppfError) as e:
        b.dppf_embedding_grad(go, ids, t, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == b.ERR_WORKSPACE and bool((t == 0).all())
    with pytest.raises(ValueError):
        b.dppf_embedding_grad(go[:3], ids, t)
    ws = b.alloc_embedding_workspace(5000, 64)
    ws.fill_(0xA5)
    for T in (5000, 4, 700):                                  # one workspace for smaller calls too
        ids = some_ids(T, 40, torch.int64, T)
        go = torch.randn(T, 64, generator=gen(T), device="cuda")
        t = torch.empty(40, 64, device="cuda")
        b.dppf_embedding_grad(go, ids, t, ws=ws)
        want, mags, count = ref.embedding_grad(go, ids, (40, 64), 1.0)
        assert bool(((t.cpu().double() - want).abs() <= (count[:, None] + 3) * EPS * mags + EPS * want.abs()).all())


# ---------------------------------------------------------------- policy loss

def policy_inputs(T, V, dtype, seed, stride=None, offset=0, masked=0.25, spread=3.0, tdtype=torch.int64):
    g = gen(seed)
    x = strided(T, V, stride or V, offset, dtype)
    x.copy_(torch.randn(T, V, generator=g, device="cuda") * spread)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    lp = torch.log_softmax(x.double(), 1).gather(1, y[:, None])[:, 0]
    # ratios from 0.5 to 2, none within 1e-3 of an edge of (0.8, 1.3)
    drift = torch.rand(T, generator=g, device="cuda").double() * 1.4 - 0.7
    for edge in (math.log(0.8), math.log(1.3)):
        drift = torch.where((drift - edge).abs() < 2e-3, drift + 5e-3, drift)
    w = torch.rand(T, generator=g, device="cuda") + 0.5
    dead = torch.rand(T, generator=g, device="cuda") < masked
    w[dead] = 0
    x[dead] = float("nan")                                    # a row that does not count may hold anything
    y[dead] = -100
    adv = torch.randn(T, generator=g, device="cuda")
    adv[::7] = 0
    return dict(logits=x, targets=y.to(tdtype), old=(lp - drift).float(), adv=adv, weight=w / T, ref=(lp + torch.randn(T, generator=g, device="cuda") * 0.5).float())


def check_policy(b, i, kl=True, temperature=1.0, grad=None, backward=True, ws=None):
    x, dtype = i["logits"], i["logits"].dtype
    kw = dict(clip_low=0.2, clip_high=0.3, kl_coef=0.1 if kl else 0.0, temperature=temperature)
    lp1 = torch.log_softmax(x.double(), 1).gather(1, i["targets"].long().clamp(min=0)[:, None])[:, 0]
    lpT = torch.log_softmax(x.double() / temperature, 1).gather(1, i["targets"].long().clamp(min=0)[:, None])[:, 0]
    shift = torch.nan_to_num(lpT - lp1).float()
    old, rf = i["old"] + shift, i["ref"] + shift               # the same ratios at this temperature
    sums, logp, slope, want = ref.policy(x, i["targets"], old, i["adv"], i["weight"], rf if kl else None, **kw)
    if backward and grad is None:
        grad = torch.full_like(x, float("nan"))
    out = b.dppf_policy_loss(x, i["targets"], old, i["adv"], i["weight"], ref_logp=rf if kl else None, grad_logits=grad, ws=ws, **kw)
    assert b.dppf_device_status(out.ws) == b.OK
    live = (i["weight"] != 0).cpu()
    got = out.logp.cpu().double()
    assert bool(((got - logp).abs() <= 1e-6 * (2 + logp.abs()) + 1e-6 * math.log(x.shape[1])).all())
    assert bool((got[~live] == 0).all())
    for k, (a, w) in enumerate(zip((out.loss, out.kl, out.clipped), sums)):
        # each term inherits lp's error times its slope; terms are of order weight * (1 + |adv| 2 + e^gap)
        bound = 4e-5 * float(i["weight"].sum()) * (1.0 if k < 2 else 0.01) + 1e-6 * abs(float(w))
        assert abs(float(a) - float(w)) <= bound, (k, float(a), float(w))
    if grad is not None:
        g = grad.cpu().double()
        c = slope.abs() / temperature
        scale = (i["weight"].cpu().double() * (i["adv"].cpu().double().abs() * 2.2 + (0.1 * 5 if kl else 0))) / temperature
        bound = HALF[dtype] * want.abs() + 1e-5 * want.abs() + (4e-6 * c + 1e-5 * scale)[:, None] * (want.abs() / c.clamp(min=1e-30)[:, None] + 1e-2)
        bad = (g - want).abs() > bound
        assert not bool(bad.any()), (float((g - want).abs().max()), int(bad.sum()))
        assert bool((g[~live] == 0).all())
    return out


@pytest.mark.parametrize("T,V", [(1, 1), (1, 2), (3, 7), (5, 8), (2, 1000), (40, 1009), (17, 4096), (9, 32_000), (3, 50_003), (2, 131_072), (1, 262_144), (300, 2048)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_policy_loss_and_gradient(b, T, V, dtype):
    check_policy(b, policy_inputs(T, V, dtype, seed=T + V, masked=0.25 if T > 2 else 0.0))
    check_policy(b, policy_inputs(T, V, dtype, seed=T + V + 1, masked=0.0, tdtype=torch.int32), kl=False, temperature=0.7)
    check_policy(b, policy_inputs(T, V, dtype, seed=T + V + 2), backward=False, temperature=1.6)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1023, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 4097, 8190])
def test_policy_rows_around_the_size_a_warp_holds(b, V, dtype):
    """128, 256 and 512 vectors of 16 bytes, aligned and not."""
    check_policy(b, policy_inputs(7, V, dtype, seed=V))
    check_policy(b, policy_inputs(7, V, dtype, seed=V + 1, stride=V + 3, offset=1), kl=False, backward=False)


@pytest.mark.parametrize("T,V,stride,dtype", [(400, 70_001, 70_001, BF16), (330, 20_001, 20_003, F32), (600, 9_000, 9_000, BF16)])
def test_policy_forward_streams_long_rows(b, T, V, stride, dtype):
    i = policy_inputs(T, V, dtype, 21, stride=stride)
    out = check_policy(b, i, backward=False)
    kept = b.dppf_policy_loss(i["logits"], i["targets"], i["old"], i["adv"], i["weight"], grad_logits=torch.empty_like(i["logits"]))
    # other slices, another order of the sums: 1e-6 (2 + |lp|), as against the reference
    again = b.dppf_policy_loss(i["logits"], i["targets"], i["old"], i["adv"], i["weight"])
    assert torch.allclose(kept.logp, again.logp, rtol=1e-6, atol=2e-6) and out.logp.shape == (T,)


@pytest.mark.parametrize("stride,offset,gstride,goffset", [(1009, 0, 1009, 0), (1009, 3, 1009, 3), (1016, 0, 1016, 0), (1016, 1, 1016, 0), (1011, 2, 1040, 5), (1024, 0, 1009, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_policy_strides_and_alignment(b, stride, offset, gstride, goffset, dtype):
    i = policy_inputs(13, 1009, dtype, 5, stride=stride, offset=offset)
    grad = strided(13, 1009, gstride, goffset, dtype)
    check_policy(b, i, grad=grad)
    grad.fill_(float("nan"))
    assert torch.isnan(storage_of(grad)).all()                # gaps untouched


@pytest.mark.parametrize("dtype,T,V,stride", [(BF16, 11, 1001, 1001), (F32, 6, 9000, 9008), (BF16, 4, 100_001, 100_001)])
def test_policy_gradient_in_place(b, dtype, T, V, stride):
    i = policy_inputs(T, V, dtype, 6, stride=stride)
    sep = torch.empty_like(i["logits"])
    kw = dict(ref_logp=i["ref"], kl_coef=0.1)
    a = b.dppf_policy_loss(i["logits"], i["targets"], i["old"], i["adv"], i["weight"], grad_logits=sep, **kw)
    c = b.dppf_policy_loss(i["logits"], i["targets"], i["old"], i["adv"], i["weight"], grad_logits=i["logits"], **kw)
    assert same_bits(i["logits"], sep) and same_bits(a.logp, c.logp) and same_bits(a.loss, c.loss)


def test_policy_masks_and_extremes(b):
    T, V = 12, 300
    i = policy_inputs(T, V, F32, 7, masked=0.0)
    x = i["logits"]
    x[0, 5:200] = float("-inf")                               # masked vocabulary
    i["targets"][0] = 250
    x[1, 5:200] = torch.finfo(F32).min                        # ... with the type's lowest value
    i["targets"][1] = 250
    i["targets"][2] = V                                       # outside
    i["targets"][3] = -100
    x[4] = torch.finfo(F32).min                               # a row of nothing but the lowest value is uniform
    x[5] = 1e4
    x[6] = -1e4
    for t in (0, 1, 4, 5, 6):
        lp = torch.log_softmax(x[t].double(), 0)[i["targets"][t]]
        i["old"][t], i["ref"][t] = lp - 0.1, lp + 0.2
    i["weight"][2:4] = 0.3                                    # skipped for the target, not for the weight
    i["weight"][7] = 0
    x[7] = float("inf")
    sums, logp, slope, want = ref.policy(x, i["targets"], i["old"], i["adv"], i["weight"], i["ref"], kl_coef=0.1)
    grad = torch.full_like(x, 9.0)
    out = b.dppf_policy_loss(x, i["targets"], i["old"], i["adv"], i["weight"], ref_logp=i["ref"], kl_coef=0.1, grad_logits=grad)
    assert torch.allclose(out.logp.cpu().double(), logp, rtol=2e-6, atol=4e-6)
    assert torch.allclose(grad.cpu().double(), want, rtol=3e-5, atol=2e-6)
    assert bool((grad[[2, 3, 7]] == 0).all()) and bool((out.logp[[2, 3, 7]] == 0).all()) and bool((grad[0, 5:200] == 0).all())
    assert abs(float(out.loss) - float(sums[0])) < 1e-4
    # rows that have no distribution are NaN, and only they
    x[8, 3], x[9], x[10, 0] = float("nan"), float("-inf"), float("inf")
    out = b.dppf_policy_loss(x, i["targets"], i["old"], i["adv"], i["weight"], grad_logits=grad)
    assert torch.isnan(out.logp[8:11]).all() and torch.isnan(grad[8:11]).any(1).all() and torch.isnan(out.loss)
    assert torch.isfinite(out.logp[:8]).all() and torch.isfinite(grad[:8]).all() and torch.isfinite(grad[11]).all()


@pytest.mark.parametrize("T", [1, 64])
def test_policy_with_every_row_masked(b, T):
    x = torch.full((T, 501), float("nan"), dtype=BF16, device="cuda")
    grad, z = torch.full_like(x, 7.0), torch.zeros(T, device="cuda")
    out = b.dppf_policy_loss(x, torch.full((T,), -100, device="cuda"), z, z + 1, z, ref_logp=z, kl_coef=0.1, grad_logits=grad)
    assert float(out.loss) == 0 and float(out.kl) == 0 and float(out.clipped) == 0
    assert bool((out.logp == 0).all()) and bool((grad == 0).all())


def test_policy_clipping_and_zero_advantage(b):
    """One row of two logits per case: closed forms."""
    p = 0.3
    x = torch.tensor([[math.log(p), math.log(1 - p)]], device="cuda").repeat(6, 1)
    q = torch.tensor([1.5, 1.5, 0.5, 0.5, 1.1, 2.0], device="cuda")
    adv = torch.tensor([1.0, -1.0, 1.0, -1.0, 2.0, 0.0], device="cuda")
    grad = torch.empty_like(x)
    out = b.dppf_policy_loss(x, torch.zeros(6, dtype=torch.int64, device="cuda"), math.log(p) - torch.log(q), adv, torch.ones(6, device="cuda"),
                             clip_low=0.2, clip_high=0.3, grad_logits=grad)
    loss = [-1.3, 1.5, -0.5, 0.8, -2.2, 0.0]
    slope = torch.tensor([0.0, 1.5, -0.5, 0.0, -2.2, 0.0])
    assert abs(float(out.loss) - sum(loss)) < 2e-5 and float(out.clipped) == 2.0 and float(out.kl) == 0
    want = torch.stack([slope * (1 - p), -slope * (1 - p)], 1)
    assert torch.allclose(grad.cpu(), want, rtol=1e-5, atol=1e-6)


def test_policy_gradient_against_differences(b):
    T, V, h = 5, 40, 1e-2
    i = policy_inputs(T, V, F32, 8, masked=0.0, spread=1.0)
    kw = dict(ref_logp=i["ref"], clip_low=0.2, clip_high=0.3, kl_coef=0.1, temperature=1.0)
    f = lambda x: float(b.dppf_policy_loss(x, i["targets"], i["old"], i["adv"], i["weight"], **kw).loss)  # noqa: E731
    grad = torch.empty(T, V, device="cuda")
    b.dppf_policy_loss(i["logits"], i["targets"], i["old"], i["adv"], i["weight"], grad_logits=grad, **kw)
    rng = np.random.default_rng(0)
    for _ in range(12):
        d = torch.from_numpy(rng.standard_normal((T, V)).astype(np.float32) * 0.1).cuda()
        # the step moves log-probabilities by about 1e-3: no ratio (2e-3 from an edge at least) crosses the clip.
        # Loss values carry 1e-6, so the quotient 1e-4; the third-order term is below h^2
        num = (f(i["logits"] + h * d) - f(i["logits"] - h * d)) / (2 * h)
        assert abs(num - float((grad.double() * d.double()).sum())) <= 5e-4


def test_policy_is_reproducible_and_reuses_its_workspace(b):
    ws = b.alloc_policy_workspace(5000)
    for T, V in ((5000, 64), (3, 40_000), (700, 1000)):
        i = policy_inputs(T, V, BF16, 9)
        a = check_policy(b, i, ws=ws)
        c = check_policy(b, i, ws=ws)
        assert same_bits(a.logp, c.logp) and same_bits(a.loss, c.loss)


def test_policy_offsets_past_32_bits(b):
    T, V = 17_000, 131_072                                    # 2.2e9 logits; all rows but a few masked
    x = torch.empty(T, V, dtype=BF16, device="cuda")
    grad = torch.full((T, V), 1.0, dtype=BF16, device="cuda")
    rows = torch.tensor([0, 16_384, 16_385, T - 1], device="cuda")
    i = policy_inputs(4, V, BF16, 10, masked=0.0)
    x[rows] = i["logits"]
    put = lambda v, fill: torch.full((T,), fill, dtype=v.dtype, device="cuda").index_copy_(0, rows, v)  # noqa: E731
    out = b.dppf_policy_loss(x, put(i["targets"], -100), put(i["old"], 0), put(i["adv"], 1), put(i["weight"], 0), grad_logits=grad)
    few = torch.empty_like(i["logits"])
    want = b.dppf_policy_loss(i["logits"], i["targets"], i["old"], i["adv"], i["weight"], grad_logits=few)
    assert torch.allclose(grad[rows].float(), few.float(), rtol=2e-2, atol=1e-7) and torch.allclose(out.logp[rows], want.logp, rtol=1e-5)
    assert float(grad.float().abs().sum(1).count_nonzero()) <= 4 and abs(float(out.loss) - float(want.loss)) < 1e-4


@pytest.mark.parametrize("V,backward", [(40_000, True), (40_000, False), (200_000, False)])
def test_policy_wait_that_gives_up_is_reported(b, V, backward):
    i = policy_inputs(6, V, BF16, 11, masked=0.0)
    grad = torch.empty_like(i["logits"]) if backward else None
    ws = b.alloc_policy_workspace(6)
    try:
        b.debug_set_poll_limits(0, -1)
        out = b.dppf_policy_loss(i["logits"], i["targets"], i["old"], i["adv"], i["weight"], grad_logits=grad, ws=ws)
        status = b.dppf_device_status(ws)
    finally:
        b.debug_set_poll_limits(-1, -1)
    assert status == b.ERR_TIMEOUT and torch.isnan(out.logp).all() and torch.isnan(out.loss)
    check_policy(b, i, ws=ws, backward=backward)               # and the workspace is good again


def test_policy_refusals(b):
    i = policy_inputs(6, 64, BF16, 12)
    args = (i["targets"], i["old"], i["adv"], i["weight"])
    with pytest.raises(ValueError):
        b.dppf_policy_loss(i["logits"].half(), *args)
    with pytest.raises(ValueError):
        b.dppf_policy_loss(i["logits"], i["targets"][:5], *args[1:])
    with pytest.raises(ValueError):
        b.dppf_policy_loss(i["logits"], i["targets"], i["old"].double(), *args[2:])
    with pytest.raises(ValueError):
        b.dppf_policy_loss(i["logits"], *args, grad_logits=torch.empty(6, 64, device="cuda"))
    with pytest.raises(b.DppfError):
        b.dppf_policy_loss(i["logits"], *args, kl_coef=0.1)   # no reference
    with pytest.raises(b.DppfError) as e:
        b.dppf_policy_loss(i["logits"], *args, ws=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == b.ERR_WORKSPACE


# ---------------------------------------------------------------- AdamW over many tensors

HP = dict(lr=5e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
SIZES = [1, 2, 7, 255, 256, 257, 2047, 2048, 2049, 5000, 70_001]


def many(sizes, dtype, seed, std, packed=False):
    """Tensors of the given sizes: views of one row back to back (any alignment), or of their own."""
    g = gen(seed)
    if packed:
        row = torch.randn(sum(sizes) + 1, generator=g, device="cuda").mul(std).to(dtype)[1:]
        return list(row.split(sizes))
    return [torch.randn(n, generator=g, device="cuda").mul(std).to(dtype) for n in sizes]


def test_adamw_tensors_equals_the_packed_step_bit_for_bit(b):
    sizes = SIZES + [123_457]
    d = sum(sizes)
    rows = [b.alloc_rows(1, d) for _ in range(4)]
    rows[0][:, :d] = torch.randn(d, generator=gen(1), device="cuda") * 0.02
    rows[1].zero_(), rows[2].zero_()
    p = [t.clone() for t in rows[0][0, :d].split(sizes)]
    tensors = b.AdamWTensors(p, [torch.zeros_like(t) for t in p])
    for step in (1, 2, 3):
        rows[3][:, :d] = torch.randn(d, generator=gen(step + 1), device="cuda") * 1e-2
        b.dppf_adamw_step(*rows, step=step, d=d, **HP)
        tensors.bind_grads([t.clone() for t in rows[3][0, :d].split(sizes)])
        b.dppf_adamw_tensors(tensors, step=step, **HP)
    for mine, row in zip((p, tensors.exp_avgs, tensors.exp_avg_sqs), rows):
        assert same_bits(torch.cat(mine), row[0, :d])


@pytest.mark.parametrize("pt,gt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("packed", [False, True])
def test_adamw_tensors_32_bits(b, pt, gt, packed):
    p, g = many(SIZES, pt, 2, 0.02, packed), many(SIZES, gt, 3, 1e-2, packed)
    m, v = many(SIZES, F32, 4, 1e-2, packed), [t.square() for t in many(SIZES, F32, 5, 1e-2, packed)]
    decay = [k % 3 / 2 for k in range(len(SIZES))]
    old = [[t.double().cpu().numpy() for t in ts] for ts in (p, g, m, v)]
    tensors = b.AdamWTensors(p, g, exp_avgs=m, exp_avg_sqs=v, decay=decay)
    b.dppf_adamw_tensors(tensors, step=7, grad_scale=torch.tensor([0.25], device="cuda"), **HP)
    for k in range(len(SIZES)):
        wp, wm, wv = ref.adamw(old[0][k], old[1][k] * 0.25, old[2][k], old[3][k], HP["lr"], HP["beta1"], HP["beta2"], HP["eps"], HP["weight_decay"] * decay[k], 7)
        got = p[k].double().cpu().numpy()
        assert np.all(np.abs(got - wp) <= HALF[pt] * np.abs(wp) + 2e-6 * (np.abs(wp) + np.abs(wp - old[0][k])) + 1e-12)
        assert np.all(np.abs(m[k].double().cpu().numpy() - wm) <= 2e-6 * np.abs(old[2][k]) + 1e-6 * np.abs(wm))
        assert np.all(np.abs(v[k].double().cpu().numpy() - wv) <= 1e-6 * np.abs(wv))


@pytest.mark.parametrize("pt,gt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("packed", [False, True])
def test_adamw_tensors_8_bits(b, pt, gt, packed):
    """Two steps from zero state: codes and scales are those of the plain fp32 sequence bit for bit, parameters those
    of the formula in 64 bits on the states before the step."""
    p, g = many(SIZES, pt, 6, 0.02, packed), many(SIZES, gt, 7, 1e-2, packed)
    for t in g:                                                # magnitudes over many orders, and exact zeros
        t.copy_((t.float() * torch.exp(torch.randn(t.shape, generator=gen(8), device="cuda") * 3)).to(gt))
        t[::5] = 0
    state = {}
    if packed:
        odd = lambda n: torch.zeros(n + 1, dtype=torch.uint8, device="cuda")[1:].view(torch.float8_e4m3fn)  # noqa: E731
        state = dict(exp_avgs=[odd(n) for n in SIZES], exp_avg_sqs=[odd(n) for n in SIZES])
    tensors = b.AdamWTensors(p, g, state_bits=8, **state)
    codes = lambda t: t.view(torch.uint8).cpu().numpy()  # noqa: E731
    for step in (1, 2):
        old = [t.double().cpu().numpy() for t in p]
        st = [(codes(tensors.exp_avgs[k]), codes(tensors.exp_avg_sqs[k]), tensors.exp_avg_scales[k].cpu().numpy(), tensors.exp_avg_sq_scales[k].cpu().numpy())
              for k in range(len(SIZES))]
        b.dppf_adamw_tensors(tensors, step=step, seed=step + 40, **HP)
        for k, n in enumerate(SIZES):
            gk = g[k].float().cpu().numpy()
            mc, rc, ms, rs = st[k]
            wm, wms, wr, wrs = ref.adamw8_states(gk, mc, rc, ms, rs, HP["beta1"], HP["beta2"], step + 40)
            assert np.array_equal(codes(tensors.exp_avgs[k]), wm) and np.array_equal(codes(tensors.exp_avg_sqs[k]), wr)
            assert np.array_equal(tensors.exp_avg_scales[k].cpu().numpy(), wms) and np.array_equal(tensors.exp_avg_sq_scales[k].cpu().numpy(), wrs)
            m64, v64 = ref.decode(mc, ms, n), ref.decode(rc, rs, n) ** 2
            wp, nm, nv = ref.adamw(old[k], gk.astype(np.float64), m64, v64, step=step, **HP)
            got = p[k].double().cpu().numpy()
            assert np.all(np.abs(got - wp) <= HALF[pt] * np.abs(wp) + 2e-6 * (np.abs(wp) + np.abs(wp - old[k])) + 1e-9)
            # and the stored moments are within e4m3's spacing of the formula's
            for x, code, sc, part in ((nm, wm, wms, 0.5), (np.sqrt(nv), wr, wrs, 1.0)):
                y = ref.blocks_of(x) / np.where(sc > 0, sc, 1)[:, None]
                d = np.abs(ref.E4M3[ref.blocks_of(code)] - y)
                assert np.all(d <= part * ref.spacing(y) * 1.001 + 1e-5 * np.abs(y))
            assert np.all((wr > 0) == (nv > 0))


def test_adamw_tensors_8_bits_follow_a_falling_gradient(b):
    """beta2 = 0.999 moves sqrt(v) by 5e-4 a step, a hundredth of e4m3's spacing: rounded in proportion it still
    falls as it should.  A few elements keep the block's scale up."""
    n, steps = 256 * 64, 1500
    g = torch.full((n,), 1e-2, device="cuda")
    p = torch.zeros(n, device="cuda")
    t8, t32 = b.AdamWTensors([p.clone()], [g], state_bits=8), b.AdamWTensors([p.clone()], [g])
    low = torch.ones(n, dtype=torch.bool, device="cuda")
    low[::64] = False
    for step in range(1, steps + 1):
        if step == 300:
            g[low] = 1e-4
        for t in (t8, t32):
            b.dppf_adamw_tensors(t, step=step, seed=step, **HP)
    r8 = (t8.exp_avg_sqs[0].float().view(-1, 256) * t8.exp_avg_sq_scales[0][:, None]).view(-1)
    r32 = t32.exp_avg_sqs[0].sqrt()
    # 1,200 steps shrink the root to e^-0.6 = 0.55 of its value. An element's random walk has a relative deviation below 0.5; the mean of 16,000 is within 5 %
    assert abs(float(r8[low].mean() / r32[low].mean()) - 1) < 0.05
    assert abs(float(r8[~low].mean() / r32[~low].mean()) - 1) < 0.02


def test_adamw_tensors_step_is_skipped_for_a_scale_that_is_not_finite(b):
    for bits in (8, 32):
        p, g = many(SIZES, F32, 9, 0.02), many(SIZES, F32, 10, 1e-2)
        t = b.AdamWTensors(p, g, state_bits=bits)
        b.dppf_adamw_tensors(t, step=1, **HP)
        keep = [x.clone() for x in (*p, *t.exp_avgs, *t.exp_avg_sqs)]
        for bad in (float("nan"), float("inf")):
            b.dppf_adamw_tensors(t, step=2, grad_scale=torch.tensor([bad], device="cuda"), **HP)
        assert all(same_bits(x, y) for x, y in zip(keep, (*p, *t.exp_avgs, *t.exp_avg_sqs)))


def test_adamw_tensors_zero_and_bad_gradients_in_8_bits(b):
    p, g = torch.ones(600, device="cuda"), torch.zeros(600, device="cuda")
    t = b.AdamWTensors([p], [g], state_bits=8, decay=[0.0])
    b.dppf_adamw_tensors(t, step=1, **HP)
    assert bool((p == 1).all()) and not t.exp_avgs[0].view(torch.uint8).any() and not t.exp_avg_sq_scales[0].any()
    g.fill_(1e-3)
    g[300] = float("inf")
    b.dppf_adamw_tensors(t, step=2, **HP)
    assert torch.isfinite(p[:256]).all() and torch.isfinite(p[512:]).all() and torch.isfinite(t.exp_avg_scales[0][[0, 2]]).all()
    assert not torch.isfinite(p[300]) and not torch.isfinite(t.exp_avg_scales[0][1])


@pytest.mark.parametrize("count", [1, 60, 61, 500, 501, 1203])
def test_adamw_tensors_many_of_them(b, count):
    sizes = [1 + (k * 37) % 700 for k in range(count)]
    sizes[count // 2] = 0                                      # skipped
    if count == 1:
        sizes = [5]
    d = sum(sizes)
    p, g = many(sizes, F32, 11, 0.02, True), many(sizes, F32, 12, 1e-2, True)
    q = torch.cat(p).clone()
    t, one = b.AdamWTensors(p, g), b.AdamWTensors([q], [torch.cat(g)])
    for x in (t, one):
        b.dppf_adamw_tensors(x, step=1, **HP)
    assert same_bits(torch.cat(p), q) and q.numel() == d
    assert same_bits(torch.cat(t.exp_avg_sqs), one.exp_avg_sqs[0])


def test_adamw_tensors_offsets_past_32_bits(b):
    n = (1 << 32) + 777
    p, g = torch.full((n,), 0.5, dtype=BF16, device="cuda"), torch.full((n,), 1e-3, dtype=BF16, device="cuda")
    t = b.AdamWTensors([p], [g], state_bits=8)
    b.dppf_adamw_tensors(t, lr=0.1, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1)
    for part in (p[:5000], p[(1 << 31) - 5000:(1 << 31) + 5000], p[-5000:]):
        assert bool((part == torch.tensor(0.4).to(BF16)).all())    # 0.5 - lr
    assert bool((t.exp_avgs[0].view(torch.uint8)[-1000:] == 0x7E).all())


def test_adamw_tensors_refusals(b):
    p, g = torch.zeros(10, device="cuda"), torch.zeros(10, device="cuda")
    for bad in (lambda: b.AdamWTensors([p], [g[:9]]), lambda: b.AdamWTensors([p], [g.half()]), lambda: b.AdamWTensors([p, p.to(BF16)], [g, g]),
                lambda: b.AdamWTensors([p], [g], exp_avgs=[torch.zeros(10, dtype=BF16, device="cuda")]), lambda: b.AdamWTensors([p], [g], decay=[1, 2]),
                lambda: b.AdamWTensors([p], [g, g]), lambda: b.AdamWTensors([p.expand(10)[::2]], [g[::2]]),
                lambda: b.dppf_adamw_tensors(b.AdamWTensors([p], [g]), grad_scale=torch.ones(2, device="cuda"), step=1, **HP)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(b.DppfError) as e:
        b.dppf_adamw_tensors(b.AdamWTensors([p], [p]), step=1, **HP)
    assert e.value.status == b.ERR_INVALID_ARG


# ---------------------------------------------------------------- streams and graphs

def test_operators_on_a_side_stream_and_in_a_graph(b):
    T, V, H = 90, 700, 64
    i = policy_inputs(T, V, BF16, 13)
    ids = some_ids(T, V, torch.int64, 14)
    table, go = torch.randn(V, H, generator=gen(15), device="cuda"), torch.randn(T, H, generator=gen(16), device="cuda")
    out, gt, gx = torch.empty(T, H, device="cuda"), torch.empty(V, H, device="cuda"), torch.empty_like(i["logits"])
    p, g = many(SIZES, F32, 17, 0.02), many(SIZES, F32, 18, 1e-2)
    start = [t.clone() for t in p]
    tensors = b.AdamWTensors(p, g, state_bits=8)
    ws_e, ws_p = b.alloc_embedding_workspace(T, H), b.alloc_policy_workspace(T)
    res = {}

    def step():
        b.dppf_embedding(table, ids, out=out)
        b.dppf_embedding_grad(go, ids, gt, ws=ws_e)
        res["loss"] = b.dppf_policy_loss(i["logits"], i["targets"], i["old"], i["adv"], i["weight"], grad_logits=gx, ws=ws_p).loss
        b.dppf_adamw_tensors(tensors, step=1, seed=3, **HP)

    def reset():
        for t in (out, gt, gx):
            t.fill_(float("nan"))
        for t, s in zip(p, start):
            t.copy_(s)
        for t in (*tensors.exp_avgs, *tensors.exp_avg_sqs):
            t.view(torch.uint8).zero_()
        for t in (*tensors.exp_avg_scales, *tensors.exp_avg_sq_scales):
            t.zero_()

    def answers():
        torch.cuda.synchronize()
        return [t.clone() for t in (out, gt, gx, res["loss"], *p, *tensors.exp_avg_sqs)]

    step()
    plain = answers()
    assert torch.isfinite(plain[1]).all()
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    other = answers()
    assert all(same_bits(x, y) for x, y in zip(plain, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        reset()
        graph.replay()
        assert all(same_bits(x, y) for x, y in zip(plain, answers()))


def test_longer_paths_on_a_side_stream_and_in_a_graph(b):
    """The gradient's chain of launches (sort, sums, joins), rows split over a cluster, rows streamed forward."""
    T, V, H = 5000, 3000 + 71, 136
    ids, go = some_ids(T, V, torch.int64, 31), torch.randn(T, H, generator=gen(32), device="cuda").to(BF16)
    whole, added = torch.empty(V, H, device="cuda"), torch.zeros(V, H, dtype=BF16, device="cuda")
    i, j = policy_inputs(24, 60_001, BF16, 33), policy_inputs(700, 50_000, BF16, 34)
    gx = torch.empty_like(i["logits"])
    ws_e, ws_p = b.alloc_embedding_workspace(T, H), b.alloc_policy_workspace(700)
    res = {}

    def step():
        b.dppf_embedding_grad(go, ids, whole, ws=ws_e)
        b.dppf_embedding_grad(go, ids, added, accumulate=True, ws=ws_e)
        res["a"] = b.dppf_policy_loss(i["logits"], i["targets"], i["old"], i["adv"], i["weight"], grad_logits=gx, ws=ws_p).logp
        res["b"] = b.dppf_policy_loss(j["logits"], j["targets"], j["old"], j["adv"], j["weight"], ws=ws_p).loss

    def answers():
        torch.cuda.synchronize()
        out = [t.clone() for t in (whole, added, gx, res["a"], res["b"])]
        whole.fill_(float("nan")), gx.fill_(float("nan")), added.zero_()
        return out

    step()
    plain = answers()
    assert torch.isfinite(plain[0]).all() and torch.isfinite(plain[4])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    assert all(same_bits(x, y) for x, y in zip(plain, answers()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        graph.replay()
        assert all(same_bits(x, y) for x, y in zip(plain, answers()))


# ---------------------------------------------------------------- seeded random shapes

@pytest.mark.parametrize("seed", range(12))
def test_random_shapes(b, seed):
    rng = np.random.default_rng(seed)
    size = lambda low, high: int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))  # noqa: E731
    pick = lambda *x: x[rng.integers(len(x))]  # noqa: E731
    for _ in range(4):
        check_grad(b, size(1, 30_000), size(1, 20_000), size(1, 700), pick(F32, BF16), pick(F32, BF16), pick(torch.int32, torch.int64), bool(rng.integers(2)), seed=size(1, 10_000))
        V = size(2, 150_000)
        T = size(1, max(2, min(400, 3_000_000 // V)))
        i = policy_inputs(T, V, pick(F32, BF16), size(1, 10_000), stride=V + int(rng.integers(0, 20)), offset=int(rng.integers(0, 9)), masked=pick(0.0, 0.3, 0.8))
        check_policy(b, i, kl=bool(rng.integers(2)), temperature=pick(0.6, 1.0, 1.7), backward=bool(rng.integers(2)))
    # many tensors at random offsets of one row, 8-bit states: the plain sequence's codes
    sizes = [size(1, 5000) for _ in range(pick(3, 40, 90))]
    lead = int(rng.integers(0, 9))
    g = gen(seed)
    rows = [torch.randn(lead + sum(sizes), generator=g, device="cuda")[lead:] * s for s in (0.02, 1e-2)]
    p, gr = list(rows[0].split(sizes)), list(rows[1].to(pick(F32, BF16)).split(sizes))
    t = b.AdamWTensors(p, gr, state_bits=8)
    for step in (1, 2):
        st = [(t.exp_avgs[k].view(torch.uint8).cpu().numpy(), t.exp_avg_sqs[k].view(torch.uint8).cpu().numpy(), t.exp_avg_scales[k].cpu().numpy(),
               t.exp_avg_sq_scales[k].cpu().numpy()) for k in range(len(sizes))]
        old = [x.double().cpu().numpy() for x in p]
        b.dppf_adamw_tensors(t, step=step, seed=seed + step, **HP)
        for k, n in enumerate(sizes):
            gk = gr[k].float().cpu().numpy()
            wm, wms, wr, wrs = ref.adamw8_states(gk, *st[k], HP["beta1"], HP["beta2"], seed + step)
            assert np.array_equal(t.exp_avgs[k].view(torch.uint8).cpu().numpy(), wm) and np.array_equal(t.exp_avg_sqs[k].view(torch.uint8).cpu().numpy(), wr)
            assert np.array_equal(t.exp_avg_scales[k].cpu().numpy(), wms) and np.array_equal(t.exp_avg_sq_scales[k].cpu().numpy(), wrs)
            wp, _, _ = ref.adamw(old[k], gk.astype(np.float64), ref.decode(st[k][0], st[k][2], n), ref.decode(st[k][1], st[k][3], n) ** 2, step=step, **HP)
            got = p[k].double().cpu().numpy()
            assert np.all(np.abs(got - wp) <= EPS * np.abs(wp) + 2e-6 * (np.abs(wp) + np.abs(wp - old[k])) + 1e-9)
