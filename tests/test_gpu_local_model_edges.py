"""Orders, extremes and longer paths of a local step's operators on the GPU (the plain cases are in test_gpu_local_model.py)."""
import numpy as np
import pytest
import torch

import local_model_ref as ref
from gpu_util import require_gpu
from test_gpu_local_model import BF16, EPS, F32, HALF, HP, check_grad, check_policy, gen, policy_inputs, same_bits, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    return require_gpu()[1]


# ---------------------------------------------------------------- embedding gradient

@pytest.mark.parametrize("T", [140_000, 600_001])
@pytest.mark.parametrize("V,H,alike", [(300, 3, False), (40_000, 8, False), (300_000, 2, False), (5000, 8, True)])
def test_lookup_gradient_sorts_long_sequences(b, T, V, H, alike):
    """A warp of the sort has more than 32 places, and more than it holds in registers; one, two and three digits."""
    check_grad(b, T, V, H, F32, F32, torch.int64, False, seed=T + V, alike=alike)
    check_grad(b, T, V, H, BF16, BF16, torch.int32, True, seed=T + V + 1, alike=alike)


def large_ids(kind, T, V, seed):
    g = gen(seed)
    if kind == "padding":
        return torch.full((T,), -1, device="cuda")
    if kind == "dense":                                        # every row, or every so manieth, once or more
        return (torch.randperm(T, generator=g, device="cuda") * V // T).clamp(max=V - 1)
    if kind == "ends":                                         # a few rows at the table's ends and where its stretches meet
        at = torch.tensor([0, 1, V // 4, V // 2, V - 20_000, V - 2, V - 1], device="cuda").clamp(min=0)
        return at[torch.randint(0, len(at), (T,), generator=g, device="cuda")]
    return (torch.exp(torch.rand(T, generator=g, device="cuda") * np.log(V + 1)) - 1).long().clamp(0, V - 1)


@pytest.mark.parametrize("kind", ["dense", "some", "ends", "padding"])
@pytest.mark.parametrize("T,V,H,ld,gt,tt", [(3000, 50_000, 1024, 1024, BF16, F32), (3001, 50_000, 1021, 1021, F32, F32), (1000, 300_007, 200, 208, F32, F32), (60_000, 60_000, 1024, 1024, BF16, BF16),
                                            (70_000, 70_000, 513, 515, F32, BF16), (600, 400, 65_536, 65_536, BF16, F32)])
def test_lookup_gradient_writes_every_row_of_a_large_table(b, kind, T, V, H, ld, gt, tt):
    """Tables of more bytes than are zeroed beside the sort and the joins: rows are zeroed beside the sums too, except where their
    ids occur."""
    ids, go = large_ids(kind, T, V, T + H), torch.randn(T, H, generator=gen(T), device="cuda").to(gt)
    table = torch.full((V, ld), float("nan"), dtype=tt, device="cuda")
    b.dppf_embedding_grad(go, ids, table[:, :H], scale=0.75)
    assert torch.isnan(table[:, H:]).all()
    ok = ids >= 0
    count = torch.bincount(ids[ok], minlength=V)
    for a in range(0, V, 20_000):                              # a stretch of rows at a time
        n = min(20_000, V - a)
        here = ok & (ids >= a) & (ids < a + n)
        rows = go[here].double() * 0.75
        want, mags = (torch.zeros(n, H, dtype=torch.float64, device="cuda").index_add_(0, ids[here] - a, x) for x in (rows, rows.abs()))
        got, c = table[a:a + n, :H].double(), count[a:a + n, None]
        assert bool(((got - want).abs() <= (c + 3) * EPS * mags + HALF[tt] * want.abs()).all())
        assert bool((got[c[:, 0] == 0] == 0).all())


# ---------------------------------------------------------------- policy loss

def edge_targets(V, count, seed):
    """Targets at the row's ends, around the ends of halves, quarters and eighths of it, and anywhere."""
    at = [0, 1, V - 2, V - 1] + [min(max(V * k // 8 + o, 0), V - 1) for k in range(1, 8) for o in range(-9, 10)]
    some = torch.randint(0, V, (count,), generator=gen(seed), device="cuda")
    n = min(count, len(at))
    some[:n] = torch.tensor(at[:n], device="cuda")
    return some


@pytest.mark.parametrize("dtype,T,V,stride", [(BF16, 700, 131_072, 131_072), (BF16, 500, 100_001, 100_001), (F32, 300, 74_003, 74_003), (F32, 150, 262_144, 262_144), (BF16, 9, 32_000, 32_000)])
def test_policy_gradient_in_place_over_clusters(b, dtype, T, V, stride):
    """The gradient replaces the logits while the blocks of a row's cluster still need the target's logit."""
    i = policy_inputs(T, V, dtype, 41, stride=stride, masked=0.0)
    i["targets"] = edge_targets(V, T, 42)
    i["old"] = torch.log_softmax(i["logits"].float(), 1).gather(1, i["targets"][:, None])[:, 0]
    keep, sep = i["logits"].clone(), torch.empty_like(i["logits"])
    args = (i["targets"], i["old"], i["adv"], i["weight"])
    a = b.dppf_policy_loss(keep, *args, grad_logits=sep)
    for _ in range(3):
        i["logits"].copy_(keep)
        c = b.dppf_policy_loss(i["logits"], *args, grad_logits=i["logits"])
        assert same_bits(i["logits"], sep) and same_bits(a.logp, c.logp) and same_bits(a.loss, c.loss)
    assert torch.allclose(a.logp, i["old"], rtol=0, atol=8e-5)    # two fp32 log-softmaxes, 1e-6 (2 + |lp| + log V) each


@pytest.mark.parametrize("stride,offset,gstride,goffset", [(100_001, 0, 100_008, 1), (100_008, 3, 100_001, 3), (100_008, 8, 100_016, 0)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_policy_gradient_rows_laid_out_otherwise_over_clusters(b, stride, offset, gstride, goffset, dtype):
    i = policy_inputs(7, 100_001, dtype, 47, stride=stride, offset=offset)
    grad = strided(7, 100_001, gstride, goffset, dtype)
    check_policy(b, i, grad=grad)
    grad.fill_(float("nan"))
    assert torch.isnan(torch.empty(0, dtype=dtype, device="cuda").set_(grad.untyped_storage())).all()      # gaps untouched


def test_policy_loss_of_no_tokens(b):
    x, z = torch.empty(0, 70, dtype=BF16, device="cuda"), torch.empty(0, device="cuda")
    y = torch.empty(0, dtype=torch.int64, device="cuda")
    for ws in (None, b.alloc_policy_workspace(5)):
        out = b.dppf_policy_loss(x, y, z, z, z, ref_logp=z, kl_coef=0.1, grad_logits=x, ws=ws)
        assert float(out.loss) == 0 and float(out.kl) == 0 and float(out.clipped) == 0 and out.logp.shape == (0,) and out.ws is ws
    with pytest.raises(ValueError):
        b.dppf_policy_loss(x, y, z, z, torch.empty(1, device="cuda"))


@pytest.mark.parametrize("polls", [0, 1, 2])
def test_policy_rows_through_the_ring_give_up_soon(b, polls):
    """A block whose threads disagree on whether a copy arrived in time waits for the copies that were started, and no others
    (for one that never was, the wait would run to its limit of about a second)."""
    i = policy_inputs(600, 131_072, BF16, 43, masked=0.0)
    args = (i["logits"], i["targets"], i["old"], i["adv"], i["weight"])
    good = b.dppf_policy_loss(*args)
    ws, a, z = b.alloc_policy_workspace(600), torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    try:
        b.debug_set_poll_limits(polls, -1)
        a.record()
        out = b.dppf_policy_loss(*args, ws=ws)
        z.record()
        status = b.dppf_device_status(ws)
    finally:
        b.debug_set_poll_limits(-1, -1)
    late = torch.isnan(out.logp)
    assert status == (b.ERR_TIMEOUT if bool(late.any()) else b.OK) and (polls or bool(late.all()))
    assert same_bits(out.logp[~late], good.logp[~late]) and a.elapsed_time(z) < 100
    again = b.dppf_policy_loss(*args, ws=ws)
    assert same_bits(again.logp, good.logp) and same_bits(again.loss, good.loss)


@pytest.mark.parametrize("dtype,T,V,stride", [(BF16, 20_000, 1000, 1000), (F32, 5000, 1021, 1025), (BF16, 9000, 257, 259), (F32, 3000, 4001, 4001)])
def test_policy_gradient_in_place_of_short_rows(b, dtype, T, V, stride):
    i = policy_inputs(T, V, dtype, 48, stride=stride)
    live = i["weight"] != 0
    i["targets"][live] = edge_targets(V, int(live.sum()), 49)
    keep, sep = strided(T, V, stride, 0, dtype), torch.empty_like(i["logits"])
    keep.copy_(i["logits"])
    args = (i["targets"], i["old"], i["adv"], i["weight"])
    a = b.dppf_policy_loss(keep, *args, grad_logits=sep)
    for _ in range(3):
        i["logits"].copy_(keep)
        c = b.dppf_policy_loss(i["logits"], *args, grad_logits=i["logits"])
        assert same_bits(i["logits"], sep) and same_bits(a.logp, c.logp) and same_bits(a.loss, c.loss)


@pytest.mark.parametrize("V", [300, 9000, 40_000])
def test_policy_kl_that_is_only_watched_leaves_loss_and_gradient_alone(b, V):
    """kl_coef 0 with reference log-probabilities: however far they are away, the KL estimate alone shows it."""
    i = policy_inputs(6, V, F32, 44, masked=0.0)
    i["adv"][:] = torch.tensor([1.0, -1.0, 0.5, 2.0, 0.0, -0.3])
    i["ref"][1] = i["old"][1] + 130.0                         # e^gap is beyond fp32
    i["logits"][3, i["targets"][3]] = float("-inf")           # a target of probability 0
    i["ref"][4] = float("-inf")
    args, grads = (i["logits"], i["targets"], i["old"], i["adv"], i["weight"]), [torch.empty_like(i["logits"]) for _ in range(3)]
    plain = b.dppf_policy_loss(*args, grad_logits=grads[0])
    out = b.dppf_policy_loss(*args, ref_logp=i["ref"], kl_coef=0.0, grad_logits=grads[1])
    assert same_bits(out.loss, plain.loss) and same_bits(out.logp, plain.logp) and same_bits(*grads[:2])
    assert torch.isfinite(out.loss) and torch.isfinite(grads[1]).all() and float(out.kl) == float("inf")
    near = torch.where(torch.isfinite(i["ref"]), i["ref"], i["old"])
    near[1], near[3] = i["old"][1], i["old"][3]
    counted = b.dppf_policy_loss(*args, ref_logp=near, kl_coef=0.1, grad_logits=grads[2])      # only the row of probability 0 is infinitely far
    assert float(counted.kl) == float("inf") and float(counted.loss) == float("inf")
    assert torch.isfinite(grads[2][[0, 1, 2, 4, 5]]).all()


@pytest.mark.parametrize("V", [300, 9000, 40_000])
@pytest.mark.parametrize("temperature", [1e30, 1e38, 1.7e38, 2.2e38, 3e38, 1e-38, 4.3e-39])
def test_policy_at_extreme_temperatures(b, V, temperature):
    """Towards infinity every logit above -inf is equally likely, towards zero the largest alone is."""
    T = 4
    x = (torch.randn(T, V, generator=gen(45), device="cuda") * 3).clamp(max=11)
    x[:, ::3] = float("-inf")
    y = torch.tensor([1, 2, 4, V - 1 if (V - 1) % 3 else V - 2], device="cuda")
    if temperature < 1:
        x[torch.arange(T), y] = 12.0
    want = -np.log(V - len(range(0, V, 3))) if temperature > 1 else 0.0
    one, grad = torch.ones(T, device="cuda"), torch.empty_like(x)
    out = b.dppf_policy_loss(x, y, torch.full((T,), float(want), device="cuda"), one, one, temperature=temperature, grad_logits=grad)
    assert torch.allclose(out.logp.cpu().double(), torch.full((T,), want, dtype=torch.float64), rtol=2e-6, atol=1e-6)
    # e^lp - 1 at the target, e^lp elsewhere, over the temperature (fp32 has three digits left of 1e-38 / 200)
    if 1 < temperature < 1e31:
        p = np.exp(want)
        d = torch.where(torch.isfinite(x), -p, 0.0).double()
        d[torch.arange(T), y] += 1.0
        assert torch.allclose(grad.double(), -d / temperature, rtol=1e-5, atol=0)
    elif temperature > 1:
        assert torch.isfinite(grad).all()


@pytest.mark.parametrize("V", [1000, 9000, 40_000])
def test_policy_gradient_far_below_the_maximum(b, V):
    """Entries of e^-30 to e^-44 of the largest, at a temperature whose log2(e)/T lies just below an fp32 number (with a
    significand near 1, where a whole step is 1.2e-7).  Relative error by the formula's steps: half a step of the exponent
    below 64, 2^-19 log 2 = 1.32e-6; log2(e)/T to the nearest number, here 0.05 steps, 44 * 6e-9 = 2.6e-7; the exponential
    2^-22 = 2.4e-7; the row's coefficient and the product four roundings, 2.4e-7: 2.1e-6 in all."""
    temps = np.arange(np.float32(1.4421), np.float32(1.4426), np.float32(2.0) ** -23, dtype=np.float64).astype(np.float32)
    k = 1.4426950408889634 / temps.astype(np.float64)
    steps = (k - 1.0) * 2.0 ** 23
    temps = temps[(steps % 1.0 > 0.95) & (steps % 1.0 < 0.99)][:4]
    assert len(temps) == 4
    for n, T in enumerate(temps.tolist()):
        x = -(30 + 14 * torch.rand(1, V, generator=gen(46 + n), device="cuda")) * T
        x[0, 17] = 0.0
        one, grad = torch.ones(1, device="cuda"), torch.empty_like(x)
        b.dppf_policy_loss(x, torch.tensor([17], device="cuda"), torch.zeros(1, device="cuda"), one, one, temperature=T, grad_logits=grad)
        want = torch.exp(x.double() / T - torch.logsumexp(x.double() / T, 1, keepdim=True)) / T
        off = ((grad.double() - want).abs() / want)[0]
        off[17] = 0
        assert float(off.max()) <= 2.1e-6, float(off.max())


# ---------------------------------------------------------------- AdamW over many tensors

def test_adamw_tensors_keep_the_memory_that_they_write(b):
    n = 5_000_000                                              # blocks of their own in the allocator
    p, g, m, v = (torch.full((n,), x, device="cuda") for x in (1.0, 0.5, 0.0, 0.0))
    t = b.AdamWTensors([p], [g], exp_avgs=[m], exp_avg_sqs=[v])
    keep = {x.data_ptr() for x in (p, g, m, v)}
    for x in (p, g, m, v):
        x.data = torch.zeros(1, device="cuda")                 # other memory; the old would be free
    others = [torch.full((n,), 7.0, device="cuda") for _ in range(8)]
    assert not keep & {x.data_ptr() for x in others}
    b.dppf_adamw_tensors(t, 0.1, 0.9, 0.999, 1e-8, 0.0, 1)
    assert all(bool((x == 7).all()) for x in others)
    del t
    assert keep & {torch.empty(n, device="cuda").data_ptr() for _ in range(1)}                # and lets it go with the object


@pytest.mark.parametrize("size", [1e-22, 1e-20, 1e-19, 2e-18, 1e-17, 1e-16, 1e-15, 1e-12, 1e-9, 1e-8, 1e-6])
@pytest.mark.parametrize("shift,spread", [(0, False), (1, False), (0, True)])
@pytest.mark.parametrize("eps", [1e-30, 1e-8])
def test_adamw_tensors_8_bits_of_tiny_gradients(b, size, shift, spread, eps):
    """Second moments below the smallest normal number: codes and scales are the plain fp32 sequence's bit for bit, and the
    update is that of its moments (rounded operations: 2e-6 relative, as for the other sizes)."""
    n, f = 5000, np.float32
    hp = dict(HP, eps=eps, weight_decay=0.0)
    g = (torch.randn(n + shift, generator=gen(51), device="cuda") * size)[shift:]
    if spread:                                                 # within a block, over twenty orders of magnitude
        g *= torch.exp(-46 * torch.rand(n, generator=gen(52), device="cuda"))
    p = torch.zeros(n + shift, device="cuda")[shift:]
    t = b.AdamWTensors([p], [g], state_bits=8)
    codes = lambda x: x.view(torch.uint8).cpu().numpy()  # noqa: E731
    for step in (1, 2, 3):
        old = codes(t.exp_avgs[0]), codes(t.exp_avg_sqs[0]), t.exp_avg_scales[0].cpu().numpy(), t.exp_avg_sq_scales[0].cpu().numpy()
        p.zero_()
        b.dppf_adamw_tensors(t, step=step, seed=step, **hp)
        gk = g.cpu().numpy()
        want = ref.adamw8_states(gk, *old, HP["beta1"], HP["beta2"], step)
        for got, w in zip((codes(t.exp_avgs[0]), t.exp_avg_scales[0].cpu().numpy(), codes(t.exp_avg_sqs[0]), t.exp_avg_sq_scales[0].cpu().numpy()), want):
            assert np.array_equal(got, w)
        gb, b1, b2 = ref.blocks_of(gk), f(HP["beta1"]), f(HP["beta2"])
        m = ref.blocks_of(ref.E4M3[old[0]].astype(f)) * old[2][:, None] * b1 + gb * f(1 - float(b1))
        root = ref.blocks_of(ref.E4M3[old[1]].astype(f)) * old[3][:, None]
        r = np.sqrt(root * root * b2 + gb * gb * f(1 - float(b2))).astype(np.float64)
        want = -float(f(HP["lr"])) / (1 - float(b1) ** step) * m.astype(np.float64) / (r / np.sqrt(1 - float(b2) ** step) + float(f(hp["eps"])))
        want = want.reshape(-1)[:n]
        err = np.abs(p.double().cpu().numpy() - want)
        assert np.all(err <= 2e-6 * np.abs(want) + 2.0 ** -149), float((err / np.abs(want).clip(2.0 ** -149)).max())


@pytest.mark.parametrize("pt,gt,eps", [(F32, F32, 1e-8), (F32, BF16, 1e-8), (BF16, F32, 1e-8), (BF16, BF16, 1e-8), (F32, F32, 1e-15), (BF16, BF16, 1e-15)])
@pytest.mark.parametrize("packed", [False, True])
def test_adamw_tensors_8_bits_of_a_large_model(b, pt, gt, eps, packed):
    """Enough elements that warps take four units at a time, and the rest of each tensor one at a time: codes and scales of two
    steps are the plain fp32 sequence's bit for bit, the parameters those of the formula in 64 bits; what lies between the
    tensors stays as it is.  Among them small tensors, one whose codes are not 8-byte aligned, one of tiny gradients."""
    hp = dict(HP, eps=eps)
    sizes = [1_300_007, 5, 900_001, 1023, 1024, 256, 70_001, 700_000, 1, 307_200, 4096 + 255]
    odd, tiny = 6, 9
    assert sum(n // 1024 for k, n in enumerate(sizes) if k != odd) >= 16 * torch.cuda.get_device_properties(0).multi_processor_count
    g = gen(61)

    def row_of(dtype, std, fill):
        """Views at odd places of one row with a guard between them, or each on a boundary of 256; the row."""
        starts, at = [], 1 if packed else 0
        for n in sizes:
            starts.append(at)
            at += n + 1 if packed else -(-(n + 1) // 256) * 256
        row = torch.full((at,), fill, dtype=dtype, device="cuda")
        for a, n in zip(starts, sizes):
            row[a:a + n] = (torch.randn(n, generator=g, device="cuda") * std).to(dtype)
        inside = torch.zeros(at, dtype=torch.bool, device="cuda")
        for a, n in zip(starts, sizes):
            inside[a:a + n] = True
        return row, [row[a:a + n] for a, n in zip(starts, sizes)], ~inside

    prow, p, outside = row_of(pt, 0.02, 7.0)
    grow, gr, _ = row_of(gt, 1e-2, float("nan"))
    gr[tiny].copy_((gr[tiny].float() * 1e-17).to(gt))
    code = lambda n, lead: torch.zeros(n + 8, dtype=torch.uint8, device="cuda")[lead:lead + n].view(torch.float8_e4m3fn)  # noqa: E731
    states = [[code(n, 3 if k == odd else 0) for k, n in enumerate(sizes)] for _ in range(2)]
    t = b.AdamWTensors(p, gr, state_bits=8, exp_avgs=states[0], exp_avg_sqs=states[1])
    codes = lambda x: x.view(torch.uint8).cpu().numpy()  # noqa: E731
    clip = torch.tensor([0.5], device="cuda")
    for step in (1, 2):
        old, st = [x.double().cpu().numpy() for x in p], [[codes(t.exp_avgs[k]), codes(t.exp_avg_sqs[k]), t.exp_avg_scales[k].cpu().numpy(), t.exp_avg_sq_scales[k].cpu().numpy()]
                                                          for k in range(len(sizes))]
        b.dppf_adamw_tensors(t, step=step, seed=step + 9, grad_scale=clip, **hp)
        for k, n in enumerate(sizes):
            gk = gr[k].float().cpu().numpy() * np.float32(0.5)
            want = ref.adamw8_states(gk, *st[k], HP["beta1"], HP["beta2"], step + 9)
            for got, w in zip((codes(t.exp_avgs[k]), t.exp_avg_scales[k].cpu().numpy(), codes(t.exp_avg_sqs[k]), t.exp_avg_sq_scales[k].cpu().numpy()), want):
                assert np.array_equal(got, w), (k, n)
            wp, _, _ = ref.adamw(old[k], gk.astype(np.float64), ref.decode(st[k][0], st[k][2], n), ref.decode(st[k][1], st[k][3], n) ** 2, step=step, **hp)
            got = p[k].double().cpu().numpy()
            assert np.all(np.abs(got - wp) <= HALF[pt] * np.abs(wp) + 2e-6 * (np.abs(wp) + np.abs(wp - old[k])) + 1e-9), (k, n)
    assert bool((prow[outside] == 7).all()) and bool(torch.isnan(grow[outside]).all())
    for ts in states:
        for k, x in enumerate(ts):
            whole = torch.empty(0, dtype=torch.uint8, device="cuda").set_(x.untyped_storage())
            lead = 3 if k == odd else 0
            assert not whole[:lead].any() and not whole[lead + sizes[k]:].any()


# ---------------------------------------------------------------- refusals

def test_workspaces_have_to_be_memory_of_the_device(b):
    i = policy_inputs(6, 64, BF16, 12)
    args = (i["logits"], i["targets"], i["old"], i["adv"], i["weight"])
    ids, go, t = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.ones(4, 8, device="cuda"), torch.zeros(3, 8, device="cuda")
    for alloc, call in ((lambda: b.alloc_policy_workspace(6), lambda ws: b.dppf_policy_loss(*args, ws=ws)),
                        (lambda: b.alloc_embedding_workspace(4, 8), lambda ws: b.dppf_embedding_grad(go, ids, t, ws=ws))):
        ws = alloc()
        for bad in (ws.cpu(), ws[:1].expand(ws.numel()), ws.repeat(2)[::2]):      # host memory; one byte said to be many; bytes with gaps
            with pytest.raises(ValueError):
                call(bad)
        call(ws)
    assert bool((t[0] == 4).all())


def test_adamw_tensors_refuse_shared_memory(b):
    row, states = torch.zeros(100, device="cuda"), [torch.zeros(40, device="cuda") for _ in range(4)]
    a, c = row[:40], row[60:]
    g = [torch.zeros(40, device="cuda")] * 2                   # gradients are read only: they may be one
    b.AdamWTensors([a, row[:0], c], [g[0], row[:0], g[1]])
    b.AdamWTensors([a, row[40:80]], g, exp_avgs=states[:2], exp_avg_sqs=states[2:])
    for params, more in (([a, a], {}), ([a, row[39:79]], {}), ([a, c], dict(exp_avgs=[states[0], states[0]])), ([a, c], dict(exp_avgs=states[:2], exp_avg_sqs=[states[2], states[1]])),
                         ([a, c], dict(exp_avgs=[states[0], a]))):
        with pytest.raises(ValueError):
            b.AdamWTensors(params, g, **more)
