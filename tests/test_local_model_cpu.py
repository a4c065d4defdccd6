"""Host-side checks of the operators of a language-model worker's local step: refusals before any CUDA
call (fake but well-formed pointers) and of the binding, and the reference's own e4m3 table and hash."""
import ctypes

import numpy as np
import pytest
import torch

import local_model_ref as ref

P = [0x10000000 * k for k in range(1, 15)]     # far apart
BIG = 1 << 27


@pytest.fixture(scope="module")
def b():
    from paper_2507_20424_b200 import binding, build
    build.build()
    binding.load()
    return binding


def test_embedding_refusals(b):
    f = b.load().dppf_embedding
    ok = dict(table=P[0], tt=0, V=100, H=64, ld=64, ids=P[1], ib=64, T=10, scale=1.0, out=P[2], ot=0, ldo=64)

    def call(**kw):
        a = {**ok, **kw}
        return f(a["table"], a["tt"], a["V"], a["H"], a["ld"], a["ids"], a["ib"], a["T"], a["scale"], a["out"], a["ot"], a["ldo"], None)

    for bad in (dict(table=None), dict(ids=None), dict(out=None), dict(tt=2), dict(ot=-1), dict(ib=16), dict(V=0), dict(V=2**31), dict(H=0), dict(H=65537),
                dict(ld=63), dict(ldo=63), dict(T=-1), dict(scale=float("nan")), dict(out=P[0] + 64), dict(out=P[1]), dict(T=2**31)):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for bad in (dict(table=P[0] + 2), dict(out=P[2] + 1), dict(ids=P[1] + 4), dict(ot=1, out=P[2] + 1)):
        assert call(**bad) == b.ERR_ALIGNMENT, bad
    assert call(T=0, ids=None, out=None) == b.OK


def test_embedding_grad_refusals(b):
    f = b.load().dppf_embedding_grad
    ok = dict(go=P[0], ot=0, ldo=64, ids=P[1], ib=32, T=10, scale=1.0, gt=P[2], tt=0, V=100, H=64, ld=64, acc=0, ws=P[3], n=BIG)

    def call(**kw):
        a = {**ok, **kw}
        return f(a["go"], a["ot"], a["ldo"], a["ids"], a["ib"], a["T"], a["scale"], a["gt"], a["tt"], a["V"], a["H"], a["ld"], a["acc"], a["ws"], a["n"], None)

    for bad in (dict(go=None), dict(ids=None), dict(gt=None), dict(ws=None), dict(ot=3), dict(tt=3), dict(ib=8), dict(V=0), dict(H=0), dict(ld=1), dict(ldo=1),
                dict(scale=float("inf")), dict(gt=P[0]), dict(gt=P[3] + 128), dict(ws=P[0] + 128), dict(ws=P[1])):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for bad in (dict(gt=P[2] + 2), dict(go=P[0] + 1), dict(ids=P[1] + 2), dict(ws=P[3] + 64)):
        assert call(**bad) == b.ERR_ALIGNMENT, bad
    assert call(n=64) == b.ERR_WORKSPACE
    assert call(T=0, go=None, ids=None, ws=None, n=0, acc=1) == b.OK


def test_embedding_workspace(b):
    assert b.embedding_workspace_bytes(0, 64) == 0 and b.embedding_workspace_bytes(5, 0) == 0
    assert b.embedding_workspace_bytes(5, 65537) == 0
    small, large = b.embedding_workspace_bytes(1, 1), b.embedding_workspace_bytes(100_000, 2048)
    assert 0 < small < large < 100_000 * 2048 * 4 and small % 256 == 0 and large % 256 == 0
    with pytest.raises(ValueError):
        b.alloc_embedding_workspace(0, 8, device="cpu")


def test_policy_refusals(b):
    f = b.load().dppf_policy_loss
    ok = dict(x=P[0], ty=1, T=8, V=100, ld=104, y=P[1], tb=64, old=P[2], ref=P[3], adv=P[4], w=P[5], lo=0.2, hi=0.2, kl=0.1, temp=1.0, sums=P[6], lp=P[7],
              g=P[8], ldg=104, ws=P[9], n=BIG)

    def call(**kw):
        a = {**ok, **kw}
        return f(*[a[k] for k in ("x", "ty", "T", "V", "ld", "y", "tb", "old", "ref", "adv", "w", "lo", "hi", "kl", "temp", "sums", "lp", "g", "ldg", "ws", "n")], None)

    for bad in ([{k: None} for k in ("x", "y", "old", "adv", "w", "sums", "lp", "ws", "ref")] +
                [dict(ty=2), dict(tb=8), dict(T=0), dict(T=2**25), dict(V=0), dict(V=262145, ld=262145), dict(ld=99), dict(ldg=99), dict(lo=-0.1), dict(lo=1.5),
                 dict(hi=-0.1), dict(kl=float("nan")), dict(temp=0.0), dict(temp=-1.0), dict(temp=float("inf")), dict(g=P[0] + 208), dict(g=P[0], ldg=112),
                 dict(lp=P[0]), dict(sums=P[7] + 4), dict(ws=P[0]), dict(lp=P[2]), dict(g=P[5])]):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for bad in (dict(x=P[0] + 1), dict(g=P[8] + 1), dict(y=P[1] + 4), dict(ws=P[9] + 8), dict(old=P[2] + 2), dict(lp=P[7] + 1)):
        assert call(**bad) == b.ERR_ALIGNMENT, bad
    assert call(n=256) == b.ERR_WORKSPACE
    assert b.load().dppf_policy_workspace_bytes(0) == 0 and b.load().dppf_policy_workspace_bytes(2**25) == 0


def test_adamw_tensors_refusals(b):
    f = b.load().dppf_adamw_tensors

    def call(n=1, tp=0, tg=0, bits=32, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.1, step=1, gs=None, null=False, **kw):
        t = (b._Tensor * 1)()
        fields = dict(param=P[0], grad=P[1], exp_avg=P[2], exp_avg_sq=P[3], exp_avg_scale=P[4], exp_avg_sq_scale=P[5], numel=1000, decay=1.0)
        for k, v in {**fields, **kw}.items():
            setattr(t[0], k, v)
        return f(None if null else t, n, tp, tg, bits, lr, b1, b2, eps, wd, step, gs, 0, None)

    nan = float("nan")
    for bad in (dict(null=True), dict(n=-1), dict(tp=2), dict(tg=5), dict(bits=16), dict(lr=nan), dict(b1=1.0), dict(b2=-0.1), dict(eps=nan), dict(wd=nan), dict(step=0),
                dict(param=None), dict(grad=None), dict(exp_avg=None), dict(exp_avg_sq=None), dict(bits=8, exp_avg_scale=None), dict(bits=8, exp_avg_sq_scale=None),
                dict(numel=-1), dict(numel=2**38), dict(decay=nan), dict(grad=P[0] + 4), dict(exp_avg=P[3] + 400), dict(bits=8, exp_avg_scale=P[5]), dict(bits=8, exp_avg_scale=P[2] + 4)):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for bad in (dict(param=P[0] + 2), dict(tg=1, grad=P[1] + 1), dict(exp_avg=P[2] + 1), dict(bits=8, exp_avg_scale=P[4] + 2), dict(gs=P[6] + 2)):
        assert call(**bad) == b.ERR_ALIGNMENT, bad
    assert call(numel=0, param=None) == b.OK and call(n=0, null=True) == b.OK
    assert ctypes.sizeof(b._Tensor) == 64


def test_binding_refuses_what_it_cannot_pass_on(b):
    cpu = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        b.dppf_embedding(cpu, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        b.dppf_embedding_grad(torch.zeros(3, 8), torch.zeros(3, dtype=torch.int64), cpu)
    with pytest.raises(ValueError):
        b.dppf_policy_loss(cpu, torch.zeros(4, dtype=torch.int64), *[torch.zeros(4)] * 3)
    with pytest.raises(ValueError):
        b.AdamWTensors([torch.zeros(4)], [torch.zeros(4)])
    with pytest.raises(ValueError):
        b.AdamWTensors([], [])
    with pytest.raises(ValueError):
        b.AdamWTensors([torch.zeros(4)], [torch.zeros(4)], state_bits=16)


def test_reference_e4m3_table_is_torchs():
    codes = torch.arange(256).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    fine = ~np.isnan(want)
    assert fine.sum() == 254 and np.array_equal(ref.E4M3[fine], want[fine])


def test_reference_hash_is_the_published_finalizer():
    # fmix32 of MurmurHash3: known values
    def fmix(h):
        h ^= h >> 16
        h = h * 0x85EBCA6B & 0xFFFFFFFF
        h ^= h >> 13
        h = h * 0xC2B2AE35 & 0xFFFFFFFF
        return h ^ h >> 16
    assert fmix(0) == 0 and fmix(1) == 0x514E28B7
    bits = ref.random_bits(6, 7)
    for i in range(6):
        h = fmix((i // 2 + 7 * 0x9E3779B9) & 0xFFFFFFFF)
        assert bits[i] == ((h >> 16) if i % 2 else (h & 0xFFFF)) << 4
