"""Host-side checks of the operators of a transformer block: refusals before any CUDA call (fake but well-formed pointers) and of
the binding, and the rotary frequencies against their formulas."""
import ctypes
import math

import pytest
import torch

P = [0x10000000 * k for k in range(1, 20)]     # far apart
BIG = 1 << 27
NAN = float("nan")


@pytest.fixture(scope="module")
def b():
    from paper_2507_20424_b200 import binding, build
    build.build()
    binding.load()
    return binding


def caller(f, ok, order):
    return lambda **kw: f(*[{**ok, **kw}[k] for k in order], None)


def test_layer_norm_refusals(b):
    ok = dict(x=P[0], xt=0, ldx=64, br=P[1], bt=1, ldb=64, w=P[2], bias=P[3], wt=0, T=10, H=64, eps=1e-5, s=P[4], lds=64, o=P[5], ot=1, ldo=64, m=P[6], r=P[7])
    call = caller(b.load().dppf_layer_norm, ok, list(ok))
    for bad in (dict(x=None), dict(w=None), dict(o=None), dict(m=None), dict(r=None), dict(s=None), dict(br=None), dict(xt=2), dict(bt=2), dict(wt=-1), dict(ot=7), dict(T=-1),
                dict(T=2**31), dict(H=0), dict(H=65537), dict(eps=-1e-5), dict(eps=NAN), dict(ldx=63), dict(ldb=63), dict(lds=63), dict(ldo=63), dict(o=P[0]), dict(o=P[4] + 4), dict(s=P[1]),
                dict(s=P[0] + 256), dict(s=P[0], lds=80), dict(m=P[7] + 4), dict(r=P[0]), dict(m=P[2] + 8), dict(o=P[3])):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for bad in (dict(x=P[0] + 2), dict(br=P[1] + 1), dict(w=P[2] + 2), dict(bias=P[3] + 1), dict(s=P[4] + 2), dict(o=P[5] + 1), dict(m=P[6] + 2), dict(r=P[7] + 1)):
        assert call(**bad) == b.ERR_ALIGNMENT, bad
    assert call(T=0, x=None, o=None) == b.OK


def test_layer_norm_grad_refusals(b):
    ok = dict(go=P[0], ot=1, ldo=64, x=P[1], xt=0, ldx=64, m=P[2], r=P[3], w=P[4], wt=0, T=10, H=64, gs=P[5], ldg=64, gx=P[6], ldgx=64, gw=P[7], gb=P[8], gt=0, acc=0, ws=P[9], n=BIG)
    call = caller(b.load().dppf_layer_norm_grad, ok, list(ok))
    for bad in (dict(go=None), dict(x=None), dict(m=None), dict(r=None), dict(w=None), dict(gx=None), dict(gw=None), dict(ws=None), dict(ot=2), dict(xt=2), dict(wt=2), dict(gt=2), dict(T=-1), dict(H=0),
                dict(ldo=63), dict(ldx=63), dict(ldg=63), dict(ldgx=63), dict(gx=P[1]), dict(gx=P[0]), dict(gx=P[5] + 256), dict(gx=P[5], ldgx=80), dict(gw=P[8]), dict(gw=P[9]), dict(gb=P[4]),
                dict(ws=P[0]), dict(ws=P[6] + 128), dict(gw=P[1])):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for bad in (dict(go=P[0] + 1), dict(x=P[1] + 2), dict(m=P[2] + 2), dict(w=P[4] + 2), dict(gs=P[5] + 2), dict(gx=P[6] + 2), dict(gw=P[7] + 2), dict(gb=P[8] + 1), dict(ws=P[9] + 64)):
        assert call(**bad) == b.ERR_ALIGNMENT, bad
    assert call(n=64) == b.ERR_WORKSPACE
    assert call(T=0, go=None, x=None, ws=None, n=0, acc=1) == b.OK
    size = b.load().dppf_layer_norm_workspace_bytes
    assert size(0, 8) == 0 and size(8, 0) == 0 and size(8, 65537) == 0
    assert 0 < size(1, 1) <= size(100, 4096) <= size(10**6, 4096) < 1 << 26
    with pytest.raises(ValueError):
        b.alloc_layer_norm_workspace(0, 8, device="cpu")


def test_rotary_refusals(b):
    ok = dict(x=P[0], t=1, ld=512, hd=64, T=10, h=8, D=64, n=64, il=0, pos=P[1], pb=64, f=P[2], s=1.0, inv=0, o=P[3], ldo=512, hdo=64)
    call = caller(b.load().dppf_rotary, ok, list(ok))
    for bad in (dict(x=None), dict(pos=None), dict(f=None), dict(o=None), dict(t=2), dict(pb=16), dict(T=-1), dict(h=0), dict(h=1025), dict(D=0), dict(D=1025, ld=9000, hd=1025, ldo=9000, hdo=1025),
                dict(n=0), dict(n=63), dict(n=66), dict(s=NAN), dict(ld=511), dict(hd=63), dict(ld=0), dict(o=P[0], ldo=520), dict(o=P[0] + 128), dict(o=P[1]), dict(o=P[2]), dict(ld=-512)):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for bad in (dict(x=P[0] + 1), dict(o=P[3] + 1), dict(pos=P[1] + 4), dict(f=P[2] + 4)):
        assert call(**bad) == b.ERR_ALIGNMENT, bad
    assert call(T=0, x=None, o=None) == b.OK


def test_rotary_frequencies(b):
    def values(n, **kw):
        f, s = b.rotary_frequencies(n, device="cpu", **kw)
        assert f.dtype == torch.float64 and len(f) == n // 2
        return f.tolist(), s

    plain = [10000.0 ** (-2 * i / 64) for i in range(32)]
    assert values(64) == (pytest.approx(plain, rel=1e-14), 1.0)
    assert values(64, scaling="interpolated", factor=4.0) == (pytest.approx([v / 4 for v in plain], rel=1e-14), 1.0)
    got, _ = values(64, scaling="stretched", factor=8.0)
    assert got[0] == 1.0 and got[-1] == pytest.approx(plain[-1] / 8, rel=1e-12)
    assert values(2, scaling="stretched", factor=8.0)[0] == [1.0]
    got, scale = values(64, scaling="by parts", factor=16.0, original_length=4096)
    assert scale == pytest.approx(0.1 * math.log(16.0) + 1, rel=1e-6)
    for f, p in zip(got, plain):
        turns = 4096 * p / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1) / 31))
        assert f == pytest.approx(p / 16 * (1 - keep) + p * keep, rel=1e-12)
    assert got[0] == 1.0 and got[-1] == pytest.approx(plain[-1] / 16)
    for bad in (dict(turned=0), dict(turned=7), dict(turned=2000), dict(base=1.0), dict(base=NAN), dict(factor=0.5, scaling="interpolated"), dict(scaling="by parts", factor=2.0)):
        with pytest.raises(b.DppfError):
            b.rotary_frequencies(**{"turned": 64, "device": "cpu", **bad})
    with pytest.raises(ValueError):
        b.rotary_frequencies(64, scaling="none", device="cpu")
    f = b.load().dppf_rotary_frequencies
    out, scale = (ctypes.c_double * 4)(), ctypes.c_float()
    assert f(8, 10000.0, 4, 1.0, 0, out, ctypes.byref(scale)) == b.ERR_INVALID_ARG and f(8, 10000.0, 0, 1.0, 0, None, ctypes.byref(scale)) == b.ERR_INVALID_ARG


def test_binding_refuses_what_it_cannot_pass_on(b):
    cpu, w = torch.zeros(4, 8), torch.ones(8)
    with pytest.raises(ValueError):
        b.dppf_layer_norm(cpu, w)
    with pytest.raises(ValueError):
        b.dppf_layer_norm_grad(cpu, cpu, torch.zeros(4), torch.zeros(4), w, w)
    with pytest.raises(ValueError):
        b.dppf_rotary(torch.zeros(4, 2, 8), torch.arange(4), torch.ones(4, dtype=torch.float64))


def test_attention_plan_refusals(b):
    size, f = b.load().dppf_attention_plan_bytes, b.load().dppf_attention_plan
    assert size(-1, 1) == 0 and size(5, 0) == 0 and size(2**24 + 1, 1) == 0 and size(5, 2**20 + 1) == 0
    assert 0 < size(0, 1) <= size(1000, 4) <= size(10**6, 4) <= size(10**6, 10**5) < 1 << 24
    ok = dict(s=P[0], sb=32, T=1000, B=4, plan=P[1], n=BIG)
    call = caller(f, ok, list(ok))
    for bad in (dict(s=None), dict(plan=None), dict(sb=16), dict(T=-1), dict(B=0), dict(s=P[1] + 256)):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for bad in (dict(s=P[0] + 2), dict(sb=64, s=P[0] + 4), dict(plan=P[1] + 64)):
        assert call(**bad) == b.ERR_ALIGNMENT, bad
    assert call(n=256) == b.ERR_WORKSPACE


def test_attention_refusals(b):
    ok = dict(q=P[0], ldq=512, hq=64, k=P[1], ldk=128, hk=64, v=P[2], ldv=128, hv=64, T=100, B=3, h=8, kv=2, D=64, c=1, w=0, s=0.1, o=P[3], ldo=512, ho=64, lse=P[4], plan=P[5], n=BIG)
    call = caller(b.load().dppf_attention, ok, list(ok))
    for bad in ([{k: None} for k in ("q", "k", "v", "o", "lse", "plan")] +
                [dict(T=-1), dict(T=2**25), dict(B=0), dict(h=0), dict(h=1025, kv=1), dict(kv=0), dict(kv=3), dict(D=0), dict(D=60), dict(D=136, ldq=2000, hq=136), dict(c=2), dict(w=-1), dict(w=5, c=0),
                 dict(s=0.0), dict(s=-1.0), dict(s=NAN), dict(s=3e38), dict(ldq=504), dict(hq=56), dict(ldk=0), dict(ldo=-8), dict(o=P[0]), dict(o=P[1]), dict(lse=P[3]), dict(lse=P[0]), dict(lse=P[5]), dict(o=P[5]),
                 dict(ldq=2**39)]):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for bad in (dict(q=P[0] + 8), dict(k=P[1] + 2), dict(v=P[2] + 8), dict(o=P[3] + 8), dict(ldq=516), dict(hk=68, ldk=200), dict(lse=P[4] + 2), dict(plan=P[5] + 64)):
        assert call(**bad) == b.ERR_ALIGNMENT, bad
    assert call(n=512) == b.ERR_WORKSPACE
    assert call(T=0, q=None, plan=None) == b.OK


def test_attention_grad_refusals(b):
    ok = dict(go=P[0], ldgo=512, hgo=64, q=P[1], ldq=512, hq=64, k=P[2], ldk=128, hk=64, v=P[3], ldv=128, hv=64, o=P[4], ldo=512, ho=64, lse=P[5], T=100, B=3, h=8, kv=2, D=64, c=1, w=0, s=0.1,
              dq=P[6], lddq=512, hdq=64, dk=P[7], lddk=128, hdk=64, dv=P[8], lddv=128, hdv=64, plan=P[9], n=BIG, ws=P[10], m=BIG)
    call = caller(b.load().dppf_attention_grad, ok, list(ok))
    for bad in ([{k: None} for k in ("go", "q", "k", "v", "o", "lse", "dq", "dk", "dv", "plan", "ws")] +
                [dict(h=7), dict(D=68), dict(s=0.0), dict(w=3, c=0), dict(ldgo=100), dict(lddq=100), dict(dq=P[0]), dict(dq=P[1]), dict(dk=P[2]), dict(dk=P[7] + 128, dv=P[7]), dict(dq=P[5]), dict(dv=P[9]),
                 dict(dv=P[10]), dict(ws=P[0]), dict(ws=P[5]), dict(ws=P[9]), dict(dk=P[4])]):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for bad in (dict(go=P[0] + 8), dict(o=P[4] + 2), dict(dq=P[6] + 8), dict(lddk=132), dict(lse=P[5] + 1), dict(ws=P[10] + 64)):
        assert call(**bad) == b.ERR_ALIGNMENT, bad
    assert call(n=512) == b.ERR_WORKSPACE and call(m=512) == b.ERR_WORKSPACE
    assert call(T=0, q=None, plan=None, ws=None) == b.OK
    assert b.load().dppf_attention_workspace_bytes(0, 4) == 0 and b.load().dppf_attention_workspace_bytes(100, 0) == 0
    # gradients beside one another in rows of one product do not overlap; shifted by one head they do
    row = dict(dq=P[6], lddq=768, dk=P[6] + 2 * 512, lddk=768, dv=P[6] + 2 * 640, lddv=768)
    assert call(**{**row, "m": 512}) == b.ERR_WORKSPACE
    assert call(**{**row, "dv": P[6] + 2 * 576, "m": 512}) == b.ERR_WORKSPACE and call(**{**row, "dv": P[6] + 2 * 576}) == b.ERR_INVALID_ARG


def test_binding_refuses_attention_on_the_host(b):
    with pytest.raises(ValueError):
        b.AttentionPlan(torch.zeros(2, dtype=torch.int32), 5)
    with pytest.raises(ValueError):
        b.alloc_attention_workspace(0, 4, device="cpu")
