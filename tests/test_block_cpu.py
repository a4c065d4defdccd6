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
