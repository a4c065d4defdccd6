"""The layer norm's gradient in matrices of more than 2^31 elements, against the formulas in 64 bits (tolerances of test_gpu_block)."""
import pytest
import torch

from gpu_util import require_gpu
from test_gpu_block import BF16, F32, norm_grads, randn, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    return require_gpu()[1]


@pytest.mark.parametrize("T,H", [(70_000, 32768), (600_000, 4096), (9_000_000, 256)])      # rows walked from memory, of a block, of a part of a warp
def test_norm_grad_past_32_bits(b, T, H):
    rows = torch.tensor([0, 1, 2 ** 31 // H - 1, 2 ** 31 // H, T - 2, T - 1], device="cuda")      # the others have no gradient
    x, dy = torch.zeros(T, H, dtype=BF16, device="cuda"), torch.zeros(T, H, dtype=BF16, device="cuda")
    x[rows], dy[rows] = randn((len(rows), H), 1, BF16), randn((len(rows), H), 2, BF16)
    w = randn(H, 3, F32, 0.2, 1.0)
    fwd = b.dppf_layer_norm(x, w)
    few = b.dppf_layer_norm(x[rows], w)
    assert torch.equal(fwd.out[rows], few.out) and torch.equal(fwd.mean[rows], few.mean) and torch.equal(fwd.rstd[rows], few.rstd)
    dw, db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    dx = b.dppf_layer_norm_grad(dy, x, fwd.mean, fwd.rstd, w, dw, db, grad_x=fwd.out if H == 256 else None)
    want, tol, want_w, tol_w, want_b, tol_b = norm_grads(dy[rows], x[rows], few.mean, few.rstd, w, None)
    within(dx[rows], want, tol)
    within(dw, want_w, tol_w)
    within(db, want_b, tol_b)
    dx[rows] = 0
    assert not dx.any()
