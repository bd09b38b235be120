"""atf_qk_norm_rope at the ends of its ranges, against the definition in more than 64 bits.  Tolerance of the norm: that of
test_gpu_norm_rope.py, 96 x 2^-24 (|p| + |q|) and half a step of the output's type."""
import numpy as np
import pytest
import torch

import paper_2608_02947_b200 as atf

pytestmark = pytest.mark.gpu


def _reference(x, w, eps, turns):
    """x [N, H, d] and the angles as exact fractions of a turn [N, d/2]: rows [H, N, d] and the size of what an element is the sum of."""
    h = x.shape[-1] // 2
    x = x.astype(np.longdouble)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + np.longdouble(eps)) * w
    a = (turns.astype(np.longdouble) * (2 * np.longdouble(np.pi)))[:, None]
    lo, hi = y[..., :h], y[..., h:]
    z = np.concatenate((lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)), -1)
    size = np.abs(lo) + np.abs(hi)
    return z.transpose(1, 0, 2), np.concatenate((size, size), -1).transpose(1, 0, 2)


def _check(out, ref, size, more=0.0):
    tol = (96 * 2.0 ** -24 + more) * size + torch.finfo(out.dtype).eps / 2 * np.abs(ref) * 1.001 + 1e-37
    off = np.abs(out[0].double().cpu().numpy() - ref)
    assert (off <= tol).all(), float((off / tol).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,H,d", [(8, 1, 64), (8, 7, 128), (4000, 9, 128)])
def test_rows_of_any_size(dtype, N, H, d):
    """Squares that leave the range of 32 bits, above and below: the rows come out as their definition says, whatever eps is."""
    x = torch.randn((1, N, H, d), generator=torch.Generator().manual_seed(2)).to(torch.float64)
    power = torch.tensor([0, 60, 63, 64, 100, 125, -60, -110])[torch.arange(N) % 8]
    x = (x * torch.exp2(power.double())[None, :, None, None]).clamp(-3e38, 3e38).to(dtype).cuda()
    w = (1 + 0.25 * torch.randn(d, generator=torch.Generator().manual_seed(3))).to(dtype).cuda()
    theta = np.zeros(d // 2)
    for eps in (0.0, 1e-6, 1e-40, 1e-60):
        out, _ = atf.atf_qk_norm_rope(x, None, theta, q_weight=w, eps=eps)
        rows = [i for i in range(N) if i < 16 or i % 97 == 0]
        ref, size = _reference(x[0, rows].double().cpu().numpy(), w.double().cpu().numpy(), eps, np.zeros((len(rows), d // 2)))
        _check(out[:, :, rows], ref, size)
    zero, _ = atf.atf_qk_norm_rope(torch.zeros_like(x), None, theta)
    assert not zero.any()
