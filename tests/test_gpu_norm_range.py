"""atf_qk_norm_rope at the ends of its ranges, against the definition in more than 64 bits.  Tolerance of the norm: that of
test_gpu_norm_rope.py, 96 x 2^-24 (|p| + |q|) and half a step of the output's type."""
import numpy as np
import pytest
import torch

import paper_2608_02947_b200 as atf

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


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
def test_far_positions(dtype):
    """Angles that are exact in 64 bits (theta = 2 pi / 2^k up to its own rounding): position / 2^k is a fraction of a turn that is
    known exactly.  The product position x theta / 2 pi, theta rounded to 64 bits and its quotient by 2 pi rounded again, is off by
    at most 3 x 2^-53 of itself, 2 pi times that as an angle."""
    d, H = 128, 3
    k = 6 + np.arange(d // 2) % 30
    theta = 2 * np.pi / np.exp2(k)
    pos = [0, 1, -1, 131071, (1 << 31) + 5, -(1 << 33) - 7, (1 << 40) + 1, (1 << 40) - 12345, -(1 << 40) + 3]
    x = torch.randn((1, len(pos), H, d), generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    out, _ = atf.atf_qk_norm_rope(x, None, theta, positions=torch.tensor([pos], device="cuda"))
    turns = np.array([[(p % (1 << int(kk))) / 2.0 ** int(kk) for kk in k] for p in pos])
    off = 3 * 2.0 ** -53 * 2 * np.pi * np.abs(np.array(pos, dtype=np.float64))[:, None] / np.exp2(k)[None]
    more = np.concatenate((off, off), -1)[None]
    ref, size = _reference(x[0].double().cpu().numpy(), 1.0, 1e-6, turns)
    _check(out, ref, size, more)
    one, _ = atf.atf_qk_norm_rope(x[:, 6:7].contiguous(), None, theta, pos0=(1 << 40) + 1)
    assert torch.equal(one[:, :, 0], out[:, :, 6])


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


def _rows(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,N,H,d", [(1, 3, 2, 64), (2, 40, 5, 128), (1, 9000, 9, 128)])
def test_norm_rows(dtype, B, N, H, d):
    """A NaN makes NaN of its row; an infinity zeros of all but its own pair, which is NaN; other rows are not touched."""
    x = _rows((B, N, H, d), 4).to(dtype)
    theta = 1e4 ** (-2.0 * np.arange(d // 2) / d)
    want = atf.atf_qk_norm_rope(x, None, theta)[0]
    y = x.clone()
    y[0, 1, 0, 7], y[0, 2, H - 1, 7], y[B - 1, N - 1, 1, d // 2 + 9] = NAN, INF, -INF
    got = atf.atf_qk_norm_rope(y, None, theta)[0]
    assert torch.isnan(got[0, 0, 1]).all()
    touched = torch.zeros(B, H, N, dtype=torch.bool, device="cuda")
    touched[0, 0, 1] = True
    pairs = {}
    for row, r in (((0, H - 1, 2), 7), ((B - 1, 1, N - 1), 9)):
        pairs.setdefault(row, []).extend((r, r + d // 2))
    for (b, h, n), at in pairs.items():
        row = got[b, h, n].float().clone()
        assert torch.isnan(row[at]).all()
        row[at] = 0
        assert (row == 0).all()
        touched[b, h, n] = True
    assert torch.equal(got[~touched], want[~touched])
