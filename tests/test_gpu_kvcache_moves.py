"""Rows of the cache that are read at one slot and written at another."""
import pytest
import torch

import paper_2608_02947_b200 as atf

pytestmark = pytest.mark.gpu


def _rows(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * torch.exp(torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))).to(torch.bfloat16)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_move_keeps(fmt, d):
    """bf16 and e4m3: a code times a power of two is a bf16 number, and every value is held again as it was.  int8: the value read is the
    held one rounded to bf16 (2^-9 of itself); held again, it is off by half a code of its new scale, and that scale is at most
    (1 + 2^-7) / 127 of the largest value read, which is at most (1 + 2^-9) of the largest held."""
    n = 500
    K, V = _rows((2, 3, n, d), 1), _rows((2, 3, n, d), 2)
    c = atf.new_kvcache(2, 3, 2 * n, d, fmt)
    atf.atf_kvcache_write(c, K, V)
    old = atf.atf_kvcache_read(c, n)
    at = torch.arange(2 * n - 1, n - 1, -1, device="cuda")[None].repeat(2, 1)
    atf.atf_kvcache_write(c, *old, slots=at)
    new = atf.atf_kvcache_read(c, n, slots=at)
    for a, b in zip(old, new):
        if fmt != "int8":
            assert torch.equal(a, b)
            continue
        a, b = a.double(), b.double()
        # both as read, 2^-9 of themselves from what is held
        top = a.abs().amax(-1, keepdim=True) * (1 + 2.0 ** -8)
        assert ((a - b).abs() <= 2.0 ** -9 * (a.abs() + b.abs()) * 1.01 + top * (1 + 2.0 ** -8) * (1 + 2.0 ** -7) / 254).all()
    # rows written again from where they came from are the same bytes
    atf.atf_kvcache_write(c, K, V, slots=at)
    again = atf.atf_kvcache_read(c, n, slots=at)
    assert all(torch.equal(a, b) for a, b in zip(old, again))
