"""A cache object stands for the tensors that it was made with."""
import pytest
import torch

import paper_2608_02947_b200 as atf

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_tensors_of_a_cache_are_not_replaced(fmt):
    """The calls work on the tensors that were checked when the object was made."""
    c = atf.new_kvcache(1, 2, 100, 64, fmt)
    for name in ("k", "v", "scales", "capacity", "format", "B", "Hkv", "d", "index"):
        kept = getattr(c, name)
        with pytest.raises(AttributeError):
            setattr(c, name, kept)
        assert getattr(c, name) is kept
    K = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16, device="cuda")
    Q = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16, device="cuda")
    for name in ("k", "v") + (() if c.scales is None else ("scales",)):
        t = getattr(c, name)
        kept, other = t.data, torch.zeros_like(t)
        t.data = other
        for call in (lambda: atf.atf_kvcache_write(c, K, K), lambda: atf.atf_kvcache_read(c, 3), lambda: atf.atf_decode_tree(Q, c, 5)):
            with pytest.raises(atf.AtfError):
                call()
        t.data = kept
        assert not other.any()
    atf.atf_kvcache_write(c, K, K)
