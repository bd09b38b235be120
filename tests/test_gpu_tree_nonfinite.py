"""Infinities and NaN that a row of the tree attention does meet: what include/atflash.h says comes out, wherever the key stands and whichever
kernel runs."""
import pytest
import torch

import paper_2608_02947_b200 as atf

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
HKV, L, CAP = 2, 700, 800
# keys that every row sees: among others like them, at the far edge of the window, in front of the nodes; and a node
PLACES = {"middle": 520, "edge": L - 300, "last": L - 1, "node": L}


def _rows(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _case(fmt, G, T, d, change):
    K, V, Q = _rows((1, HKV, CAP, d), 1), _rows((1, HKV, CAP, d), 2), _rows((1, HKV * G, T, d), 3)
    change(K, V)
    c = atf.new_kvcache(1, HKV, CAP, d, fmt)
    atf.atf_kvcache_write(c, K, V)
    W = torch.tensor([300] * (d // 2))
    par = torch.tensor([-1] * T, dtype=torch.int32, device="cuda")  # at one position: each sees all committed keys within 300 and itself
    lens = torch.tensor([L], dtype=torch.int32, device="cuda")
    out = [atf.atf_decode_tree(Q, c, lens, par, table=W, max_len=most, return_lse=True) for most in (L, CAP - T)]
    atf.binding.check_status()
    return Q, K, V, out


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d,G,T", [(128, 1, 1), (64, 1, 3), (128, 2, 5), (64, 4, 3), (128, 3, 9), (64, 2, 70)])
@pytest.mark.parametrize("place", sorted(PLACES))
@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_values(fmt, d, G, T, place, value):
    """One element of one value: the rows that see it are NaN in O and in LSE, the others finite; the other KV head is not touched."""
    def change(K, V):
        V[0, 1, PLACES[place], 5] = value

    for O, LSE in _case(fmt, G, T, d, change)[3]:
        meets = torch.zeros(HKV * G, T, dtype=torch.bool, device="cuda")
        meets[G:, :1 if place == "node" else T] = True
        assert torch.isnan(O[0].float())[meets].all() and torch.isnan(LSE[0])[meets].all()
        assert torch.isfinite(O[0].float())[~meets].all() and torch.isfinite(LSE[0])[~meets].all()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d,G,T", [(128, 1, 1), (64, 1, 3), (128, 2, 5), (64, 4, 3), (128, 3, 9), (64, 2, 70)])
@pytest.mark.parametrize("place", sorted(PLACES))
@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_keys(fmt, d, G, T, place, value):
    """One element of one key.  8 bits: its rows are NaN.  bf16: the score is what q k gives, a NaN or +inf makes NaN of the row, with
    -inf the key has no weight."""
    def change(K, V):
        K[0, 1, PLACES[place], 5] = value

    Q, K, V, outs = _case(fmt, G, T, d, change)
    for O, LSE in outs:
        meets = torch.zeros(HKV * G, T, dtype=torch.bool, device="cuda")
        meets[G:, :1 if place == "node" else T] = True
        if fmt == "bf16" and value == value:
            meets &= Q[0, :, :, 5].float() * value > 0
        assert torch.isnan(O[0].float())[meets].all() and torch.isnan(LSE[0])[meets].all()
        assert torch.isfinite(O[0].float())[~meets].all() and torch.isfinite(LSE[0])[~meets].all()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d,G,T", [(128, 1, 1), (64, 1, 3), (128, 2, 5), (64, 4, 3), (128, 3, 9), (64, 2, 70)])
@pytest.mark.parametrize("length,bad", [(30, 10), (30, 30), (0, 0), (500, 80)])
def test_values_in_one_split(fmt, d, G, T, length, bad):
    """The same where a block of its own finishes its rows: one tile of keys, and a batch that fills the GPU."""
    B = 1 if length < 100 else 300
    K, V, Q = _rows((B, HKV, length + T, d), 1), _rows((B, HKV, length + T, d), 2), _rows((B, HKV * G, T, d), 3)
    V[0, 1, bad, d - 1] = -INF
    c = atf.new_kvcache(B, HKV, length + T, d, fmt)
    atf.atf_kvcache_write(c, K, V)
    par = torch.tensor([-1] * T, dtype=torch.int32, device="cuda")
    O, LSE = atf.atf_decode_tree(Q, c, length, par, return_lse=True)
    atf.binding.check_status()
    meets = torch.zeros(B, HKV * G, T, dtype=torch.bool, device="cuda")
    meets[0, G:, :1 if bad >= length else T] = True
    assert torch.isnan(O.float())[meets].all() and torch.isnan(LSE)[meets].all()
    assert torch.isfinite(O.float())[~meets].all() and torch.isfinite(LSE)[~meets].all()


def test_a_key_with_no_weight():
    """What a score of -inf leaves out changes nothing else: the row is the one without the key."""
    for d, G, T in ((128, 1, 1), (64, 4, 3), (128, 3, 9)):
        def change(K, V):
            K[0, :, 400, 5] = INF

        Q, K, V, outs = _case("bf16", G, T, d, change)
        q = Q.double()
        for i in range(T):
            slots = torch.tensor([s for s in range(L - 300, L) if s != 400] + [L + i], device="cuda")
            k, v = K[0, :, slots].double().repeat_interleave(G, 0), V[0, :, slots].double().repeat_interleave(G, 0)
            s = torch.einsum("hd,hnd->hn", q[0, :, i], k) / d ** 0.5
            p = torch.softmax(s, -1)
            want, size = torch.einsum("hn,hnd->hd", p, v), torch.einsum("hn,hnd->hd", p, v.abs())
            rows = Q[0, :, i, 5].float() < 0
            for O, LSE in outs:
                # weights 2^-8 of themselves, then half a step of bf16; scores under 2^-18 sum |q k| / sqrt(d) < 2^-18 x 64
                assert ((O[0, :, i].double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.001 + (2.0 ** -8 + 2.0 ** -11) * size)[rows].all()
                assert ((LSE[0, :, i].double() - torch.logsumexp(s, -1)).abs() <= 2.0 ** -12 + 2.0 ** -11)[rows].all()
