"""atf_decode_tree: slots that a row does not see, keys that no row sees and slots that were never written do not change the row,
whatever they hold, in the kernels for up to 8, up to 16 and more rows a KV head."""
import numpy as np
import pytest
import torch

import paper_2608_02947_b200 as atf
import step_reference as ref

pytestmark = pytest.mark.gpu
FORMATS = ["bf16", "e4m3", "int8"]
ROWS = [1, 2, 3, 16]  # heads of a KV head: 8, 16, 24 and 128 rows beside the 8 nodes below
PARENTS = [-1, 0, 1, -1, -1, 4, 5, 2]
NOBODYS = 3           # a node that no other node follows
HKV, D, T, L, CAP, REACH = 2, 128, 8, 300, 400, 100


def _rows(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _inputs(G):
    return _rows((1, HKV, CAP, D), 1), _rows((1, HKV, CAP, D), 2), _rows((1, HKV * G, T, D), 3)


def _attend(c, Q, W, return_lse=True):
    out = atf.atf_decode_tree(Q, c, L, torch.tensor(PARENTS, dtype=torch.int32, device="cuda"), table=W, return_lse=return_lse)
    atf.binding.check_status()
    return out


def _check(fmt, Q, K, V, W, O, LSE, nodes, parents=PARENTS, length=L):
    """Rows of these nodes against the definition on what the cache holds of K, V.

    Tolerances as in test_gpu_tree.py, but for what f16 weights lose below 2^-14: half a step of 2^-24, in units in which the row's
    largest weight times its value's scale, so far, is at least 2 (kept at 2^7, against a reference that is at most 2^6 too high): 2^-26 of
    that largest product a key, times a code of at most 448 (or 127), where 448 times a scale is less than 2 max|v| of the row
    of values (127 times a scale: (1 + 2^-7) max|v|).  2^-25 of the largest p max|v| among the keys that the row sees, a key."""
    k, v = (ref.held(t[0, :, :length + len(parents)].double().cpu().numpy(), fmt) for t in (K, V))
    apart = np.abs(np.log2(v[1])).max()
    k, v = k[0] * k[1][..., None], v[0] * v[1][..., None]
    G, h = Q.shape[1] // HKV, D // 2
    depth, line = ref.tree(parents)
    place = np.concatenate((np.arange(length), length + depth))
    q = Q[0].double().cpu().numpy()
    o, lse = O[0].double().cpu().numpy(), LSE[0].double().cpu().numpy()
    W = np.asarray(W)
    for i in nodes:
        z = length + depth[i] - place
        seen = np.concatenate((np.ones(length, dtype=bool), line[i])) & (z <= W.max())
        ks, z = seen.nonzero()[0], z[seen]
        live = z[:, None] <= W
        live = np.concatenate((live, live), -1)
        for hq in range(HKV * G):
            kk, vv, qq = k[hq // G, ks] * live, v[hq // G, ks], q[hq, i]
            s = kk @ qq / np.sqrt(D)
            m = s.max()
            p = np.exp(s - m)
            rl = m + np.log(p.sum())
            p /= p.sum()
            A = (np.abs(kk) @ np.abs(qq)).max() / np.sqrt(D)
            w, u = 2.0 ** -18 * A + 2.0 ** -20, (len(ks) / 8 + 64) * 2.0 ** -24
            if fmt != "bf16":
                w += 2.0 ** -22 * apart
            assert abs(lse[hq, i] - rl) <= w + u + 2.0 ** -20 * abs(rl), (i, hq, lse[hq, i], rl)
            tol = (2.0 ** (-8 if fmt == "bf16" else -11) + 2 * w + 2 * u) * (p @ np.abs(vv)) + 2.0 ** -8 * np.abs(p @ vv) * 1.001
            if fmt != "bf16":
                tol = tol + len(ks) * 2.0 ** -25 * (p * np.abs(vv).max(-1)).max()
            off = np.abs(o[hq, i] - p @ vv)
            assert (off <= tol).all(), (i, hq, (off / tol).max())


def _written(fmt, K, V, fill):
    """A cache whose slots hold K and V where a row but NOBODYS sees them, and elsewhere what `fill` leaves."""
    c = atf.new_kvcache(1, HKV, CAP, D, fmt)
    fill(c)
    near = torch.arange(L - REACH, L + T, device="cuda")
    near = near[near != L + NOBODYS]
    atf.atf_kvcache_write(c, K[:, :, near].contiguous(), V[:, :, near].contiguous(), slots=near[None])
    return c


def _scales(value):
    def fill(c):
        if c.scales is not None:
            c.scales.fill_(value)
    return fill


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("G", ROWS)
@pytest.mark.parametrize("scale", [0.0, -1.0, -float("inf"), float("inf"), float("nan"), 2.0 ** 126, 2.0 ** -140])
def test_slots_that_were_never_written(fmt, G, scale):
    """A fresh cache holds zeros, scales among them; one made of other memory holds anything."""
    K, V, Q = _inputs(G)
    W = torch.tensor([REACH] * (D // 2))
    O, LSE = _attend(_written(fmt, K, V, _scales(scale)), Q, W)
    _check(fmt, Q, K, V, W.tolist(), O, LSE, [i for i in range(T) if i != NOBODYS])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("G", ROWS)
@pytest.mark.parametrize("byte", [0x7f, 0xff, 0x80, 0x55, 0x7e, 0x01])
def test_bytes_of_slots_that_were_never_written(fmt, G, byte):
    """0x7f and 0xff are the NaN of e4m3, which no row that is written gets, and of a bf16 bytewise."""
    K, V, Q = _inputs(G)
    W = torch.tensor([REACH] * (D // 2))

    def fill(c):
        for t in (c.k, c.v) + (() if c.scales is None else (c.scales,)):
            t.view(torch.uint8).fill_(byte)
        if c.scales is not None:
            c.scales[..., ::2] = 1.0

    O, LSE = _attend(_written(fmt, K, V, fill), Q, W)
    _check(fmt, Q, K, V, W.tolist(), O, LSE, [i for i in range(T) if i != NOBODYS])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("G", ROWS)
@pytest.mark.parametrize("power", [20, 40, 90, -90])
def test_finite_rows_of_other_sizes(fmt, G, power):
    """Values of 2^power and more in a node and in keys out of the window (or, the other way, only there of ordinary size): finite,
    and not seen."""
    K, V, Q = _inputs(G)
    W = torch.tensor([REACH] * (D // 2))
    far = torch.arange(CAP, device="cuda") < L - REACH
    far[L + NOBODYS] = True
    V = torch.where(far[:, None], (V.double() * 2.0 ** max(power, 0)), V.double() * 2.0 ** min(power, 0)).to(torch.bfloat16)
    c = atf.new_kvcache(1, HKV, CAP, D, fmt)
    atf.atf_kvcache_write(c, K, V)
    O, LSE = _attend(c, Q, W)
    _check(fmt, Q, K, V, W.tolist(), O, LSE, range(T))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("G", ROWS)
@pytest.mark.parametrize("first", [True, False])
def test_large_values_of_no_weight(fmt, G, first):
    """Keys that every row sees, whose values are 2^40 times as large and whose weights are e^-70 and less; where they come first the
    other keys are met after them."""
    K, V, Q = _inputs(G)
    Q = Q.abs()
    at = torch.arange(CAP, device="cuda")
    low = (at < 60) if first else (at >= 200) & (at < L) & (at % 3 == 0)
    K = torch.where(low[:, None], torch.full_like(K, -12.0), K * 0.25)
    V = torch.where(low[:, None], (V.double() * 2.0 ** 40).to(torch.bfloat16), V)
    c = atf.new_kvcache(1, HKV, CAP, D, fmt)
    atf.atf_kvcache_write(c, K, V)
    O, LSE = _attend(c, Q, None)
    _check(fmt, Q, K, V, [CAP] * (D // 2), O, LSE, range(T))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("G", ROWS)
@pytest.mark.parametrize("power", [-30, -60, -100])
@pytest.mark.parametrize("zeros", ["one", "first", "most"])
def test_rows_of_zeros_among_small_values(fmt, G, power, zeros):
    """A row of zeros has scale 1, whatever the size of its neighbours."""
    K, V, Q = _inputs(G)
    at = torch.arange(CAP, device="cuda")
    none = {"one": at == 150, "first": at < 140, "most": at % 9 != 4}[zeros]
    V = torch.where(none[:, None], torch.zeros_like(V), (V.double() * 2.0 ** power).to(torch.bfloat16))
    c = atf.new_kvcache(1, HKV, CAP, D, fmt)
    atf.atf_kvcache_write(c, K, V)
    O, LSE = _attend(c, Q, None)
    _check(fmt, Q, K, V, [CAP] * (D // 2), O, LSE, range(T))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("G", ROWS)
@pytest.mark.parametrize("zeros", ["first", "last"])
@pytest.mark.parametrize("low,high", [(-45, 45), (45, -45), (-90, -20), (100, 100)])
def test_rows_of_zeros_beside_sizes_that_change(fmt, G, zeros, low, high):
    """Whole blocks of zeros, whose weights count in every sum, beside values whose size changes along the text."""
    K, V, Q = _inputs(G)
    at = torch.arange(CAP, device="cuda")
    none = at < 140 if zeros == "first" else at >= 170
    power = low + (high - low) * at.double() / CAP
    V = torch.where(none[:, None], torch.zeros_like(V), (V.double() * torch.exp2(power)[:, None]).to(torch.bfloat16))
    c = atf.new_kvcache(1, HKV, CAP, D, fmt)
    atf.atf_kvcache_write(c, K, V)
    O, LSE = _attend(c, Q, None)
    _check(fmt, Q, K, V, [CAP] * (D // 2), O, LSE, range(T))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("G,nodes", [(1, 5), (2, 8), (3, 64)])
def test_sizes_that_change_along_the_text(fmt, G, nodes):
    """Values that grow and shrink by 2^80 along a long text, in steps and from row to row, over several splits."""
    length = 9000
    K, V, Q = _rows((1, HKV, length + nodes, D), 1), _rows((1, HKV, length + nodes, D), 2), _rows((1, HKV * G, nodes, D), 3)
    at = torch.arange(length + nodes, device="cuda", dtype=torch.float64)
    par = [i // 2 - 1 for i in range(nodes)]
    pt = torch.tensor(par, dtype=torch.int32, device="cuda")
    for power in (40 * torch.sin(at / 700), torch.floor(at / 1500) * 13 - 40, -torch.floor(at / 1500) * 13 + 40,
                  40 - 80 * torch.rand(at.shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda", dtype=torch.float64)):
        Vp = (V.double() * torch.exp2(power)[:, None]).to(torch.bfloat16)
        Kp = K.double().clone()
        Kp[..., 7] -= power * 2  # the larger the values, the smaller the weights where q[7] is positive, and the other way round
        Kp = Kp.to(torch.bfloat16)
        c = atf.new_kvcache(1, HKV, length + nodes, D, fmt)
        atf.atf_kvcache_write(c, Kp, Vp)
        O, LSE = atf.atf_decode_tree(Q, c, length, pt, return_lse=True)
        atf.binding.check_status()
        _check(fmt, Q, Kp, Vp, [length + nodes] * (D // 2), O, LSE, range(0, nodes, 7), par, length)
