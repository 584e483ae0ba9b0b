"""Pins of the packed oracle (CPU): published Philox vectors, the plain oracle
where no option is on, central differences with every option on, and the
masks' meaning."""
import math

import numpy as np
import pytest

import oracle
from oracle.packed import graph_forward


def _case(nq, nk, d, nb, seed=0):
    g = np.random.default_rng(seed)
    q, k, v, do = (g.standard_normal((n, d)) for n in (nq, nk, nk, nq))
    return q, k, v, do, g.integers(0, nb + 2, (nq, nk)).astype(np.uint8), 0.5 * g.standard_normal(nb)


@pytest.mark.parametrize("rounds,ctr,key,want", [
    # known answers published with the generator's reference implementation
    (10, 0, 0, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
    (10, 0xffffffff, 0xffffffff, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
    (7, 0, 0, "5f6fb709 0d893f64 4f121f81 4f730a48"),
])
def test_philox_known_answers(rounds, ctr, key, want):
    got = oracle.philox4x32([np.uint64(ctr)] * 4, (key, key), rounds)
    assert " ".join(f"{int(x):08x}" for x in got) == want


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.97])
def test_keep_rate(p):
    z = oracle.keep_mask(range(400), 1000, 3, p, 0x123456789abcdef0, 17)
    t = math.floor(p * 65536 + 0.5) / 65536
    # 400000 draws: the mean is within 5 standard deviations
    assert abs(z.mean() - (1 - t)) <= 5 * math.sqrt(t * (1 - t) / z.size)
    if p:
        for kw in (dict(head=4), dict(seed=0x123456789abcdef1), dict(seed=0x123456799abcdef0), dict(offset=18)):
            a = dict(head=3, seed=0x123456789abcdef0, offset=17) | kw
            y = oracle.keep_mask(range(400), 1000, a["head"], p, a["seed"], a["offset"])
            # another stream agrees as often as chance has it
            assert abs((y == z).mean() - ((1 - t) ** 2 + t ** 2)) <= 0.01


def test_keep_mask_goes_by_the_packed_row():
    z = oracle.keep_mask(range(20), 50, 1, 0.3, 5, 6)
    assert np.array_equal(oracle.keep_mask(range(7, 20), 33, 1, 0.3, 5, 6), z[7:, :33])


def test_plain_where_no_option_is_on():
    n_q, H, d, nb = [5, 1, 30], 2, 8, 6
    g = np.random.default_rng(1)
    q, k, v, do = (g.standard_normal((H, sum(n_q), d)) for _ in range(4))
    table = g.standard_normal((H, nb))
    mats = [g.integers(0, nb + 1, (n, n)).astype(np.uint8) for n in n_q]
    spd = np.concatenate([m.ravel() for m in mats])
    o, lse = oracle.packed_forward(q, k, v, spd, table, 0.4, n_q, n_q)
    grads = oracle.packed_backward(q, k, v, spd, table, 0.4, do, n_q, n_q)
    a, dt = 0, 0.0
    for n, m in zip(n_q, mats):
        s = slice(a, a + n)
        ro, rl = oracle.forward(q[:, s], k[:, s], v[:, s], m, table, 0.4)
        rg = oracle.backward(q[:, s], k[:, s], v[:, s], m, table, 0.4, do[:, s])
        assert np.allclose(o[:, s], ro, atol=1e-13) and np.allclose(lse[:, s], rl, atol=1e-13)
        for x, y in zip(grads[:3], rg[:3]):
            assert np.allclose(x[:, s], y, atol=1e-12)
        dt = dt + rg[3]
        a += n
    assert np.allclose(grads[3], dt, atol=1e-12)


@pytest.mark.parametrize("cap", [0.0, 1.5])
@pytest.mark.parametrize("prefix", [None, 0, 3])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_gradients_against_differences(cap, prefix, p):
    nq, nk, d, nb = 6, 9, 4, 5
    q, k, v, do, spd, table = _case(nq, nk, d, nb)
    z = oracle.keep_mask(range(nq), nk, 0, p, 7, 8) if p else None
    kw = dict(cap=cap, prefix=prefix, keep=z, p=p)

    def loss(q, k, v, table):
        return float((graph_forward(q, k, v, spd, table, 0.6, **kw)[0] * do).sum())

    from oracle.packed import graph_backward
    grads = graph_backward(q, k, v, spd, table, 0.6, do, **kw)
    args, eps = [q, k, v, table], 1e-5
    for n, gr in enumerate(grads):
        num = np.zeros_like(args[n])
        for ix in np.ndindex(num.shape):
            for sgn in (1, -1):
                x = [a.copy() for a in args]
                x[n][ix] += sgn * eps
                num[ix] += sgn * loss(*x) / (2 * eps)
        # truncation eps^2 times third derivatives of order ten, rounding 1e-15 / eps
        assert np.abs(num - gr).max() <= 1e-8, n


def test_cap_bounds_and_vanishes():
    q, k, v, _, spd, table = _case(4, 5, 8, 3)
    o, lse = graph_forward(40 * q, k, v, spd, 0 * table, 1.0, cap=2.0)
    assert np.all(lse <= 2.0 + math.log(5)) and np.all(lse >= -2.0 + math.log(5))
    a = graph_forward(q, k, v, spd, table, 0.3, cap=1e7)
    b = graph_forward(q, k, v, spd, table, 0.3)
    # u - cap tanh(u / cap) = u^3 / (3 cap^2) to first order
    assert np.allclose(a[0], b[0], atol=1e-12) and np.allclose(a[1], b[1], atol=1e-12)


def test_masks_that_leave_nothing():
    q, k, v, do, spd, table = _case(5, 3, 8, 4)
    # two more queries than keys: the first two stand before every key
    o, lse = graph_forward(q, k, v, spd, table, 0.5, prefix=0)
    assert np.all(o[:2] == 0) and np.all(np.isneginf(lse[:2])) and np.all(np.isfinite(lse[2:]))
    assert np.allclose(o[2], v[0])
    low = np.full(4, -3.4028234663852886e38)
    spd = np.minimum(spd, 3)
    o, lse = graph_forward(q, k, v, spd, low, 0.5)
    assert np.all(o == 0) and np.all(np.isneginf(lse))
    # a prefix shows its keys to every row
    _, a = graph_forward(q, k, v, spd, table, 0.5, prefix=3)
    _, b = graph_forward(q, k, v, spd, table, 0.5)
    assert np.array_equal(a, b)
