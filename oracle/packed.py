"""Reference (oracle) of packed attention with capped scores, a prefix mask and
dropout, in fp64 NumPy. TEST INFRASTRUCTURE.

One graph and one head at a time, with the full score matrix. Pinned by
tests/test_packed_oracle.py: the published Philox vectors, the plain oracle
where no option is on, and central differences for every gradient.

    u = scale q_i . k_j          c = cap tanh(u / cap)   (u without a cap)
    S = c + bias                 row i sees key j if j < prefix or j <= i + n_k - n_q
    P = softmax over seen keys   O = (P z / (1 - p)) V
"""
from __future__ import annotations

import numpy as np

from .attention import bias_block

__all__ = ["philox4x32", "keep_mask", "graph_forward", "graph_backward", "packed_forward", "packed_backward"]

_M32 = np.uint64(0xFFFFFFFF)


def philox4x32(ctr, key, rounds: int):
    """Philox4x32 of a [4, ...] counter and a (low, high) key, as the definition
    has it: two 32 x 32 bit products per round, the key raised after each."""
    c = [np.asarray(x, dtype=np.uint64) for x in ctr]
    k = [np.uint64(key[0]), np.uint64(key[1])]
    for _ in range(rounds):
        a = c[0] * np.uint64(0xD2511F53)
        b = c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & _M32, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & _M32]
        k = [(k[0] + np.uint64(0x9E3779B9)) & _M32, (k[1] + np.uint64(0xBB67AE85)) & _M32]
    return np.stack(c)


def keep_mask(rows, n_k: int, head: int, p: float, seed: int, offset: int) -> np.ndarray:
    """z [len(rows), n_k] of packed rows `rows`: 1 where the pair is kept."""
    t = int(np.floor(p * 65536 + 0.5))
    rows = np.asarray(rows, dtype=np.uint64)
    z = np.ones((len(rows), n_k), dtype=np.float64)
    if t == 0:
        return z
    j8 = np.arange((n_k + 7) // 8, dtype=np.uint64)
    shape = (len(rows), len(j8))
    ctr = [np.broadcast_to(j8, shape), np.broadcast_to(rows[:, None], shape),
           np.full(shape, head, np.uint64), np.full(shape, offset & 0xFFFFFFFF, np.uint64)]
    w = philox4x32(ctr, (seed & 0xFFFFFFFF, seed >> 32), 7)
    for j in range(n_k):
        word = w[(j % 8) // 2, :, j // 8]
        half = ((word >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF)).astype(np.int64)
        signed = np.where(half >= 32768, half - 65536, half)
        z[:, j] = signed >= t - 32768
    return z


def _rate(p: float) -> float:
    return 65536.0 / (65536 - int(np.floor(p * 65536 + 0.5)))


def _probabilities(q, k, spd, table_h, scale, cap, prefix):
    """P, LSE and dc/du of one graph and head."""
    nq, nk = q.shape[0], k.shape[0]
    u = scale * (q @ k.T)
    t = np.tanh(u / cap) if cap else None
    tab = np.asarray(table_h, dtype=np.float64)
    S = (cap * t if cap else u) + bias_block(spd, np.where(tab <= -6e4, -np.inf, tab))
    if prefix is not None:
        i, j = np.arange(nq)[:, None], np.arange(nk)[None]
        S = np.where((j < prefix) | (j <= i + nk - nq), S, -np.inf)
    m = S.max(1, initial=-np.inf)
    e = np.exp(S - np.where(np.isneginf(m), 0.0, m)[:, None])
    l = e.sum(1)
    with np.errstate(divide="ignore"):
        lse = np.where(l > 0, m + np.log(np.where(l > 0, l, 1.0)), -np.inf)
    return e / np.where(l > 0, l, 1.0)[:, None], lse, (1.0 - t * t if cap else 1.0)


def graph_forward(q, k, v, spd, table_h, scale, cap=0.0, prefix=None, keep=None, p=0.0):
    """O, LSE of one graph and head; keep: z, or None."""
    P, lse, _ = _probabilities(q, k, spd, table_h, scale, cap, prefix)
    return (P if keep is None else P * keep * _rate(p)) @ v, lse


def graph_backward(q, k, v, spd, table_h, scale, d_o, cap=0.0, prefix=None, keep=None, p=0.0):
    """dQ, dK, dV, dtable of L = sum(O dO) of one graph and head."""
    P, _, slope = _probabilities(q, k, spd, table_h, scale, cap, prefix)
    z = 1.0 if keep is None else keep * _rate(p)
    O = (P * z) @ v
    dS = P * (z * (d_o @ v.T) - (d_o * O).sum(1, keepdims=True))
    dt = np.zeros(len(table_h))
    inside = spd < len(table_h)
    np.add.at(dt, spd[inside], dS[inside])
    dU = dS * slope
    return scale * (dU @ k), scale * (dU.T @ q), (P * z).T @ d_o, dt


def _walk(n_q, n_k, spd, spd_off, spd_ld):
    a = b = s = 0
    for g, (x, y) in enumerate(zip(n_q, n_k)):
        off = s if spd_off is None else spd_off[g]
        ld = y if spd_ld is None else spd_ld[g]
        if x and y:
            m = np.lib.stride_tricks.as_strided(spd[off:], (x, y), (ld, 1))
        else:
            m = np.zeros((x, y), np.uint8)
        yield g, slice(a, a + x), slice(b, b + y), m
        a, b, s = a + x, b + y, s + x * ld


def packed_forward(q, k, v, spd, table, scale, n_q, n_k, cap=0.0, prefix=None, dropout=None, spd_off=None, spd_ld=None):
    """O, LSE of a packed batch: q [H, T_q, d], k, v [H, T_k, d], spd flat uint8;
    dropout: (p, seed, offset) or None."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    o, lse = np.zeros_like(q), np.zeros(q.shape[:2])
    for g, a, b, m in _walk(n_q, n_k, spd, spd_off, spd_ld):
        for h in range(q.shape[0]):
            z = None if dropout is None else keep_mask(range(a.start, a.stop), n_k[g], h, *dropout)
            o[h, a], lse[h, a] = graph_forward(q[h, a], k[h, b], v[h, b], m, table[h], scale, cap,
                                               None if prefix is None else prefix[g], z, dropout[0] if dropout else 0.0)
    return o, lse


def packed_backward(q, k, v, spd, table, scale, d_o, n_q, n_k, cap=0.0, prefix=None, dropout=None, spd_off=None,
                    spd_ld=None):
    """dQ, dK, dV, dtable of a packed batch."""
    q, k, v, d_o = (np.asarray(x, dtype=np.float64) for x in (q, k, v, d_o))
    dq, dk, dv, dt = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros(np.shape(table))
    for g, a, b, m in _walk(n_q, n_k, spd, spd_off, spd_ld):
        for h in range(q.shape[0]):
            z = None if dropout is None else keep_mask(range(a.start, a.stop), n_k[g], h, *dropout)
            x = graph_backward(q[h, a], k[h, b], v[h, b], m, table[h], scale, d_o[h, a], cap,
                               None if prefix is None else prefix[g], z, dropout[0] if dropout else 0.0)
            dq[h, a], dk[h, b], dv[h, b] = x[:3]
            dt[h] += x[3]
    return dq, dk, dv, dt
