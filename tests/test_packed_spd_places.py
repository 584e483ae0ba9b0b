"""Strides of a packed batch's distances without places: padded matrices one behind the
other (CPU only)."""
import numpy as np

import oracle
import paper_2609_34420_amd as gt
from test_packed_no_pairs import records


def test_strides_without_places():
    pack = gt.gt_attn_pack([10, 10], 2, spd_ld=[64, 64], device="cpu")
    w = records(pack)
    w = w[w["nq"] > 0]
    assert set(zip(w["q0"].tolist(), w["spd"].tolist(), w["ld"].tolist())) == {(0, 0, 64), (10, 640, 64)}
    assert pack.spd_bytes == 640 + 9 * 64 + 10
    n_q, n_k, ld = [3, 0, 40, 5, 200], [7, 9, 0, 5, 130], [16, 9, 33, 5, 160]
    a = gt.gt_attn_pack(n_q, 2, n_k=n_k, spd_ld=ld, device="cpu")
    off = np.concatenate([[0], np.cumsum(np.array(n_q) * ld)[:-1]])
    b = gt.gt_attn_pack(n_q, 2, n_k=n_k, spd_ld=ld, spd_off=off, device="cpu")
    assert a.spd_bytes == b.spd_bytes and np.array_equal(records(a), records(b))
    c = gt.gt_attn_pack(n_q, 2, n_k=n_k, spd_ld=n_k, device="cpu")          # the dense layout
    e = gt.gt_attn_pack(n_q, 2, n_k=n_k, device="cpu")
    assert c.spd_bytes == e.spd_bytes
    pairs = records(e)["nq"] * records(e)["nk"] > 0
    assert np.array_equal(records(c)[pairs], records(e)[pairs])


def test_the_oracle_has_the_same_strides():
    g = np.random.default_rng(0)
    n, ld = [4, 6], [9, 6]
    m = [g.integers(0, 5, (x, x)).astype(np.uint8) for x in n]
    padded = np.full(4 * 9 + 36, 255, np.uint8)
    padded[:36].reshape(4, 9)[:, :4], padded[36:] = m[0], m[1].ravel()
    x = [g.standard_normal((2, 10, 8)) for _ in range(3)]
    t = g.standard_normal((2, 5))
    a = oracle.packed_forward(*x, np.concatenate([y.ravel() for y in m]), t, 0.3, n, n)
    b = oracle.packed_forward(*x, padded, t, 0.3, n, n, spd_ld=ld)
    assert all(np.array_equal(u, v) for u, v in zip(a, b))
