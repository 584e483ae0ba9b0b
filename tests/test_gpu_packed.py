"""Packed attention (capped scores, prefix mask, dropout) against the fp64 oracle.

Tolerances (2-norm of the error over that of the result), from the roundings on
the way. A bf16 rounding is off by at most 2^-8 of the value:
  bf16 O: P and O are rounded, 2 * 2^-8; dQ, dK, dV: O inside D, dU (or P), and
  the result, 3 * 2^-8.
  fp32 outputs of bf16 inputs (LSE, dtable): a capped score in base 2 is a sum of
  terms of up to 2 cap log2 e <= 87 (cap 30), each off by half a step of 2^-24
  relative, the reciprocal by 2^-23: P is off by at most 87 (2^-23 + 2^-24) ln 2 = 1.1e-5,
  twice that for a difference from an LSE off as much: 2e-5.
  fp32: 30 (2^-23 + 2^-24) = 5.4e-6 from the cap in P the same way, twice that and the sums: 2e-5.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2609_34420_amd as gt
import synth
from gpu_common import DEV, rel_l2, say, to_dev, to_np

pytestmark = pytest.mark.gpu

TOL = {"bf16": dict(o=2 * 2.0 ** -8, grad=3 * 2.0 ** -8, f32=2e-5), "f32": dict(o=2e-5, grad=2e-5, f32=2e-5)}


def make(n_q, n_k, H, d, nb, dt, seed=0, gain=1.0, mask=0.0):
    """Host arrays of a packed batch; mask: share of -inf table entries."""
    g = np.random.default_rng(seed)
    td = torch.bfloat16 if dt == "bf16" else torch.float32

    def t(n, s):
        x = (s * g.standard_normal((H, n, d))).astype(np.float32)
        return synth.round_bf16(x) if dt == "bf16" else x

    tq, tk = sum(n_q), sum(n_k)
    a = dict(q=t(tq, gain), k=t(tk, gain), v=t(tk, 1), do=t(tq, 1), td=td,
             table=(0.5 * g.standard_normal((H, nb))).astype(np.float32),
             spd=g.integers(0, min(256, nb + 2), sum(x * y for x, y in zip(n_q, n_k))).astype(np.uint8))
    if mask:
        a["table"][g.random((H, nb)) < mask] = -np.inf
    return a


def upload(a):
    r = {k: to_dev(a[k], a["td"]) for k in ("q", "k", "v", "do")}
    r["spd"], r["table"] = to_dev(a["spd"], torch.uint8), to_dev(a["table"])
    return r


def compare(tag, dt, got, want, f32=None):
    names = ("O", "LSE", "dQ", "dK", "dV", "dtable")
    for name, x, y in zip(names, got, want):
        x = to_np(x)
        assert np.array_equal(np.isneginf(x), np.isneginf(y)), (tag, name, "-inf rows")
        fin = np.isfinite(y)
        assert np.isfinite(x[fin]).all(), (tag, name, "non-finite")
        e = rel_l2(x[fin], y[fin])
        lim = TOL[dt]["f32" if name in ("LSE", "dtable") else ("o" if name == "O" else "grad")]
        if f32 is not None and (dt == "f32" or name in ("LSE", "dtable")):
            lim = f32
        say(f"{tag}: {name} {e:.2e} (limit {lim:.1e})")
        assert e <= lim, (tag, name, e)


def check(tag, n_q, H, d, nb, dt, n_k=None, prefix=None, cap=None, drop=None, seed=0, gain=1.0, mask=0.0, bwd=True):
    say(tag)
    n_k = n_q if n_k is None else n_k
    a = make(n_q, n_k, H, d, nb, dt, seed, gain, mask)
    r = upload(a)
    pack = gt.gt_attn_pack(n_q, H, n_k=n_k, prefix=prefix, device=DEV)
    kw = dict(cap=cap, dropout=drop)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    o, lse = gt.gt_attn_pack_fwd(*args, **kw)
    got = [o, lse]
    scale = 1 / math.sqrt(d)
    okw = dict(cap=cap or 0.0, prefix=prefix, dropout=drop and (drop.p, drop.seed, drop.offset))
    want = list(oracle.packed_forward(a["q"], a["k"], a["v"], a["spd"], a["table"], scale, n_q, n_k, **okw))
    if bwd:
        got += gt.gt_attn_pack_bwd(*args, o, lse, r["do"], **kw)
        want += oracle.packed_backward(a["q"], a["k"], a["v"], a["spd"], a["table"], scale, a["do"], n_q, n_k, **okw)
    torch.cuda.synchronize()
    compare(tag, dt, got, want)
    return r, pack, got


RAGGED = [1, 31, 0, 32, 33, 64, 65, 100, 7, 129, 200]
DROP = gt.GTDropout(0.1, 0x0123456789abcdef, 0xfffffffe)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 16, 32, 64])
@pytest.mark.parametrize("cap,drop", [(None, None), (3.0, None), (None, DROP), (30.0, DROP)])
def test_ragged_batch(dt, d, cap, drop):
    check(f"ragged {dt} d={d} cap={cap} drop={drop is not None}", RAGGED, 2, d, 20, dt, cap=cap, drop=drop, gain=1.5)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("cap,drop", [(None, None), (5.0, gt.GTDropout(0.5, 3))])
@pytest.mark.parametrize("prefix", ["causal", "some", "past"])
def test_prefix_mask(dt, cap, drop, prefix):
    p = {"causal": 0, "some": 40, "past": 1000}[prefix]
    check(f"prefix {dt} {prefix} cap={cap}", RAGGED, 2, 32, 30, dt, prefix=[p] * len(RAGGED), cap=cap, drop=drop)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [None, 0, 50])
def test_more_keys_than_rows_and_the_other_way(dt, prefix):
    n_q, n_k = [1, 3, 40, 0, 70, 5, 129], [300, 0, 100, 9, 33, 5, 2]
    check(f"rectangles {dt} prefix={prefix}", n_q, 3, 64, 40, dt, n_k=n_k, cap=10.0, drop=DROP,
          prefix=None if prefix is None else [prefix] * len(n_q))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [16, 64])
@pytest.mark.parametrize("n", [1, 2, 33])
def test_new_rows_against_a_long_cache(dt, d, n):
    """Few rows, keys split over workgroups and merged."""
    n_q, n_k = [n, n], [6000, 2345]
    _, pack, _ = check(f"cache {dt} d={d} n={n}", n_q, 2, d, 64, dt, n_k=n_k, cap=30.0, drop=DROP, bwd=n == 2)
    assert pack._info.parts > 0
    check(f"cache causal {dt} d={d} n={n}", n_q, 2, d, 64, dt, n_k=n_k, prefix=[0, 100], bwd=n == 2)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_generation_in_node_order(dt):
    """Two graphs that grow node by node from the prefix they start with: each new
    row against the keys so far, on the stored tensors as they lie, is the row of
    the training forward (two results, each off by the tolerance)."""
    n, H, d, pre = [60, 70], 2, 32, [20, 45]
    r = upload(make(n, n, H, d, 22, dt, seed=17))
    full = gt.gt_attn_pack(n, H, prefix=pre, device=DEV)
    want, wl = gt.gt_attn_pack_fwd(r["q"], r["k"], r["v"], r["spd"], r["table"], full, cap=8.0)
    # each graph's keys at the start of a slab of its own, 80 rows a graph
    k, v = (torch.full((H, 160, d), float("nan"), device=DEV, dtype=r["q"].dtype) for _ in range(2))
    for x, y in ((k, r["k"]), (v, r["v"])):
        x[:, :60], x[:, 80:150] = y[:, :60], y[:, 60:]
    for g, (n0, k0, q0, s0) in enumerate(((60, 0, 0, 0), (70, 80, 60, 3600))):
        for t in range(pre[g] + 1, n0 + 1):
            pack = gt.gt_attn_pack([1], H, n_k=[t], prefix=[pre[g]], spd_off=[s0 + (t - 1) * n0], spd_ld=[n0], device=DEV,
                                   backward=False)
            row = q0 + t - 1
            o, lse = gt.gt_attn_pack_fwd(r["q"][:, row:row + 1], k[:, k0:], v[:, k0:], r["spd"], r["table"], pack, cap=8.0)
            assert rel_l2(to_np(o[:, 0]), to_np(want[:, row])) <= 2 * TOL[dt]["o"], (g, t)
            assert rel_l2(to_np(lse[:, 0]), to_np(wl[:, row])) <= 2 * TOL[dt]["f32"], (g, t)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("N", [300, 1000])
@pytest.mark.parametrize("H", [1, 40])
def test_split_and_unsplit_grids(dt, N, H):
    """Columns shared by 4, 2 or 1 groups of waves."""
    check(f"one graph {dt} N={N} H={H}", [N], H, 32, 22, dt, cap=20.0, drop=DROP)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("nb", [1, 2, 127, 128, 256])
def test_bucket_counts(dt, nb):
    check(f"buckets {dt} nb={nb}", [150, 40], 2, 16, nb, dt, cap=8.0)


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    """Seeded batches: sizes, heads, buckets, masks and options at random."""
    g = np.random.default_rng(1000 + seed)
    dt = ("bf16", "f32")[seed % 2]
    top = int(g.choice([6, 40, 130, 400]))
    n_k = [int(x) for x in g.integers(0, top + 1, int(g.integers(1, 24 if top < 400 else 5)))] + [top]
    n_q = n_k if g.random() < 0.6 else [int(x) for x in g.integers(0, int(g.choice([3, top + 20])) + 1, len(n_k))]
    if sum(n_q) == 0:
        n_q = n_k
    prefix = None if g.random() < 0.4 else [int(x) for x in g.integers(0, top + 2, len(n_k))]
    drop = None if g.random() < 0.5 else gt.GTDropout(float(g.uniform(0.02, 0.6)), int(g.integers(1 << 62)), int(g.integers(1 << 32)))
    # (a cap up to 30, uncapped scores up to some 8: the tolerances' sizes)
    check(f"random {seed}", n_q, int(g.choice([1, 3, 8])), int(g.choice([8, 16, 32, 64])), int(g.choice([1, 20, 64, 130, 256])),
          dt, n_k=n_k, prefix=prefix, cap=None if g.random() < 0.4 else float(g.uniform(1.0, 30.0)), drop=drop, seed=seed,
          mask=0.0 if g.random() < 0.7 else 0.2)


@pytest.mark.parametrize("drop", [None, gt.GTDropout(0.1, 21, 5)])
def test_table_gradient_of_many_pairs(drop):
    """The table gradient sums some millions of terms of either sign: roundings that
    lean to one side would show. Uncapped scores of up to 20 are 29 in base 2, rounded
    twice: P is off by up to 2 * 29 * 2^-24 ln 2 = 2.4e-6, twice that with the LSE's."""
    n, H, d, nb = [2500], 2, 8, 20
    a = make(n, n, H, d, nb, "bf16", seed=31)
    r = upload(a)
    pack = gt.gt_attn_pack(n, H, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    o, lse = gt.gt_attn_pack_fwd(*args, dropout=drop)
    got = gt.gt_attn_pack_bwd(*args, o, lse, r["do"], dropout=drop)[3]
    torch.cuda.synchronize()
    want = oracle.packed_backward(a["q"], a["k"], a["v"], a["spd"], a["table"], d ** -0.5, a["do"], n, n,
                                  dropout=drop and (drop.p, drop.seed, drop.offset))[3]
    e = rel_l2(to_np(got), want)
    say(f"table gradient of 2500 nodes: {e:.2e}")
    assert e <= 5e-6


@pytest.mark.parametrize("cap,drop", [(20.0, None), (None, DROP)])
def test_wide_fp32_on_a_full_grid(cap, drop):
    _, pack, _ = check("fp32 d=64, more workgroups than compute units", [400, 333, 260], 40, 64, 20, "f32", cap=cap, drop=drop)
    assert pack._info.jobs[1] * 40 > 256


@pytest.mark.parametrize("cap,drop", [(None, None), (9.0, None), (None, DROP), (9.0, DROP)])
@pytest.mark.parametrize("nb", [31, 32, 33, 63, 64, 65, 129])
def test_bucket_layouts(nb, cap, drop):
    """Buckets at the histogram's layouts' ends, with distances past the table and
    past the layout, in batches of the two-pass and the one-pass backward."""
    for n in ([150, 33], [60, 33]):
        H, d = 2, 16
        a = make(n, n, H, d, nb, "bf16", seed=22)
        a["spd"][::7] = 255
        a["spd"][3::7] = 129
        r = upload(a)
        pack = gt.gt_attn_pack(n, H, device=DEV)
        args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
        o, lse = gt.gt_attn_pack_fwd(*args, cap=cap, dropout=drop)
        got = gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=cap, dropout=drop)
        torch.cuda.synchronize()
        okw = dict(cap=cap or 0.0, dropout=drop and (drop.p, drop.seed, drop.offset))
        want = oracle.packed_backward(a["q"], a["k"], a["v"], a["spd"], a["table"], d ** -0.5, a["do"], n, n, **okw)
        compare(f"layout nb={nb} n={n}", "bf16", [o, lse, *got], [to_np(o), to_np(lse), *want])


def test_many_small_graphs():
    g = np.random.default_rng(5)
    check("many small", [int(x) for x in g.integers(1, 50, 300)], 4, 8, 22, "bf16", cap=20.0, drop=DROP)


@pytest.mark.parametrize("mask", [-1e9, float(np.finfo(np.float16).min)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_masked_entries_and_empty_rows(dt, mask):
    """Table masks (-inf, and large negative values, which count as one: the lowest
    of fp32 and of fp16, and -1e9), with rows that they leave nothing."""
    n = [70, 40]
    a = make(n, n, 2, 32, 10, dt, seed=4)
    a["table"][:, 3], a["table"][:, 4], a["table"][:, 5] = -np.inf, np.finfo(np.float32).min, mask
    for base, w in ((0, 70), (70 * 70, 40)):
        a["spd"][base + 7 * w:base + 8 * w] = 3 + np.arange(w) % 3        # row 7 of each graph
    r = upload(a)
    pack = gt.gt_attn_pack(n, 2, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    for cap in (None, 4.0):
        o, lse = gt.gt_attn_pack_fwd(*args, cap=cap)
        grads = gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=cap)
        torch.cuda.synchronize()
        okw = dict(cap=cap or 0.0)
        s = 1 / math.sqrt(32)
        want = (*oracle.packed_forward(a["q"], a["k"], a["v"], a["spd"], a["table"], s, n, n, **okw),
                *oracle.packed_backward(a["q"], a["k"], a["v"], a["spd"], a["table"], s, a["do"], n, n, **okw))
        compare(f"masks {dt} cap={cap}", dt, (o, lse, *grads), want)
        for row in (7, 77):
            assert bool((o[:, row] == 0).all()) and bool(torch.isneginf(lse[:, row]).all())
            assert bool((grads[0][:, row] == 0).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("nb", [9, 256])
def test_a_head_of_masks_alone(dt, nb):
    """Every entry of one head's table a mask (256 buckets: of every byte)."""
    n, H, d = [45, 130], 2, 16
    a = make(n, n, H, d, nb, dt, seed=16)
    a["spd"] %= min(nb, 255)
    a["table"][1] = -np.inf
    r = upload(a)
    pack = gt.gt_attn_pack(n, H, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    for cap in (None, 6.0):
        o, lse = gt.gt_attn_pack_fwd(*args, cap=cap, dropout=DROP)
        grads = gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=cap, dropout=DROP)
        torch.cuda.synchronize()
        assert bool((o[1] == 0).all()) and bool(torch.isneginf(lse[1]).all())
        assert all(bool((x[1] == 0).all()) for x in grads)
        assert all(bool(torch.isfinite(x[0].float()).all()) for x in (o, lse, *grads))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("cap,spread", [(200.0, 0.0), (30.0, 60.0), (30.0, 5.0), (1000.0, 0.0), (0.01, 0.0)])
def test_ranges_of_capped_scores(dt, cap, spread):
    """Caps and biases whose scores span more than a fixed reference allows, and
    less; biases of rows that differ by the spread. fp32 outputs: a cap of 200
    makes terms of up to 2 cap log2 e = 577 of the score, 577 (2^-23 + 2^-24) ln 2 = 7.2e-5,
    twice that. At a cap of 0.01 the slope 1 - tanh^2(u / cap) takes up u's rounding:
    a sum of 32 products of up to 10, times 0.18, is off by up to 32 * 10 * 0.18 * 2^-24 =
    3.4e-6, 3.4e-4 of the cap. A cap of 1000: 5 times that of 200, 7.2e-4, for O too."""
    n, H, d, nb = [70, 130], 2, 32, 12
    a = make(n, n, H, d, nb, dt, seed=12, gain=2.0)
    if spread:
        a["table"] += (spread * (np.arange(nb) % 3 - 1)).astype(np.float32)
    r = upload(a)
    pack = gt.gt_attn_pack(n, H, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    o, lse = gt.gt_attn_pack_fwd(*args, cap=cap)
    grads = gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=cap)
    torch.cuda.synchronize()
    assert all(bool(torch.isfinite(x.float()).all()) for x in (o, lse, *grads))
    s = d ** -0.5
    want = (*oracle.packed_forward(a["q"], a["k"], a["v"], a["spd"], a["table"], s, n, n, cap=cap),
            *oracle.packed_backward(a["q"], a["k"], a["v"], a["spd"], a["table"], s, a["do"], n, n, cap=cap))
    compare(f"range {dt} cap={cap} spread={spread}", dt, (o, lse, *grads), want, f32={200.0: 1.5e-4, 0.01: 3.4e-4, 1000.0: 7.2e-4}.get(cap))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_large_scores(dt):
    """Scores of some thousands, capped and not: no overflow, and saturated tanh."""
    n = [90]
    a = make(n, n, 2, 32, 8, dt, seed=9, gain=30.0)
    r = upload(a)
    pack = gt.gt_attn_pack(n, 2, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    for cap in (30.0, None):
        o, lse = gt.gt_attn_pack_fwd(*args, cap=cap)
        grads = gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=cap)
        torch.cuda.synchronize()
        want = oracle.packed_forward(a["q"], a["k"], a["v"], a["spd"], a["table"], 32 ** -0.5, n, n, cap=cap or 0.0)
        # uncapped scores of up to 2e4 are off by up to 2^-24 of that: P by 2e-3
        e = rel_l2(to_np(o), want[0])
        say(f"large {dt} cap={cap}: O {e:.2e}")
        assert e <= (TOL[dt]["o"] if cap else TOL[dt]["o"] + 3e-3)
        assert all(bool(torch.isfinite(x.float()).all()) for x in grads)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_nonfinite_values_stay_in_their_graph(bad):
    n, H = [20, 40, 9, 100, 33, 64], 2
    a = make(n, n, H, 32, 12, "bf16", seed=2)
    ref = upload(a)
    pack = gt.gt_attn_pack(n, H, device=DEV)

    def run(r):
        args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
        o, lse = gt.gt_attn_pack_fwd(*args, cap=9.0, dropout=DROP)
        return o, lse, *gt.gt_attn_pack_bwd(*args, ref_o[0], ref_o[1], r["do"], cap=9.0, dropout=DROP)

    ref_o = gt.gt_attn_pack_fwd(ref["q"], ref["k"], ref["v"], ref["spd"], ref["table"], pack, cap=9.0, dropout=DROP)
    want = run(ref)
    for name in ("q", "k", "v", "do"):
        r = dict(ref)
        r[name] = ref[name].clone()
        r[name][:, 25, 3] = bad                        # in the second graph, rows 20 .. 59
        got = run(r)
        torch.cuda.synchronize()
        for x, y in zip(got[:5], want[:5]):
            assert torch.equal(x[:, :20], y[:, :20]) and torch.equal(x[:, 60:], y[:, 60:]), name
        # (an infinite K gives scores of +-inf, which the cap makes +-cap: finite)
        if name == "v" or (name == "k" and math.isnan(bad)):
            assert not bool(torch.isfinite(got[0][:, 20:60].float()).all())
            assert bool(torch.isnan(got[5]).all())


def test_rows_behind_the_batch_and_layouts():
    """T beyond the batch's total: nothing there is read or written. Row-major
    [T, H, d] storage, K shared by the heads, padded distances."""
    n, H, d, T = [50, 21], 2, 32, 90
    a = make(n, n, H, d, 12, "bf16", seed=3)
    r = upload(a)
    pack = gt.gt_attn_pack(n, H, device=DEV)
    want = gt.gt_attn_pack_fwd(r["q"], r["k"], r["v"], r["spd"], r["table"], pack, cap=5.0)
    gw = gt.gt_attn_pack_bwd(r["q"], r["k"], r["v"], r["spd"], r["table"], pack, *want, r["do"], cap=5.0)
    nan = float("nan")

    def wide(x, layout):
        shape = (H, T, d) if layout == "htd" else (T, H, d)
        y = torch.full(shape, nan, device=DEV, dtype=x.dtype)
        y = y if layout == "htd" else y.transpose(0, 1)
        y[:, :x.shape[1]] = x
        return y

    # the same distances with row strides 64 and 33, the second graph's first
    ld, off = [64, 33], [33 * 21 + 5, 3]
    spd = torch.full((off[0] + 64 * 50,), 255, dtype=torch.uint8, device=DEV)
    for g, (s0, w) in enumerate(((0, 50), (2500, 21))):
        for i in range(w):
            spd[off[g] + i * ld[g]:off[g] + i * ld[g] + w] = r["spd"][s0 + i * w:s0 + (i + 1) * w]
    pack2 = gt.gt_attn_pack(n, H, spd_off=off, spd_ld=ld, device=DEV)
    for layout in ("htd", "thd"):
        x = {k: wide(r[k], layout) for k in ("q", "k", "v", "do")}
        out = wide(torch.zeros(H, 0, d, device=DEV, dtype=torch.bfloat16), layout)
        lse = torch.full((H, T), nan, device=DEV)
        gt.gt_attn_pack_fwd(x["q"], x["k"], x["v"], spd, r["table"], pack2, cap=5.0, out=out, lse=lse)
        grads = [wide(torch.zeros(H, 0, d, device=DEV, dtype=torch.bfloat16), layout) for _ in range(3)]
        grads.append(torch.empty_like(r["table"]))
        gt.gt_attn_pack_bwd(x["q"], x["k"], x["v"], spd, r["table"], pack2, out, lse, x["do"], cap=5.0, grads=grads)
        torch.cuda.synchronize()
        for y, w in zip((out, lse, *grads[:3]), (*want, *gw[:3])):
            assert torch.equal(y[:, :71], w) and bool(torch.isnan(y[:, 71:]).all()), layout
        assert torch.equal(grads[3], gw[3])
    shared = r["k"][:1].expand(H, -1, -1)
    got = gt.gt_attn_pack_fwd(r["q"], shared, r["v"], r["spd"], r["table"], pack)
    ref = gt.gt_attn_pack_fwd(r["q"], shared.contiguous(), r["v"], r["spd"], r["table"], pack)
    torch.cuda.synchronize()
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("cap,drop", [(None, None), (7.0, DROP)])
def test_gradients_scale_with_d_o(dt, cap, drop):
    """d_o times a power of two: every gradient times it, bit by bit (nothing
    of the fixed-point sums or the staged values leaves its range)."""
    n, H = [150, 40], 2
    r = upload(make(n, n, H, 32, 22, dt, seed=14))
    pack = gt.gt_attn_pack(n, H, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    o, lse = gt.gt_attn_pack_fwd(*args, cap=cap, dropout=drop)
    want = gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=cap, dropout=drop)
    for e in (-50, -25, 35, 60):
        got = gt.gt_attn_pack_bwd(*args, o, lse, r["do"] * 2.0 ** e, cap=cap, dropout=drop)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y * 2.0 ** e) for x, y in zip(got, want)), e


def test_offsets_past_32_bits():
    """Rows 2^23 elements apart, so that the last ones lie past 2^32 elements, in
    one buffer for all tensors; distances past 5 GiB; against dense tensors."""
    n, H, d, rs = [400, 150], 2, 32, 1 << 23
    r = upload(make(n, n, H, d, 22, "bf16", seed=15))
    pack = gt.gt_attn_pack(n, H, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    want = gt.gt_attn_pack_fwd(*args, cap=9.0)
    want = (*want, *gt.gt_attn_pack_bwd(*args, *want, r["do"], cap=9.0))
    T = sum(n)
    buf = torch.empty(T * rs, device=DEV, dtype=torch.bfloat16)
    q, k, v, do, o, dq, dk, dv = (buf.as_strided((H, T, d), (d, rs, 1), i * 1024) for i in range(8))
    for x, y in ((q, "q"), (k, "k"), (v, "v"), (do, "do")):
        x.copy_(r[y])
    off = [5 << 30, 17]
    spd = torch.empty(off[0] + n[0] * n[0], device=DEV, dtype=torch.uint8)
    spd[off[0]:] = r["spd"][:n[0] * n[0]]
    spd[off[1]:off[1] + n[1] * n[1]] = r["spd"][n[0] * n[0]:]
    pack = gt.gt_attn_pack(n, H, spd_off=off, device=DEV)
    args = (q, k, v, spd, r["table"], pack)
    lse = torch.empty_like(want[1])
    gt.gt_attn_pack_fwd(*args, cap=9.0, out=o, lse=lse)
    dt = torch.empty_like(r["table"])
    gt.gt_attn_pack_bwd(*args, o, lse, do, cap=9.0, grads=(dq, dk, dv, dt))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((o, lse, dq, dk, dv, dt), want))


# Batches whose graphs have at most 64 nodes take the one-pass backward in bf16.
SHORT = [1, 31, 0, 32, 33, 64, 9, 50, 2, 60]


@pytest.mark.parametrize("d", [8, 16, 32, 64])
@pytest.mark.parametrize("cap,drop", [(None, None), (3.0, None), (None, DROP), (30.0, DROP)])
@pytest.mark.parametrize("prefix", [None, "some"])
def test_short_batch(d, cap, drop, prefix):
    check(f"short d={d} cap={cap} drop={drop is not None} {prefix}", SHORT, 3, d, 20, "bf16", cap=cap, drop=drop,
          prefix=prefix and [0, 40, 0, 5, 33, 0, 9, 20, 1, 0])


@pytest.mark.parametrize("d", [8, 16, 32, 64])
@pytest.mark.parametrize("cap,drop", [(None, None), (3.0, None), (0.05, None), (None, DROP), (30.0, DROP)])
@pytest.mark.parametrize("prefix", [None, "some"])
def test_short_batch_of_four_blocks(d, cap, drop, prefix):
    """Up to 128 nodes, the second list of sizes with unlike sides."""
    n = [128, 65, 1, 33, 64, 0, 97, 96, 100, 31]
    kw = dict(cap=cap, drop=drop, prefix=prefix and [0, 40, 0, 5, 33, 0, 9, 120, 1, 0])
    check(f"four blocks d={d} cap={cap} drop={drop is not None} {prefix}", n, 3, d, 20, "bf16", **kw)
    check("unlike sides", n, 1, d, 20, "bf16", n_k=[3, 128, 70, 0, 100, 40, 97, 128, 1, 31], **kw)


@pytest.mark.parametrize("nb", [1, 31, 32, 64, 127, 128, 256])
def test_short_batch_buckets(nb):
    check(f"short nb={nb}", SHORT, 2, 16, nb, "bf16", cap=9.0)


def test_short_batch_unlike_sides():
    """Keys without queries, queries without keys, and one block against two."""
    check("short sides", [0, 5, 20, 64, 40, 1, 33], 2, 32, 12, "bf16", n_k=[40, 0, 64, 20, 33, 64, 32], cap=5.0, drop=DROP)
    check("short sides causal", [0, 5, 20, 64, 40, 1, 33], 2, 8, 12, "bf16", n_k=[40, 0, 64, 20, 33, 64, 32], prefix=[0] * 7)


def test_short_batch_of_unlike_gradients():
    """d_o of a graph up to 2^40 times another's, rising: the table gradient's scale
    falls from job to job, of which a workgroup has several."""
    n = [20 + g % 40 for g in range(800)]
    H, d, nb = 8, 8, 4
    a = make(n, n, H, d, nb, "bf16", seed=18)
    at = 0
    for g, w in enumerate(n):
        a["do"][:, at:at + w] *= 2.0 ** (40 * g // len(n) - 20)
        at += w
    r = upload(a)
    pack = gt.gt_attn_pack(n, H, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    o, lse = gt.gt_attn_pack_fwd(*args, cap=9.0)
    got = gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=9.0)
    torch.cuda.synchronize()
    assert pack._info.short_jobs > 2 * pack._info.short_slots
    want = oracle.packed_backward(a["q"], a["k"], a["v"], a["spd"], a["table"], d ** -0.5, a["do"], n, n, cap=9.0)
    at = 0
    for w in n[:8]:                                        # the smallest gradients keep their own precision
        for x, y in zip(got[:3], want[:3]):
            assert rel_l2(to_np(x[:, at:at + w]), y[:, at:at + w]) <= 4 * TOL["bf16"]["grad"]
        at += w
    compare("unlike gradients", "bf16", [o, lse, *got], [to_np(o), to_np(lse), *want])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_short_batch_nonfinite_and_repeated(bad):
    n, H = [20, 40, 9, 60, 33, 64] * 30, 2
    a = make(n, n, H, 32, 12, "bf16", seed=19)
    r = upload(a)
    pack = gt.gt_attn_pack(n, H, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    o, lse = gt.gt_attn_pack_fwd(*args, cap=9.0, dropout=DROP)
    want = gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=9.0, dropout=DROP)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=9.0, dropout=DROP), want))
    for e in (-45, 40):
        got = gt.gt_attn_pack_bwd(*args, o, lse, r["do"] * 2.0 ** e, cap=9.0, dropout=DROP)
        assert all(torch.equal(x, y * 2.0 ** e) for x, y in zip(got, want)), e
    do = r["do"].clone()
    do[0, 25, 3] = bad                                     # head 0, the second graph, rows 20 .. 59
    got = gt.gt_attn_pack_bwd(*args, o, lse, do, cap=9.0, dropout=DROP)
    torch.cuda.synchronize()
    for x, y in zip(got[:3], want[:3]):
        assert torch.equal(x[:, :20], y[:, :20]) and torch.equal(x[:, 60:], y[:, 60:]) and torch.equal(x[1], y[1])
    assert bool(torch.isnan(got[3][0]).all()) and torch.equal(got[3][1], want[3][1])


def test_short_batch_captured():
    n, H = [20, 40, 9, 60] * 40, 4
    r = upload(make(n, n, H, 16, 22, "bf16", seed=20))
    pack = gt.gt_attn_pack(n, H, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    step = lambda: (lambda f: (*f, *gt.gt_attn_pack_bwd(*args, *f, r["do"], dropout=DROP)))(
        gt.gt_attn_pack_fwd(*args, dropout=DROP))
    want = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), k
        step()
        torch.cuda.synchronize()


def test_empty_batches():
    H, d = 2, 16
    t = torch.zeros(H, 3, device=DEV)
    e = torch.zeros(H, 0, d, device=DEV, dtype=torch.bfloat16)
    spd = torch.zeros(0, dtype=torch.uint8, device=DEV)
    pack = gt.gt_attn_pack([0, 0], H, device=DEV)
    o, lse = gt.gt_attn_pack_fwd(e, e, e, spd, t, pack)
    g = gt.gt_attn_pack_bwd(e, e, e, spd, t, pack, o, lse, e)
    torch.cuda.synchronize()
    assert o.shape == (H, 0, d) and bool((g[3] == 0).all())
    x = torch.ones(H, 40, d, device=DEV, dtype=torch.bfloat16)
    pack = gt.gt_attn_pack([40, 0], H, n_k=[0, 40], device=DEV)      # rows without keys, keys without rows
    o, lse = gt.gt_attn_pack_fwd(x, x, x, spd, t, pack, cap=3.0)
    g = gt.gt_attn_pack_bwd(x, x, x, spd, t, pack, o, lse, x, cap=3.0)
    torch.cuda.synchronize()
    assert bool((o == 0).all()) and bool(torch.isneginf(lse).all())
    assert all(bool((y == 0).all()) for y in g)


def test_bitwise_reproducible():
    n = [700, 90, 33, 1200]
    a = make(n, n, 4, 64, 40, "bf16", seed=6)
    r = upload(a)
    pack = gt.gt_attn_pack(n, 4, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)

    def run():
        o, lse = gt.gt_attn_pack_fwd(*args, cap=20.0, dropout=DROP)
        return o, lse, *gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=20.0, dropout=DROP)

    want = run()
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(run(), want))


def test_dropout_is_the_generators():
    """V of unit vectors shows each kept pair; its share and place are the
    oracle's; another offset gives another mask, offset_dev adds to offset."""
    n, H, d, p = 64, 2, 64, 0.3
    q = torch.zeros(H, n, d, device=DEV)
    v = torch.eye(n, device=DEV).expand(H, n, n).contiguous()
    t, spd = torch.zeros(H, 1, device=DEV), torch.zeros(n * n, dtype=torch.uint8, device=DEV)
    pack = gt.gt_attn_pack([n], H, device=DEV)

    def mask(**kw):
        return gt.gt_attn_pack_fwd(q, q, v, spd, t, pack, dropout=gt.GTDropout(p, 99, **kw))[0] > 0

    got = mask(offset=5)
    for h in range(H):
        assert np.array_equal(got[h].cpu().numpy(), oracle.keep_mask(range(n), n, h, p, 99, 5) > 0)
    assert not torch.equal(got, mask(offset=6))
    dyn = torch.tensor([-1], dtype=torch.int32, device=DEV)
    assert torch.equal(got, mask(offset=6, offset_dev=dyn))


def test_captured_steps_draw_anew():
    """A training step captured into a graph and replayed, with eager work and
    synchronisation between the replays; the offset moves on the device."""
    n, H = [300, 45], 4
    a = make(n, n, H, 32, 22, "bf16", seed=8)
    r = upload(a)
    pack = gt.gt_attn_pack(n, H, device=DEV)
    dyn = torch.zeros(1, dtype=torch.int32, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)

    def step(drop):
        o, lse = gt.gt_attn_pack_fwd(*args, cap=20.0, dropout=drop)
        return o, lse, *gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=20.0, dropout=drop)

    drop = gt.GTDropout(0.2, 7, 100, dyn)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(drop)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(drop)
        dyn.add_(1)
    dyn.zero_()
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = step(gt.GTDropout(0.2, 7, 100 + k))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), k


def test_streams_and_workspaces():
    """Two streams at once with workspaces of the caller's and of the call's own."""
    n, H = [400, 100], 4
    runs = []
    for seed in (1, 2):
        r = upload(make(n, n, H, 32, 22, "bf16", seed=seed))
        pack = gt.gt_attn_pack(n, H, device=DEV)
        args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
        o, lse = gt.gt_attn_pack_fwd(*args, dropout=DROP)
        runs.append((args, r["do"], (o, lse, *gt.gt_attn_pack_bwd(*args, o, lse, r["do"], dropout=DROP))))
    torch.cuda.synchronize()
    need = gt.gt_attn_pack_bwd_workspace_size(runs[0][0][5], 22)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ws = [None, torch.empty(need, dtype=torch.uint8, device=DEV)]
    for _ in range(3):
        got = []
        for (args, do, _), s, w in zip(runs, streams, ws):
            o, lse = gt.gt_attn_pack_fwd(*args, dropout=DROP, stream=s)
            got.append((o, lse, *gt.gt_attn_pack_bwd(*args, o, lse, do, dropout=DROP, workspace=w, stream=s)))
        torch.cuda.synchronize()
        for (_, _, want), g in zip(runs, got):
            assert all(torch.equal(x, y) for x, y in zip(g, want))
    with pytest.raises(ValueError, match="workspace"):
        gt.gt_attn_pack_bwd(*runs[0][0], *runs[0][2][:2], runs[0][1], workspace=ws[1][:need - 1])


@pytest.mark.parametrize("how", ["current", "argument"])
def test_plan_outlives_a_call_on_another_stream(how):
    """A plan dropped while a side stream still has the call before it: its memory
    is not handed out again until that stream has passed."""
    n, H = [300, 45], 2
    r = upload(make(n, n, H, 32, 22, "bf16", seed=23))
    pack = gt.gt_attn_pack(n, H, device=DEV)
    args = [r["q"], r["k"], r["v"], r["spd"], r["table"]]
    want = gt.gt_attn_pack_fwd(*args, pack)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
        if how == "current":
            got = gt.gt_attn_pack_fwd(*args, pack)
    if how == "argument":
        got = gt.gt_attn_pack_fwd(*args, pack, stream=side)
    at, size = pack._plan.data_ptr(), pack._plan.untyped_storage().nbytes()
    del pack
    new = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(64)]
    assert all(x.data_ptr() != at for x in new)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_agrees_with_the_unpacked_calls():
    """No option on: the packed call is the framework's attention of each graph."""
    n, H, d = [256, 77, 500], 2, 32
    a = make(n, n, H, d, 22, "bf16", seed=11)
    r = upload(a)
    pack = gt.gt_attn_pack(n, H, device=DEV)
    o, lse = gt.gt_attn_pack_fwd(r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    grads = gt.gt_attn_pack_bwd(r["q"], r["k"], r["v"], r["spd"], r["table"], pack, o, lse, r["do"])
    s0 = t0 = 0
    dt = torch.zeros_like(r["table"])
    for w in n:
        x = [r[k][:, t0:t0 + w].contiguous() for k in ("q", "k", "v", "do")]
        m = r["spd"][s0:s0 + w * w].view(w, w).clone()
        oo, ll = gt.gt_attn_fwd(*x[:3], m, r["table"])
        gg = gt.gt_attn_bwd(*x[:3], m, r["table"], oo, ll, x[3])
        # two results, each off by the bf16 tolerances
        for y, z, tol in zip((o, *grads[:3]), (oo, *gg[:3]), (2, 3, 3, 3)):
            assert rel_l2(to_np(y[:, t0:t0 + w]), to_np(z)) <= 2 * tol * 2.0 ** -8
        dt += gg[3]
        s0, t0 = s0 + w * w, t0 + w
    # the unpacked table gradient takes D from the rounded O
    assert rel_l2(to_np(grads[3]), to_np(dt)) <= 1e-2
