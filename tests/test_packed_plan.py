"""Plans of packed batches and the packed calls' refusals (CPU only)."""
import ctypes
import random

import numpy as np
import pytest
import torch

import paper_2609_34420_amd as gt

WAVE = np.dtype([(n, "<i4") for n in ("q0", "nq", "k0", "nk", "row", "c0", "c1", "prefix")]
                + [("spd", "<i8")] + [(n, "<i4") for n in ("ld", "part", "log2w", "combine", "steps", "pad")])
MERGE = np.dtype([(n, "<i4") for n in ("row", "rows", "part", "parts")])
FULL = np.iinfo(np.int32).max


def lists(pack):
    i, buf = pack._info, pack._plan.numpy()
    out = []
    for s in range(3):
        out.append(buf[i.job_off[s]:][:4 * i.jobs[s] * WAVE.itemsize].view(WAVE).reshape(-1, 4))
    return out, buf[i.merge_off:][:i.merges * MERGE.itemsize].view(MERGE)


def visible(nq, nk, prefix):
    i, j = np.arange(nq)[:, None], np.arange(nk)[None]
    return np.ones((nq, nk), bool) if prefix is None else (j < prefix) | (j <= i + nk - nq)


def check(n_q, n_k, prefix, H):
    pack = gt.gt_attn_pack(n_q, H, n_k=n_k, prefix=prefix, device="cpu")
    stages, merges = lists(pack)
    starts = {}
    a = b = s = 0
    for g, (x, y) in enumerate(zip(n_q, n_k)):
        if x or y:
            starts[(a, x, b, y)] = g
        a, b, s = a + x, b + y, s + x * y
    assert (pack.total_q, pack.total_k) == (a, b)
    assert 0 < pack._info.slots <= len(stages[2]) or len(stages[2]) == 0
    for st, jobs in enumerate(stages):
        seen = [np.zeros((x, y), np.int32) for x, y in zip(n_q, n_k)]
        rows_done = [np.zeros(y if st == 2 else x, np.int32) for x, y in zip(n_q, n_k)]
        parts = {}
        for waves in jobs:
            job = waves[0]
            w = 1 << job["log2w"]
            assert w in (1, 2, 4)
            same = [n for n in WAVE.names if n != "row"]
            for k in range(0, 4, w):                       # a group's waves: 32 rows after 32 rows
                for e in range(w):
                    assert all(waves[k + e][n] == waves[k][n] for n in same)
                    assert waves[k + e]["row"] == waves[k]["row"] + 32 * e
            assert all(x[n] == job[n] for x in waves for n in ("log2w", "combine", "steps"))
            mine = waves[::w]
            if job["combine"]:
                assert len({(x["q0"], x["nq"], x["k0"], x["nk"], x["row"], x["part"]) for x in mine}) == 1
            for k, x in enumerate(mine):
                n_rows, n_cols = (x["nk"], x["nq"]) if st == 2 else (x["nq"], x["nk"])
                if n_rows == 0 and n_cols == 0:
                    assert x["part"] == -1 and x["c0"] == x["c1"] == 0        # no graph
                    continue
                g = starts[(x["q0"], x["nq"], x["k0"], x["nk"])]
                assert x["prefix"] == (FULL if prefix is None else prefix[g]) and x["ld"] == n_k[g]
                assert x["spd"] == sum(p * q for p, q in zip(n_q[:g], n_k[:g]))
                assert x["row"] % 32 == 0 and x["c0"] % 32 == 0 and 0 <= x["c0"] <= x["c1"] or x["c0"] >= x["c1"]
                assert x["c1"] <= n_cols or x["c0"] >= x["c1"]
                assert job["steps"] * 32 * w >= x["c1"] - x["c0"]
                r = slice(x["row"], min(n_rows, x["row"] + 32 * w))
                c = slice(x["c0"], max(x["c0"], x["c1"]))
                if st == 2:
                    seen[g][c, r] += 1
                else:
                    seen[g][r, c] += 1
                if x["part"] >= 0:
                    assert st == 0 and job["combine"] and w == 1
                    parts.setdefault(int(x["part"]), (g, r.start))
                if not job["combine"] or k == 0:
                    if x["part"] < 0:
                        rows_done[g][r] += 1
        if st == 0:
            assert sorted(parts) == list(range(pack._info.parts))
            for m in merges:
                at = {parts[p] for p in range(m["part"], m["part"] + m["parts"])}
                assert len(at) == 1
                g, r0 = at.pop()
                assert m["row"] == sum(n_q[:g]) + r0 and m["rows"] == min(32, n_q[g] - r0)
                rows_done[g][r0:r0 + m["rows"]] += 1
        for g, (x, y) in enumerate(zip(n_q, n_k)):
            vis = visible(x, y, None if prefix is None else prefix[g])
            assert seen[g].max(initial=0) <= 1 and np.all(seen[g][vis] == 1), (st, g)
            assert np.all(rows_done[g] == 1), (st, g)
    return pack


@pytest.mark.parametrize("n_q", [[1], [0], [200], [32, 33, 64, 65, 128, 129, 0, 1], [9] * 50, [3000], [5, 700, 20]])
@pytest.mark.parametrize("H", [1, 8])
@pytest.mark.parametrize("mask", ["full", "causal", "prefix"])
def test_training_plans_cover_every_pair_once(n_q, H, mask):
    prefix = {"full": None, "causal": [0] * len(n_q), "prefix": [n // 3 for n in n_q]}[mask]
    check(n_q, n_q, prefix, H)


@pytest.mark.parametrize("H", [1, 8, 200])
def test_new_rows_against_many_keys(H):
    pack = check([1, 2, 1, 40], [5000, 0, 17, 3000], None, H)
    assert (pack._info.parts > 0) == (H < 200)          # few rows: their keys are split over workgroups
    check([1, 2, 1, 40], [5000, 0, 17, 3000], [0, 0, 3, 2000], H)
    check([50, 7], [3, 0], [0, 0], H)                  # rows that stand before every key


def test_random_plans():
    rng = random.Random(3)
    for _ in range(40):
        G = rng.randint(1, 30)
        top = rng.choice([5, 100, 600])
        n_k = [rng.randint(0, top) for _ in range(G)]
        n_q = list(n_k) if rng.random() < 0.5 else [rng.randint(0, rng.choice([2, top])) for _ in range(G)]
        prefix = None if rng.random() < 0.4 else [rng.randint(0, top) for _ in range(G)]
        check(n_q, n_k, prefix, rng.choice([1, 4, 16]))


def test_plans_of_the_forward_alone():
    """The forward's list is the same; the backward refuses the plan."""
    n_q, n_k = [1, 3, 40, 0], [900, 5000, 40, 7]
    a = gt.gt_attn_pack(n_q, 4, n_k=n_k, device="cpu")
    b = gt.gt_attn_pack(n_q, 4, n_k=n_k, device="cpu", backward=False)
    (x, y), (u, v) = lists(a), lists(b)
    assert np.array_equal(x[0], u[0]) and np.array_equal(y, v) and len(u[1]) == len(u[2]) == 0
    assert b._plan.numel() < a._plan.numel() and a.backward and not b.backward
    assert (a.total_q, a.total_k, a.spd_bytes) == (b.total_q, b.total_k, b.spd_bytes)


def test_stages_share_a_list_where_they_can():
    off = lambda **kw: list(gt.gt_attn_pack([700, 33, 90], 8, device="cpu", **kw)._info.job_off)
    a, b = off(), off(prefix=[0, 5, 90])
    assert a[0] == a[1] == a[2]
    assert b[0] == b[1] < b[2]


def test_short_list_has_every_graph_once():
    def short(n_q, **kw):
        p = gt.gt_attn_pack(n_q, 4, device="cpu", **kw)
        i = p._info
        return p, p._plan.numpy()[i.short_off:][:4 * i.short_jobs * WAVE.itemsize].view(WAVE).reshape(-1, 4)

    n_q = [1, 31, 0, 32, 33, 64, 9, 50, 2, 60, 5, 0, 128, 65, 3]
    n_k = [1, 31, 7, 0, 64, 20, 9, 50, 40, 60, 5, 0, 7, 128, 96]
    p, jobs = short(n_q, n_k=n_k, prefix=list(range(15)))
    assert 0 < p._info.short_slots <= p._info.short_jobs
    seen = []
    for job in jobs:
        lw = int(job[0]["log2w"])
        assert (job["log2w"] == lw).all()
        for grp in range(4 >> lw):
            w = job[grp << lw:(grp + 1) << lw]
            if max(w[0]["nq"], w[0]["nk"]) == 0:
                continue
            assert list(w["row"]) == [32 * k for k in range(1 << lw)]
            assert max(w[0]["nq"], w[0]["nk"]) <= 32 << lw and max(w[0]["nq"], w[0]["nk"]) > [0, 32, 64][lw]
            assert all((w[f] == w[0][f]).all() for f in ("q0", "nq", "k0", "nk", "prefix", "spd", "ld"))
            seen.append(tuple(int(w[0][f]) for f in ("q0", "nq", "k0", "nk", "prefix")))
    a = np.concatenate([[0], np.cumsum(n_q)])
    b = np.concatenate([[0], np.cumsum(n_k)])
    assert sorted(seen) == sorted((int(a[g]), n_q[g], int(b[g]), n_k[g], g) for g in range(15) if n_q[g] or n_k[g])
    blocks = lambda *a, **kw: (lambda i: (i.short_jobs, i.short_blocks))(short(*a, **kw)[0]._info)
    assert blocks([64, 3]) == (2, 2) and blocks([65, 3]) == (2, 4) and short([129, 3])[0]._info.short_jobs == 0
    assert short([5, 5], n_k=[5, 129])[0]._info.short_jobs == 0 and short([5], backward=False)[0]._info.short_jobs == 0


def test_plan_refusals():
    ok = dict(n_q=[3, 4], H=2, device="cpu")
    gt.gt_attn_pack(**ok)
    for bad, what in [(dict(n_q=[]), "n_q"), (dict(n_q=[-1, 4]), "n_q"), (dict(n_q=[1.5, 2.0]), "n_q"),
                      (dict(n_k=[3]), "n_k"), (dict(n_k=[3, 1 << 31]), "n_k"), (dict(prefix=[1]), "prefix"),
                      (dict(prefix=[-1, 0]), "prefix"), (dict(H=0), "H"), (dict(H=70000), "H"),
                      (dict(spd_off=[0]), "spd_off"), (dict(spd_ld=[-3, 4]), "spd_ld")]:
        with pytest.raises(ValueError, match=what):
            gt.gt_attn_pack(**{**ok, **bad})
    for bad, code in [(dict(spd_ld=[2, 4]), 1), (dict(n_q=[1 << 25, 1]), 2), (dict(spd_ld=[1 << 25, 4]), 2),
                      (dict(spd_off=[0, (1 << 63) - 5]), 1),
                      (dict(n_q=[128 * 260, 1], H=65535), 2)]:                   # 2^24 workgroups
        with pytest.raises(gt.GTError) as e:
            gt.gt_attn_pack(**{**ok, **bad})
        assert e.value.status == code, bad


def test_plan_c_abi():
    L, info = gt.lib(), gt.packed._Info()
    n = np.array([300, 20], np.int32)
    p = n.ctypes.data
    assert L.gt_attn_pack_plan(2, 4, p, p, None, None, None, 1, None, 0, ctypes.byref(info)) == 0
    need = info.plan_bytes
    assert need > 0 and info.total_q == 320 and info.spd_bytes == 300 * 300 + 20 * 20
    buf = np.zeros(need, np.uint8)
    assert L.gt_attn_pack_plan(2, 4, p, p, None, None, None, 1, buf.ctypes.data, need - 1, ctypes.byref(info)) == 3
    assert not buf.any()
    assert L.gt_attn_pack_plan(2, 4, p, p, None, None, None, 1, buf.ctypes.data, need, ctypes.byref(info)) == 0
    for a in [(0, 4, p, p), (2, 0, p, p), (2, 4, None, p), (2, 4, p, None)]:
        assert L.gt_attn_pack_plan(*a, None, None, None, 1, None, 0, ctypes.byref(info)) == 1
    assert L.gt_attn_pack_plan(2, 4, p, p, None, None, None, 1, None, 0, None) == 1


# ---------------------------------------------------------------------------
# refusals of the two calls, at the C ABI (nothing is launched)
# ---------------------------------------------------------------------------
FAKE, MIS = 0x10000, 0x10008


def call(entry="fwd", **kw):
    a = dict(H=2, d=64, dtype=1, nb=8, scale=0.1, cap=0.0, p=None, ws=FAKE, wsb=1 << 30, plan=FAKE, spd=FAKE,
             table=FAKE, lse=FAKE, ld=40, dtable=FAKE, offset_dev=None, info=True, backward=1)
    rows = {n: (FAKE, 40 * 64, 64) for n in ("q", "k", "v", "o", "d_o", "dq", "dk", "dv")}
    for k, x in kw.items():
        (rows if k in rows else a)[k] = x
    P = gt.packed
    n = np.array([30, 10], np.int32)
    info = P._Info()
    assert gt.lib().gt_attn_pack_plan(2, a["H"], n.ctypes.data, n.ctypes.data, None, None, None, a["backward"], None, 0,
                                      ctypes.byref(info)) == 0
    b = ctypes.byref
    r = {k: None if x is None else b(P._Rows(*x)) for k, x in rows.items()}
    drop = None if a["p"] is None else b(P._Dropout(a["p"], 1, 2, a["offset_dev"]))
    ip = b(info) if a["info"] else None
    head = (ip, a["plan"], r["q"], r["k"], r["v"], a["spd"], a["table"], a["nb"], r["o"], a["lse"], a["ld"])
    tail = (a["ws"], a["wsb"], a["d"], a["dtype"], a["scale"], a["cap"], drop, None)
    if entry == "fwd":
        return gt.lib().gt_attn_pack_fwd(*head, *tail)
    return gt.lib().gt_attn_pack_bwd(*head, r["d_o"], r["dq"], r["dk"], r["dv"], a["dtable"], *tail)


BOTH = [(dict(info=False), 1), (dict(plan=None), 1), (dict(plan=MIS), 1), (dict(q=None), 1), (dict(k=None), 1),
        (dict(v=(None, 2560, 64)), 1), (dict(o=(MIS, 2560, 64)), 1), (dict(q=(FAKE, 2560, 56)), 1),
        (dict(q=(FAKE, 2560, 68)), 1), (dict(k=(FAKE, 2564, 64)), 1), (dict(k=(FAKE, -2560, 64)), 1),
        (dict(v=(FAKE, 2560, (1 << 23) + 8)), 1), (dict(spd=None), 1), (dict(table=None), 1), (dict(lse=None), 1),
        (dict(ld=39), 1), (dict(nb=0), 1), (dict(nb=257), 1), (dict(d=48), 2), (dict(d=128), 2), (dict(dtype=2), 2),
        (dict(scale=0.0), 1), (dict(scale=float("nan")), 1), (dict(scale=2.0 ** -65), 1), (dict(scale=2.0 ** 65), 1), (dict(cap=-1.0), 1), (dict(cap=float("inf")), 1),
        (dict(cap=float("nan")), 1), (dict(cap=2.0 ** -11), 1), (dict(cap=1025.0), 1), (dict(p=-0.1), 1), (dict(p=1.0), 1), (dict(p=1 - 1e-6), 1),
        (dict(p=float("nan")), 1), (dict(p=0.1, offset_dev=0x10002), 1)]


@pytest.mark.parametrize("entry", ["fwd", "bwd"])
@pytest.mark.parametrize("kw,code", BOTH)
def test_call_refusals(entry, kw, code):
    assert call(entry, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(d_o=None), 1), (dict(dq=(None, 2560, 64)), 1), (dict(dk=(MIS, 2560, 64)), 1), (dict(dv=None), 1),
    (dict(dtable=None), 1), (dict(backward=0), 1), (dict(ws=None), 3), (dict(wsb=0), 3), (dict(ws=FAKE + 16), 3)])
def test_bwd_refusals(kw, code):
    assert call("bwd", **kw) == code


# ---------------------------------------------------------------------------
# refusals of the binding: a well-formed call fails only at the device check
# ---------------------------------------------------------------------------
def z(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def args(**kw):
    pack = gt.gt_attn_pack([30, 10], 2, device="cpu")
    a = dict(q=z(2, 40, 64), k=z(2, 40, 64), v=z(2, 40, 64), spd=z(1000, dtype=torch.uint8),
             table=z(2, 8, dtype=torch.float32), pack=pack)
    return {**a, **kw}


def test_binding_reaches_the_device_check():
    for kw in (dict(), dict(q=z(2, 50, 64)), dict(q=z(40, 2, 64).transpose(0, 1)), dict(k=z(1, 40, 64).expand(2, -1, -1)),
               dict(spd=z(40, 40, dtype=torch.uint8))):
        with pytest.raises(ValueError, match="device tensors"):
            gt.gt_attn_pack_fwd(**args(**kw))
        with pytest.raises(ValueError, match="device tensors"):
            gt.gt_attn_pack_bwd(**args(**kw), o=z(2, 40, 64), lse=z(2, 40, dtype=torch.float32), d_o=z(2, 40, 64))


@pytest.mark.parametrize("kw,what", [
    (dict(q=None), "q"), (dict(q=z(2, 39, 64)), "q"), (dict(q=z(3, 40, 64)), "heads"), (dict(q=z(2, 40, 48)), "head dim"),
    (dict(q=z(2, 40, 64, dtype=torch.float16)), "q"), (dict(k=z(2, 39, 64)), "k"), (dict(k=z(2, 40, 32)), "k"),
    (dict(v=z(2, 40, 64, dtype=torch.float32)), "v"), (dict(v=z(2, 41, 64)), "one shape"),
    (dict(q=z(2, 40, 128)[..., ::2]), "q"), (dict(q=z(2, 40, 65)[..., :64]), "q"),
    (dict(k=z(1, 1, 64).expand(2, 40, 64)), "k"), (dict(v=z(2, 40, 72)[..., 4:68]), "v"),
    (dict(spd=z(999, dtype=torch.uint8)), "spd"), (dict(spd=z(2000, dtype=torch.uint8)[::2]), "spd"),
    (dict(spd=z(1000, dtype=torch.int32)), "spd"), (dict(table=z(3, 8, dtype=torch.float32)), "table"),
    (dict(table=z(2, 300, dtype=torch.float32)), "table"), (dict(table=z(8, 2, dtype=torch.float32).t()), "table"),
    (dict(pack=None), "pack")])
def test_binding_refusals(kw, what):
    with pytest.raises(ValueError, match=what):
        gt.gt_attn_pack_fwd(**args(**kw))


@pytest.mark.parametrize("drop,what", [
    (0.1, "GTDropout"), ((0.1, 3), "GTDropout"), (gt.GTDropout(1.0, 3), "dropout"), (gt.GTDropout(-0.1, 3), "dropout"),
    (gt.GTDropout(float("nan"), 3), "dropout"), (gt.GTDropout(0.1, -1), "seed"), (gt.GTDropout(0.1, 1 << 64), "seed"),
    (gt.GTDropout(0.1, 3, 1 << 32), "offset"), (gt.GTDropout(0.1, 3, -1), "offset"),
    (gt.GTDropout(0.1, 3, 0, torch.zeros(1, dtype=torch.int32)), "offset_dev")])
def test_dropout_refusals(drop, what):
    with pytest.raises(ValueError, match=what):
        gt.packed._dropout(drop, 0)
    assert gt.packed._dropout(gt.GTDropout(0.0, 3), 0) is None
