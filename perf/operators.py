"""Packed attention and attention dropout as a user calls them, as timed cases.

Two operators, one pair of entry points:

  * cap: attention over a packed batch of graphs of unlike sizes (a pair of
    nodes of two graphs is masked), scores capped by a tanh before the
    shortest-path bias is added, optionally with a prefix mask; training steps,
    evaluation, and a few new nodes against all the keys of their graphs;
  * drop: the same attention with dropout of the probabilities, drawn from a
    counter-based generator and never stored.

`listed()` names the fixed cases, `draw(rng)` gives more of the same ranges,
`prepare` builds what the program holds before the call, `run` makes the calls
(or their plain form in elementary torch operations, where `own` is false) and
`exact` is the same result in 64 bits.

Graph g has nq query rows and nk keys (nq = nk but for new nodes), its rows
packed one graph behind the other; query i stands at position i + nk - nq.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
_CHUNK = 1 << 28            # score elements the plain form holds at a time


def listed():
    return [
        # evaluation of one small graph: latency of one launch
        dict(name="cap_eval_small", op="cap", kind="eval", dtype="bf16", G=1, lo=200, hi=200, H=8, d=8, nb=22,
             mask="full", cap=20.0, p=0.0),
        # one new node each in 16 graphs of some thousand nodes: reading K and V
        dict(name="cap_new_nodes", op="cap", kind="new", dtype="bf16", G=16, lo=1000, hi=16000, new=1, H=8, d=64,
             nb=64, mask="full", cap=30.0, p=0.0),
        # a training batch of molecule-sized graphs: 8 heads over a 64-wide model
        dict(name="cap_step_small_graphs", op="cap", kind="step", dtype="bf16", G=1024, lo=9, hi=60, H=8, d=8,
             nb=22, mask="full", cap=20.0, p=0.0),
        # a training batch of sampled subgraphs of a few hundred to two thousand nodes
        dict(name="cap_step_ragged", op="cap", kind="step", dtype="bf16", G=48, lo=200, hi=2000, H=8, d=64, nb=64,
             mask="full", cap=30.0, p=0.0),
        # generation in node order: each node sees a prefix and the nodes before it
        dict(name="cap_step_prefix", op="cap", kind="step", dtype="bf16", G=16, lo=500, hi=3000, H=8, d=32, nb=40,
             mask="prefix", cap=30.0, p=0.0),
        # fp32 training on a few mid-sized graphs
        dict(name="cap_step_f32", op="cap", kind="step", dtype="f32", G=6, lo=300, hi=1200, H=4, d=32, nb=22,
             mask="full", cap=20.0, p=0.0),
        # the 16384-node benchmark workload with capped scores, and the largest case
        dict(name="cap_step_16k", op="cap", kind="step", dtype="bf16", G=1, lo=16384, hi=16384, H=8, d=64, nb=32,
             mask="full", cap=50.0, p=0.0),
        # the fp32 benchmark workload (512 nodes) with dropout
        dict(name="drop_step_512_f32", op="drop", kind="step", dtype="f32", G=1, lo=512, hi=512, H=4, d=32, nb=22,
             mask="full", cap=0.0, p=0.1),
        # a training batch of sampled sequences of up to 256 nodes: 8 heads over a 64-wide model
        dict(name="drop_step_sequences", op="drop", kind="step", dtype="bf16", G=512, lo=100, hi=256, H=8, d=8,
             nb=64, mask="full", cap=0.0, p=0.1),
        # training on one mid-sized graph with an odd node count, 8 heads over a 512-wide model
        dict(name="drop_step_7651", op="drop", kind="step", dtype="bf16", G=1, lo=7651, hi=7651, H=8, d=64, nb=64,
             mask="full", cap=0.0, p=0.1),
        # everything at once: a ragged batch, prefix mask, capped scores and dropout
        dict(name="drop_step_prefix_cap", op="drop", kind="step", dtype="bf16", G=64, lo=50, hi=1000, H=8, d=16,
             nb=40, mask="prefix", cap=30.0, p=0.2),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: graph sizes spread over the logarithm of their range, the
    number of graphs so that the batch has 2^19 to 2^27 pairs (2^24 in fp32)."""
    op = rng.choice(["cap", "drop"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    kind = rng.choice(["step", "step", "step", "eval", "new"])
    c = dict(op=op, kind=kind, dtype=dtype, H=rng.choice([4, 8, 8, 16]), d=rng.choice([8, 16, 32, 64, 64]))
    c["nb"] = rng.choice([22, 32, 40, 64, rng.randint(8, 127), 256])
    c["mask"] = rng.choice(["full", "full", "prefix", "causal"])
    c["cap"] = rng.choice([15.0, 30.0, 50.0]) if op == "cap" or rng.random() < 0.3 else 0.0
    c["p"] = rng.choice([0.05, 0.1, 0.2, 0.5]) if op == "drop" else 0.0
    if kind == "new":
        c["new"] = rng.choice([1, 1, 2, 7, 33])
        lo = _log_uniform(rng, 100, 6000)
        c["G"] = _log_uniform(rng, 1, 64)
        hi = _log_uniform(rng, lo, 12000)
    else:
        top = 4000 if dtype == "f32" else 11000
        lo = _log_uniform(rng, 5, top)
        hi = min(top, _log_uniform(rng, lo, 6 * lo))
        pairs = _log_uniform(rng, 1 << 19, 1 << (24 if dtype == "f32" else 27))
        c["G"] = max(1, min(2048, 16 * pairs // (c["H"] * (lo + hi) ** 2)))
    c["lo"], c["hi"] = lo, hi
    return c


# ---------------------------------------------------------------------------
# sizes and inputs
# ---------------------------------------------------------------------------
def _sizes(case):
    """(query rows, keys, prefix or None) of each graph, from the case alone."""
    rng = random.Random(f"{case['G']} {case['lo']} {case['hi']} {case['d']}")
    nk = [_log_uniform(rng, case["lo"], case["hi"]) for _ in range(case["G"])]
    nq = [min(n, case["new"]) for n in nk] if case["kind"] == "new" else list(nk)
    prefix = None
    if case["mask"] == "causal":
        prefix = [0] * case["G"]
    elif case["mask"] == "prefix":
        prefix = [rng.randint(0, n // 2) for n in nk]
    return nq, nk, prefix


def _visible_pairs(case):
    nq, nk, prefix = _sizes(case)
    total = 0
    for g, (a, b) in enumerate(zip(nq, nk)):
        if prefix is None:
            total += a * b
        else:
            f = prefix[g]                       # row at position t sees max(f, t + 1) keys
            total += sum(max(f, t + 1) for t in range(b - a, b))
    return total


def _cum(sizes):
    out = [0]
    for n in sizes:
        out.append(out[-1] + n)
    return out


def _spd(gen, nb, nq, nk):
    """The graphs' [nq, nk] matrices one behind the other, uint8, with the
    shape of shortest-path distances on a clustered graph: a distance between
    the two nodes' clusters plus each node's own depth, clipped, about a quarter
    of the cluster pairs unreachable (bucket nb - 1), 0 on the diagonal."""
    nc = 64 if max(nk) >= 4096 else 8
    top = max(1, min(nb - 2, 12))
    dist = torch.randint(1, top + 1, (nc, nc), device=DEV, generator=gen, dtype=torch.int16)
    dist[torch.rand((nc, nc), device=DEV, generator=gen) < 0.25] = 1000
    dist = torch.minimum(dist, dist.t()).contiguous()
    dist.fill_diagonal_(1)
    out, g = [], 0
    while g < len(nq):
        e = g + 1
        while e < len(nq) and (e + 1 - g) * max(nq[g:e + 1]) * max(nk[g:e + 1]) <= 1 << 26:
            e += 1
        a, b, n = max(nq[g:e]), max(nk[g:e]), e - g
        tq, tk = torch.tensor(nq[g:e], device=DEV), torch.tensor(nk[g:e], device=DEV)
        cl = torch.randint(0, nc, (n, b), device=DEV, generator=gen)
        dep = torch.randint(0, 4, (n, b), device=DEV, generator=gen, dtype=torch.int16)
        i, j = torch.arange(a, device=DEV), torch.arange(b, device=DEV)
        pos = (i[None] + (tk - tq)[:, None]).clamp_(max=b - 1)          # [n, a]
        x = dist.view(-1)[torch.gather(cl, 1, pos)[:, :, None] * nc + cl[:, None, :]]
        x += torch.gather(dep, 1, pos)[:, :, None]
        x += dep[:, None, :]
        x = torch.where(x >= 900, nb - 1, x.clamp_(max=max(nb - 2, 0))).to(torch.uint8)
        x[pos[:, :, None] == j] = 0
        real = (i[None, :, None] < tq[:, None, None]) & (j[None, None] < tk[:, None, None])
        out.append(x[real])
        g = e
    return torch.cat(out)


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    td = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    H, d, nb = case["H"], case["d"], case["nb"]
    nq, nk, prefix = _sizes(case)

    # products that reach a good part of the cap, as late in training
    gain = 2.0 if case["cap"] else 1.0
    s = {"case": case, "nq": nq, "nk": nk, "prefix": prefix}
    s["q"] = (gain * torch.randn((H, sum(nq), d), device=DEV, generator=gen)).to(td)
    s["k"] = (gain * torch.randn((H, sum(nk), d), device=DEV, generator=gen)).to(td)
    s["v"] = torch.randn((H, sum(nk), d), device=DEV, generator=gen).to(td)
    if case["kind"] == "step":
        s["do"] = torch.randn((H, sum(nq), d), device=DEV, generator=gen).to(td)
    s["table"] = 0.3 * torch.randn((H, nb), device=DEV, generator=gen)
    s["spd"] = _spd(gen, nb, nq, nk)
    s["rng"] = (random.Random(seed).getrandbits(64), seed % 1000)       # dropout seed, offset
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2609_34420_amd as gt

        s["pack"] = gt.gt_attn_pack(s["nq"], case["H"], n_k=s["nk"], prefix=s["prefix"], device=DEV)
        s["drop"] = gt.GTDropout(case["p"], *s["rng"]) if case["p"] else None
    else:
        s["chunks"] = _chunks(s)
    return s


def run(s):
    if not own:
        return _plain(s)
    import paper_2609_34420_amd as gt

    c = s["case"]
    a = (s["q"], s["k"], s["v"], s["spd"], s["table"], s["pack"])
    kw = dict(cap=c["cap"] or None, dropout=s["drop"])
    o, lse = gt.gt_attn_pack_fwd(*a, **kw)
    if c["kind"] != "step":
        return o, lse
    return (o, lse, *gt.gt_attn_pack_bwd(*a, o, lse, s["do"], **kw))


def work(case):
    """Every input once and every output once (of spd the visible pairs); 4 d
    operations per visible pair and head forward, 10 d backward (the score
    again, and four products)."""
    nq, nk, _ = _sizes(case)
    H, d = case["H"], case["d"]
    es = 2 if case["dtype"] == "bf16" else 4
    pairs, tq, tk = _visible_pairs(case), sum(nq), sum(nk)
    step = case["kind"] == "step"
    byts = pairs + 4 * H * case["nb"] + H * d * es * 2 * (tq + tk) + 4 * H * tq
    if step:
        byts += H * d * es * 2 * (tq + tk) + 4 * H * case["nb"]          # dO, dQ; dK, dV; dtable
    return {"bytes": byts, "flops": (14 if step else 4) * H * d * pairs}


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _chunks(s):
    """Graphs padded to one size, as many at a time as _CHUNK allows, and the
    heads at a time: index tensors of the rows they gather and scatter."""
    nq, nk, H = s["nq"], s["nk"], s["case"]["H"]
    cq, ck, cs = _cum(nq), _cum(nk), _cum([a * b for a, b in zip(nq, nk)])
    order = sorted(range(len(nq)), key=lambda g: nk[g])
    out, x = [], 0
    while x < len(order):
        y = x + 1
        while y < len(order) and (y + 1 - x) * nk[order[y]] * max(nq[g] for g in order[x:y + 1]) * H <= _CHUNK:
            y += 1
        gs = order[x:y]
        a, b = max(nq[g] for g in gs), max(nk[g] for g in gs)
        t = {n: torch.tensor([v[g] for g in gs], device=DEV)
             for n, v in (("nq", nq), ("nk", nk), ("cq", cq), ("ck", ck), ("cs", cs))}
        i, j = torch.arange(a, device=DEV), torch.arange(b, device=DEV)
        c = {"heads": max(1, min(H, _CHUNK // (len(gs) * a * b)))}
        c["iok"] = i[None] < t["nq"][:, None]
        c["jok"] = j[None] < t["nk"][:, None]
        c["qrow"] = torch.where(c["iok"], t["cq"][:, None] + i, 0)
        c["krow"] = torch.where(c["jok"], t["ck"][:, None] + j, 0)
        c["spd0"], c["nk"], c["off"] = t["cs"], t["nk"], t["nk"] - t["nq"]
        if s["prefix"] is not None:
            c["prefix"] = torch.tensor([s["prefix"][g] for g in gs], device=DEV)
        out.append(c)
        x = y
    return out


def _philox7(c0, c1, c2, c3, seed):
    """Philox4x32 with 7 rounds on int64 tensors that hold 32-bit words."""
    M = 0xffffffff
    k0, k1 = seed & M, seed >> 32
    for _ in range(7):
        x, y = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((y >> 32) & M) ^ c1 ^ k0, y & M, ((x >> 32) & M) ^ c3 ^ k1, x & M
        k0, k1 = (k0 + 0x9E3779B9) & M, (k1 + 0xBB67AE85) & M
    return c0, c1, c2, c3


def _plain_keep(rows, heads, b, p, rng):
    """Kept pairs [len(heads), *rows.shape, b]: 16 bits per pair, 8 keys of a
    row from one draw, kept unless below the threshold as signed integers."""
    seed, offset = rng
    j8 = torch.arange((b + 7) // 8, device=DEV)
    shape = (len(heads), *rows.shape, len(j8))
    h = torch.tensor(heads, device=DEV).view(-1, *[1] * (rows.dim() + 1))
    w = _philox7(j8.expand(shape), rows[None, ..., None].expand(shape), h.expand(shape),
                 torch.full((), offset, device=DEV).expand(shape), seed)
    r = torch.stack([x for v in w for x in (v & 0xffff, v >> 16)], -1).flatten(-2)[..., :b]
    r = torch.where(r >= 32768, r - 65536, r)
    return r >= round(p * 65536) - 32768


def _plain(s):
    c = s["case"]
    H, d, nb, cap, p = c["H"], c["d"], c["nb"], c["cap"], c["p"]
    td = s["q"].dtype
    scale, rp = 1.0 / math.sqrt(d), 65536.0 / (65536 - round(p * 65536))
    step = c["kind"] == "step"
    o, lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device=DEV)
    if step:
        dq, dk, dv = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
        dtab = torch.zeros((H, 256), device=DEV)
    table = torch.nn.functional.pad(s["table"], (0, 256 - nb))
    for ch in s["chunks"]:
        iok, jok, qrow, krow = ch["iok"], ch["jok"], ch["qrow"], ch["krow"]
        a, b = iok.shape[1], jok.shape[1]
        i, j = torch.arange(a, device=DEV), torch.arange(b, device=DEV)
        seen = iok[:, :, None] & jok[:, None, :]
        at = torch.where(seen, ch["spd0"][:, None, None] + i[None, :, None] * ch["nk"][:, None, None] + j, 0)
        bucket = s["spd"][at].long()
        if "prefix" in ch:
            pos = i[None] + ch["off"][:, None]
            seen = seen & ((j < ch["prefix"][:, None, None]) | (j <= pos[:, :, None]))
        for h0 in range(0, H, ch["heads"]):
            hs = list(range(h0, min(H, h0 + ch["heads"])))
            sl = slice(h0, hs[-1] + 1)
            q, k, v = s["q"][sl, qrow].float(), s["k"][sl, krow].float(), s["v"][sl, krow].float()
            x = torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale
            if cap:
                t = torch.tanh(x / cap)
                x = cap * t
            x = x + table[sl][:, bucket]
            x = torch.where(seen, x, -math.inf)
            m = x.amax(-1, keepdim=True)
            m = torch.where(m == -math.inf, 0.0, m)
            x = torch.exp(x - m)
            l = x.sum(-1, keepdim=True)
            lse[sl, qrow[iok]] = (m + torch.log(l))[..., 0][:, iok]
            x = x / torch.where(l == 0, 1.0, l)
            z = None
            pz = x
            if p:
                z = _plain_keep(qrow, hs, b, p, s["rng"]) * rp
                pz = x * z
            of = torch.matmul(pz, v)
            o[sl, qrow[iok]] = of[:, iok].to(td)
            if not step:
                continue
            do = torch.where(iok[..., None], s["do"][sl, qrow].float(), 0.0)
            dv[sl, krow[jok]] = torch.matmul(pz.transpose(-1, -2).contiguous(), do)[:, jok].to(td)
            g = torch.matmul(do, v.transpose(-1, -2).contiguous())
            if p:
                g = g * z
            g = x * (g - (do * of).sum(-1, keepdim=True))
            bins = torch.zeros((*g.shape[:3], 256), device=DEV)
            dtab[sl] += bins.scatter_add_(3, bucket.expand(g.shape), g).sum((1, 2))
            if cap:
                g = g * (1.0 - t * t)
            dq[sl, qrow[iok]] = (torch.matmul(g, k) * scale)[:, iok].to(td)
            dk[sl, krow[jok]] = (torch.matmul(g.transpose(-1, -2).contiguous(), q) * scale)[:, jok].to(td)
    if not step:
        return o, lse
    return o, lse, dq, dk, dv, dtab[:, :nb].contiguous()


# ---------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------
def _mul32(x, m):
    """High and low 32 bits of x m by 16-bit halves."""
    lo = x * (m & 0xffff)
    hi = x * (m >> 16) + (lo >> 16)
    return hi >> 16, ((hi & 0xffff) << 16) | (lo & 0xffff)


def _exact_keep(h, r0, n, nk, p, rng):
    """Kept pairs of the packed rows r0 .. r0 + n - 1 of head h."""
    seed, offset = rng
    blocks = -(-nk // 8)
    ctr = torch.empty((4, n, blocks), dtype=torch.int64, device=DEV)
    ctr[0] = torch.arange(blocks, device=DEV)
    ctr[1] = torch.arange(r0, r0 + n, device=DEV)[:, None]
    ctr[2], ctr[3] = h, offset
    for rnd in range(7):
        ka = (seed + rnd * 0x9E3779B9) % 2 ** 32
        kb = ((seed >> 32) + rnd * 0xBB67AE85) % 2 ** 32
        ha, la = _mul32(ctr[0], 0xD2511F53)
        hb, lb = _mul32(ctr[2], 0xCD9E8D57)
        ctr = torch.stack([hb ^ ctr[1] ^ ka, lb, ha ^ ctr[3] ^ kb, la])
    bits = torch.empty((n, blocks, 8), dtype=torch.int64, device=DEV)
    for e in range(8):
        bits[:, :, e] = (ctr[e // 2] >> (16 * (e % 2))) % 65536
    # a signed comparison of 16-bit words is an unsigned one of the words with the top bit turned
    return (bits.view(n, -1)[:, :nk] ^ 0x8000) >= round(p * 65536)


def exact(case, seed):
    nq, nk, prefix = _sizes(case)
    if case["H"] * sum(a * b for a, b in zip(nq, nk)) > 3e9 or (case["p"] and case["G"] * case["H"] > 12000):
        return None                                       # would take too long
    s = _inputs(case, seed)
    f = torch.float64
    H, d, nb, cap, p = case["H"], case["d"], case["nb"], case["cap"], case["p"]
    sc = d ** -0.5
    keep = 1.0 - round(p * 65536) / 65536
    step = case["kind"] == "step"
    q, k, v = s["q"].to(f), s["k"].to(f), s["v"].to(f)
    tab = torch.zeros((H, 256), dtype=f, device=DEV)
    tab[:, :nb] = s["table"]
    o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=f, device=DEV)
    if step:
        do, dq, dk, dv = s["do"].to(f), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        dtab = torch.zeros((H, 256), dtype=f, device=DEV)
    q0 = k0 = s0 = 0
    for g, (a, b) in enumerate(zip(nq, nk)):
        # all heads of a small graph at once; a large one by head and row block
        hn = H if H * a * b <= 1 << 24 else 1
        rn = a if hn > 1 else max(1, (1 << 26) // b)
        for r in range(0, a, rn):
            n = min(rn, a - r)
            bucket = s["spd"][s0 + r * b:s0 + (r + n) * b].long()
            hide = None
            if prefix is not None:
                j = torch.arange(b, device=DEV)
                pos = torch.arange(r, r + n, device=DEV) + (b - a)
                hide = (j[None] > pos[:, None]) & (j[None] >= prefix[g])
            qr = slice(q0 + r, q0 + r + n)
            kr = slice(k0, k0 + b)
            for h in range(0, H, hn):
                hs = slice(h, h + hn)
                kt = k[hs, kr].transpose(1, 2).contiguous()
                u = torch.bmm(q[hs, qr], kt).mul_(sc)
                slope = None
                if cap:
                    u = u.div_(cap).tanh_()
                    slope = 1.0 - u * u if step else None
                    u = u.mul_(cap)
                u += tab[hs][:, bucket].view(hn, n, b)
                if hide is not None:
                    u.masked_fill_(hide, -math.inf)
                lg = torch.logsumexp(u, 2)
                lse[hs, qr] = lg
                pr = torch.exp_(u.sub_(torch.where(lg == -math.inf, 0.0, lg)[..., None]))
                z = None
                if p:
                    z = torch.stack([_exact_keep(x, q0 + r, n, b, p, s["rng"]) for x in range(h, h + hn)]).to(f) / keep
                pz = pr * z if p else pr
                o[hs, qr] = torch.bmm(pz, v[hs, kr])
                if not step:
                    continue
                dg = do[hs, qr]
                dv[hs, kr] += torch.bmm(pz.transpose(1, 2).contiguous(), dg)
                ds = torch.bmm(dg, v[hs, kr].transpose(1, 2).contiguous())
                if p:
                    ds *= z
                ds -= (dg * o[hs, qr]).sum(2, keepdim=True)
                ds *= pr
                bins = torch.zeros((hn * n, 256), dtype=f, device=DEV)
                bins.scatter_add_(1, bucket.view(n, b).repeat(hn, 1), ds.view(hn * n, b))
                dtab[hs] += bins.view(hn, n, 256).sum(1)
                if cap:
                    ds *= slope
                dq[hs, qr] = torch.bmm(ds, k[hs, kr]) * sc
                dk[hs, kr] += torch.bmm(ds.transpose(1, 2).contiguous(), q[hs, qr]) * sc
        q0, k0, s0 = q0 + a, k0 + b, s0 + a * b
    if not step:
        return o, lse
    return o, lse, dq, dk, dv, dtab[:, :nb]
