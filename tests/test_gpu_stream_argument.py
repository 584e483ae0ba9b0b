"""Calls with stream=: memory that a call allocates has nothing pending on it, and is
not handed out again before the caller's stream has passed the results."""
import pytest
import torch

import paper_2609_34420_amd as gt
from gpu_common import DEV
from test_gpu_packed import DROP, make, upload

pytestmark = pytest.mark.gpu


def packed(seed):
    n, H = [300, 45], 2
    r = upload(make(n, n, H, 32, 22, "bf16", seed=seed))
    pack = gt.gt_attn_pack(n, H, device=DEV)
    args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
    o, lse = gt.gt_attn_pack_fwd(*args, dropout=DROP)
    return {"pack_fwd": lambda s: gt.gt_attn_pack_fwd(*args, dropout=DROP, stream=s),
            "pack_bwd": lambda s: gt.gt_attn_pack_bwd(*args, o, lse, r["do"], dropout=DROP, stream=s)}


def new_nodes(seed):
    r = upload(make([1, 2], [6000, 2345], 2, 16, 22, "bf16", seed=seed))
    pack = gt.gt_attn_pack([1, 2], 2, n_k=[6000, 2345], device=DEV)
    assert gt.gt_attn_pack_fwd_workspace_size(pack, 16)
    return {"pack_parts": lambda s: gt.gt_attn_pack_fwd(r["q"], r["k"], r["v"], r["spd"], r["table"], pack, stream=s)}


def unpacked(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, H, N, d = 3, 2, 320, 32
    q, k, v, do = (torch.randn(B, H, N, d, device=DEV, generator=g).bfloat16() for _ in range(4))
    spd = torch.randint(0, 22, (N, N), device=DEV, generator=g, dtype=torch.uint8)
    t = torch.randn(H, 22, device=DEV, generator=g)
    one, parts = (q[0], k[0], v[0], spd, t), torch.randn(4, H, N, d, device=DEV, generator=g)
    lses = torch.randn(4, H, N, device=DEV, generator=g)
    f, fb = gt.gt_attn_fwd(*one), gt.gt_attn_fwd_batch(q, k, v, spd, t)
    return {"fwd": lambda s: gt.gt_attn_fwd(*one, stream=s),
            "bwd": lambda s: gt.gt_attn_bwd(*one, *f, do[0], stream=s),
            "fwd_batch": lambda s: gt.gt_attn_fwd_batch(q, k, v, spd, t, stream=s),
            "bwd_batch": lambda s: gt.gt_attn_bwd_batch(q, k, v, spd, t, *fb, do, stream=s),
            "ring_step": lambda s: gt.gt_attn_ring_step(q[0], k[0], v[0], spd, 0, 0, t, stream=s),
            "bwd_ring_step": lambda s: gt.gt_attn_bwd_ring_step(q[0], *f, do[0], k[0], v[0], spd, 0, 0, t, stream=s),
            "merge": lambda s: gt.gt_attn_merge(parts, lses, stream=s)}


CALLS = {"pack_fwd": packed, "pack_bwd": packed, "pack_parts": new_nodes,
         **{n: unpacked for n in ("fwd", "bwd", "fwd_batch", "bwd_batch", "ring_step", "bwd_ring_step", "merge")}}


def same(name, got, want):
    """Bit by bit; the unpacked backward's fp32 sums over workgroups are atomics, whose order
    varies: some 30 additions, each off by half a step of 2^-24 of partial sums up to five
    times the result, 1e-5 of it."""
    loose = name.startswith("bwd")
    return all(torch.equal(x, y) or (loose and y.dtype == torch.float32
                                     and float((x - y).double().norm()) <= 1e-5 * float(y.double().norm()))
               for x, y in zip(got, want))


def fill_pending(tensors):
    """Blocks of the tensors' sizes (and of workspaces') freed on the current stream with a
    write to them still to come."""
    torch.cuda._sleep(50_000_000)
    sizes = [t.numel() * t.element_size() for t in tensors] + [1 << k for k in range(9, 24)]
    blocks = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(3)]
    for b in blocks:
        b.fill_(0x7f)


@pytest.mark.parametrize("name", CALLS)
def test_memory_has_nothing_pending(name):
    call = CALLS[name](51)[name]
    want = call(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    fill_pending(want)
    got = call(side)
    side.synchronize()
    assert same(name, [x.cpu() for x in got], [y.cpu() for y in want])
    torch.cuda.synchronize()
    assert same(name, got, want)


@pytest.mark.parametrize("name", CALLS)
def test_results_outlive_the_callers_use(name):
    """Results read on the current stream and dropped while that read is pending; calls
    on the side stream go on."""
    call, other = (CALLS[name](seed)[name] for seed in (52, 53))
    want = call(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(50_000_000)
    copies = [x.clone() for x in got]
    del got
    for _ in range(3):
        other(side)
    torch.cuda.synchronize()
    assert same(name, copies, want)


@pytest.mark.parametrize("name", CALLS)
def test_captured_on_a_forked_stream(name):
    call = CALLS[name](54)[name]
    side = torch.cuda.Stream()
    want = call(None)
    call(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = call(side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert same(name, got, want)
        call(None)
        torch.cuda.synchronize()
