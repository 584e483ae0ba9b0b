"""Packed attention at the edges of what its documentation allows."""
import pytest
import torch

import paper_2609_34420_amd as gt
from gpu_common import DEV, say
from test_gpu_packed import DROP, make, upload

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n", [40, 150])                       # the one-pass and the two-pass backward
@pytest.mark.parametrize("prefix", [None, 0])
def test_places_of_graphs_without_pairs(dt, n, prefix):
    """Places and strides given for graphs without queries or without keys change
    nothing (no distance is read for them)."""
    n_q, n_k, H = [n, n, 0, 33, 7], [0, n, n, 33, 0], 2
    a = make(n_q, n_k, H, 32, 12, dt, seed=41)
    r = upload(a)
    kw = dict(n_k=n_k, device=DEV, prefix=None if prefix is None else [prefix] * 5)
    far, wide = 1 << 40, 1 << 24
    plans = [gt.gt_attn_pack(n_q, H, **kw),
             gt.gt_attn_pack(n_q, H, spd_off=[far, 0, far, n * n, far], spd_ld=[wide, n, wide, 33, wide], **kw)]
    say(f"no pairs {dt} n={n} prefix={prefix}")
    got = []
    for pack in plans:
        assert pack.spd_bytes == r["spd"].numel()
        args = (r["q"], r["k"], r["v"], r["spd"], r["table"], pack)
        o, lse = gt.gt_attn_pack_fwd(*args, cap=9.0, dropout=DROP)
        got.append((o, lse, *gt.gt_attn_pack_bwd(*args, o, lse, r["do"], cap=9.0, dropout=DROP)))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(*got))
