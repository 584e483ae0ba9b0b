"""Copies of a plan are plans of their own (CPU only)."""
import copy
import ctypes
import pickle

import pytest
import torch

import paper_2609_34420_amd as gt


@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x))])
def test_a_copy_holds_its_own_addresses(how):
    a = gt.gt_attn_pack([30, 700, 0], 4, n_k=[30, 700, 5], prefix=[0, 3, 9], device="cpu")
    b = how(a)
    assert b._at == ctypes.addressof(b._info) and b._plan_at == b._plan.data_ptr()
    assert b._at != a._at or b._info is a._info
    assert bytes(b._info) == bytes(a._info) and torch.equal(a._plan, b._plan)
    for n in ("total_q", "total_k", "spd_bytes", "H", "n_graphs", "backward", "device"):
        assert getattr(a, n) == getattr(b, n)
    want = gt.gt_attn_pack_bwd_workspace_size(a, 20)
    del a
    assert gt.gt_attn_pack_bwd_workspace_size(b, 20) == want > 0
