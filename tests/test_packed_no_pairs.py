"""Graphs without queries or without keys in a packed batch whose distances' places
are given: nothing of them is counted in spd_bytes, so their records may lead nowhere
(CPU only: the records are looked at, nothing is run on them)."""
import numpy as np
import pytest

import paper_2609_34420_amd as gt
from test_packed_plan import WAVE, lists


def records(pack):
    """All waves of a plan's lists."""
    i, buf = pack._info, pack._plan.numpy()
    short = buf[i.short_off:][:4 * i.short_jobs * WAVE.itemsize].view(WAVE).reshape(-1, 4)
    return np.concatenate([*lists(pack)[0], short]).reshape(-1)


@pytest.mark.parametrize("n_q,n_k,off,ld", [
    ([40, 40], [0, 40], [1 << 40, 0], [1 << 20, 40]),          # shares a workgroup with a graph that has keys
    ([40], [0], [0], [1 << 20]), ([40], [0], [1 << 40], [0]),  # nothing but itself
    ([0, 40], [300, 40], [1 << 40, 0], [1 << 20, 40]),
    ([200, 0, 70], [0, 200, 70], [1 << 50, 1 << 50, 7], [1 << 24, 1 << 24, 128]),
    ([1, 1], [0, 9000], [1 << 40, 3], [1 << 20, 9000])])
@pytest.mark.parametrize("prefix", [None, 0])
def test_records_lead_nowhere(n_q, n_k, off, ld, prefix):
    pack = gt.gt_attn_pack(n_q, 4, n_k=n_k, spd_off=off, spd_ld=ld, device="cpu",
                           prefix=None if prefix is None else [prefix] * len(n_q))
    w = records(pack)
    assert len(w)
    none = (w["nq"] == 0) | (w["nk"] == 0)
    assert not w["spd"][none].any() and (w["ld"] == w["nk"])[none].all()
    # every byte that a record's rows and keys span lies within the batch's distances
    some = w[~none]
    assert (some["spd"] + (some["nq"] - 1).astype(np.int64) * some["ld"] + some["nk"] <= pack.spd_bytes).all()
