"""Row offsets that are not what a plan writes: rows before the first request's, offsets that are
negative, past T or descending.  Whatever they are, nothing outside the T rows is written, and
requests whose own offsets are in order have their rows where no other request claims them."""
import numpy as np
import pytest
import torch

import paper_2310_01889_amd as ra
from oracle import serving as OS
from tests.gpu_util import log, np64
from tests.test_gpu_paged_attention import make

pytestmark = pytest.mark.gpu
BIG = 2 ** 31 - 1


def _run(s, cu, T, max_new):
    """o and lse as T rows in the middle of larger buffers."""
    Hq, D = s["q"].shape[1:]
    ob = torch.full((T + 16, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lb = torch.full((T + 16, Hq), 7.0, device="cuda")
    o, lse = ob[8:8 + T], lb[8:8 + T]
    ra.paged_attn_decode(s["q"], s["k"], s["v"], s["table"], s["lens"], torch.tensor(cu, dtype=torch.int32, device="cuda"),
                         o, lse, max_new, s["ks"], s["vs"])
    torch.cuda.synchronize()
    for b in (ob, lb):
        assert (b[:8] == 7).all() and (b[8 + T:] == 7).all()
    return np64(o), np64(lse)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("Hq,Hkv,max_new", [(16, 2, 32), (16, 2, 1), (64, 1, 3), (4, 4, 8)])
def test_rows_before_the_first_request(Hq, Hkv, max_new, wide):
    R, T = 70, 300
    lens = [(37 * i) % 90 for i in range(R)]
    news = [min(lens[i], i % 6) for i in range(R)]
    s = make(140, lens, news, Hq, Hkv, 64, 8, False, pad=T - sum(news), extra_cols=9000 if wide else 1)
    cu = 41 + np.concatenate([[0], np.cumsum(news)])
    log("first row 41 of %d, %d / %d heads, max_new=%d, wide=%d" % (T, Hq, Hkv, max_new, wide))
    o, lse = _run(s, cu, T, max_new)
    ref, lref, mag = OS.attention(np64(s["q"]), *s["ref"], s["table_np"], s["lens_np"], cu, max_new)
    none = np.isnan(lref)
    assert (o[none] == 7).all() and (lse[none] == 7).all() and none[:41].all()
    empty = np.isneginf(lref)
    assert (o[empty] == 0).all() and np.isneginf(lse[empty]).all()
    fine = ~none & ~empty
    assert (np.abs(o - ref) <= 2.0 ** -8 * 1.01 * (np.abs(ref) + mag) + 1e-4 * mag)[fine].all()
    assert (np.abs(lse - lref) <= 1e-4)[fine].all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("Hq,Hkv,max_new", [(16, 2, 32), (64, 1, 2), (4, 4, 1)])
def test_offsets_out_of_order(Hq, Hkv, max_new, wide):
    T = 24
    lens = [30, 9, 50, 17, 40, 6]
    s = make(141, lens, [4] * 6, Hq, Hkv, 64, 8, False, extra_cols=9000 if wide else 1)
    for cu in ([-5, 3, 2, 900, BIG, 4, 7], [BIG] * 7, [-BIG] * 7, [24, 20, 16, 12, 8, 4, 0], [0, 24, 0, 24, 0, 24, 0],
               [0, 4, BIG, -1, 8, BIG, 0]):
        log("offsets %s" % cu)
        _run(s, cu, T, max_new)
