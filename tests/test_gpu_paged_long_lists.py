"""Groups that hundreds of waves share: one long request, alone and among many short ones, with one or
two key heads (so that the teams are many).  Results against the fp64 oracle with the tolerance of
tests/test_gpu_paged_attention.py; parts that hold NaN or see no key among the later ones; and the
time of the long request among short ones against its time alone."""
import numpy as np
import pytest
import torch

import paper_2310_01889_amd as ra
from oracle import serving as OS
from tests.gpu_util import log, np64
from tests.test_gpu_paged_attention import call, check, make

pytestmark = pytest.mark.gpu

CASES = [  # lens, Hq, Hkv, D: parts a wave joins: some 120; 900 of one; 450 of one; 60 of one; 70; 128
    ([40000], 8, 1, 128), ([60000] + [5] * 69, 8, 1, 128), ([60000] + [5] * 40, 4, 2, 128),
    ([21000] * 3 + [7] * 80, 6, 1, 64), ([50000] + [3] * 20, 32, 4, 64), ([30000, 9, 2] + [11] * 10, 16, 8, 128)]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_long_lists_of_parts(case, e4m3):
    lens, Hq, Hkv, D = CASES[case]
    log("paged attention of %d requests, longest %d, %d / %d heads of %d, e4m3=%d" % (len(lens), lens[0], Hq, Hkv, D, e4m3))
    s = make(100 + case, lens, [1] * len(lens), Hq, Hkv, D, 16, e4m3)
    o, lse = call(s, 1)
    check(s, o, lse)
    again = call(s, 1)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def test_entries_a_wave_each():
    """More groups than waves (an entry a wave), one of them long."""
    lens = [20000] + [6] * 1100
    s = make(110, lens, [1] * len(lens), 2, 1, 64, 16, False)
    check(s, *call(s, 1))


@pytest.mark.parametrize("short", [0, 69])
def test_later_parts_that_hold_nan_or_nothing(short):
    n, D = 50000, 128
    s = make(111, [n] + [5] * short, [1] * (1 + short), 8, 1, D, 16, False)
    s["q"][0] = s["q"][0].abs() + 0.5
    flat = s["table"][0, torch.arange(n, device="cuda") // 16].long() * 16 + torch.arange(n, device="cuda") % 16
    s["k"].view(-1, D)[flat[21000:45000]] = float("-inf")  # their scores are -inf: parts that weigh nothing
    s["ref"] = (OS.cached(np64(s["k"])), s["ref"][1])
    o, lse = call(s, 1)
    ref, lref, mag = OS.attention(np64(s["q"]), *s["ref"], s["table_np"], s["lens_np"], s["cu_np"])
    assert (np.abs(np64(o) - ref) <= 2.0 ** -8 * 1.01 * (np.abs(ref) + mag) + 4e-3 * mag).all()
    assert np.abs(np64(lse) - lref).max() <= 4e-3
    s["v"].view(-1, D)[flat[49000], 5] = float("nan")
    o2, lse2 = call(s, 1)
    assert torch.isnan(o2[0, :, 5]).all() and torch.equal(lse, lse2)
    o2[0, :, 5] = o[0, :, 5]
    assert torch.equal(o, o2)


def _us(s):
    o, lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")
    run = lambda: ra.paged_attn_decode(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"], o, lse, 1, s["ks"], s["vs"])
    best = float("inf")
    for _ in range(8):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        run()
        a.record()
        for _ in range(20):
            run()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b) * 50)
    return best


@pytest.mark.parametrize("Hkv,short", [(1, 69), (2, 40)])
def test_short_requests_beside_a_long_one_cost_little(Hkv, short):
    """The lengths of a batch do not matter for its time: a long request's, with requests of five keys
    beside it (0.1 % of the keys), is far below three times what it is alone."""
    alone, among = (_us(make(112, [60000] + [5] * n, [1] * (n + 1), 8 * Hkv, Hkv, 128, 16, False)) for n in (0, short))
    log("  alone %.1f us, among %d short ones %.1f us" % (alone, short, among))
    assert among <= 3 * alone
