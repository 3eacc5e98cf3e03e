"""max_new only bounds the new tokens of a request: calls whose rows are the same give the same bits
whatever bound they name, as the launch goes by the rows that there are (a launch of another kind adds
in another order)."""
import pytest
import torch

from tests.gpu_util import log
from tests.test_gpu_paged_attention import call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("R,Hq,Hkv,D,keys,page", [
    (16, 64, 8, 128, 1000, 16), (16, 64, 8, 128, 250, 16), (32, 64, 8, 128, 700, 16), (64, 32, 8, 64, 700, 32),
    (4, 64, 8, 128, 600, 8)])
def test_a_larger_bound_changes_nothing(R, Hq, Hkv, D, keys, page, e4m3):
    log("R=%d %d / %d heads of %d, %d keys, e4m3=%d" % (R, Hq, Hkv, D, keys, e4m3))
    s = make(120, [max(1, keys - keys * 3 * i // (4 * R)) for i in range(R)], [1] * R, Hq, Hkv, D, page, e4m3)
    o, lse = call(s, 1)
    check(s, o, lse)
    for max_new in (4, 32):
        o2, lse2 = call(s, max_new)
        assert torch.equal(o, o2) and torch.equal(lse, lse2), max_new


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("R,Hq,Hkv,D,keys,most", [
    (130, 16, 2, 128, 60, 20), (200, 64, 1, 64, 500, 3), (70, 8, 1, 128, 700, 32), (300, 8, 1, 64, 90, 1),
    (5, 1024, 1, 64, 30, 2)])
def test_rounds_of_many_requests(R, Hq, Hkv, D, keys, most, wide):
    """Requests of no row to many rounds of slots, more of them than a wave's lanes, fewer rows than
    requests, heads of one token that take several rounds."""
    log("R=%d %d / %d heads of %d, %d keys, %d new tokens at most, wide=%d" % (R, Hq, Hkv, D, keys, most, wide))
    lens = [(keys * (7 * i % R)) // R for i in range(R)]
    news = [min(lens[i], (5 * i % 11) * most // 8 if most > 1 else i % 3 == 0, most) for i in range(R)]
    s = make(130 + R, lens, news, Hq, Hkv, D, 16, False, pad=3, extra_cols=4000 if wide else 1)
    check(s, *call(s, 32))
