"""paged_attn_decode against the fp64 oracle: lengths from nothing to thousands, grouped heads,
pages of every size, both cache types, masked places that hold anything, padding rows.

Tolerances.  Products are exact, sums float32.  Probabilities may be rounded to bf16 once: half a
step, 2^-8 of each, so of the weighted mean of |v|; the output's own rounding is 2^-8 of it.  A
score of D terms, each rounded, is off by at most D 2^-24 of the sum of their sizes, the sum of n
probabilities and its logarithm by n 2^-24 and a few units: that bounds lse, and moves o by as
much of the mean of |v|, twice."""
import math

import numpy as np
import pytest
import torch

import paper_2310_01889_amd as ra
from oracle import serving as OS
from tests.gpu_util import log, np64

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def make(seed, lens, news, Hq, Hkv, D, page, e4m3, pad=0, extra_cols=1):
    """Inputs on the GPU and the oracle's cache; places no request owns hold NaN and infinities."""
    g, rng = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
    R = len(lens)
    held = [-(-max(n, 0) // page) for n in lens]
    n_pages, cols = sum(held) + 2, max(held) + extra_cols
    shape = (n_pages, page, Hkv, D)
    ids = rng.permutation(n_pages)
    table = np.full((R, cols), -1)
    owned = np.zeros((n_pages, page), bool)
    at = 0
    for r in range(R):
        table[r, :held[r]] = ids[at:at + held[r]]
        for p in range(lens[r]):
            owned[table[r, p // page], p % page] = True
        at += held[r]
    k, v = (torch.randn(shape, generator=g) for _ in range(2))
    if e4m3:
        k, v = ((x * 100).clamp(-448, 448).to(E4M3) for x in (k, v))
        ks, vs = (torch.randint(118, 123, shape[:3], generator=g, dtype=torch.uint8) for _ in range(2))
        hole = torch.tensor(~owned)
        for x in (k, v):
            x.view(torch.uint8)[hole] = 0x7f
        ks[hole] = 254
    else:
        k, v, ks, vs = k.to(torch.bfloat16), v.to(torch.bfloat16), None, None
        hole = torch.tensor(~owned)
        k[hole], v[hole] = float("nan"), float("inf")
    cu = np.concatenate([[0], np.cumsum(news)])
    T = int(cu[-1]) + pad
    q = torch.randn(T, Hq, D, generator=g).to(torch.bfloat16)
    ref = (OS.cached(np64(k), None if ks is None else ks.numpy()), OS.cached(np64(v), None if vs is None else vs.numpy()))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    up = lambda x: None if x is None else x.cuda()
    return dict(q=up(q), k=up(k), v=up(v), ks=up(ks), vs=up(vs), table=i32(table), lens=i32(lens), cu=i32(cu), cu_np=cu,
                table_np=table, lens_np=np.array(lens), ref=ref, T=T)


def call(s, max_new, cu=True, workspace=None):
    o = torch.full_like(s["q"], 7.0)
    lse = torch.full(s["q"].shape[:2], 7.0, device="cuda")
    ra.paged_attn_decode(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"] if cu else None, o, lse, max_new,
                         s["ks"], s["vs"], workspace=workspace)
    torch.cuda.synchronize()
    return o, lse


def check(s, o, lse, max_new=32):
    q = np64(s["q"])
    o_ref, lse_ref, mag = OS.attention(q, *s["ref"], s["table_np"], s["lens_np"], s["cu_np"], max_new)
    none = np.isnan(lse_ref)
    go, gl = np64(o), np64(lse)
    assert (go[none] == 7).all() and (gl[none] == 7).all()
    empty = np.isneginf(lse_ref)
    assert (go[empty] == 0).all() and np.isneginf(gl[empty]).all()
    fine = ~none & ~empty
    if not fine.any():
        return
    D, n = q.shape[-1], int(s["lens_np"].max())
    big_k = np.sqrt(np.nanmax(np.where(np.isfinite(s["ref"][0]), s["ref"][0], 0) ** 2, axis=(0, 1, 2)).sum())
    size = np.sqrt((q ** 2).sum(-1)) * big_k / math.sqrt(D)  # bounds the sum of a score's terms
    tol = (D * size + n + 64) * 2.0 ** -24
    el = np.abs(gl[fine] - lse_ref[fine]) - 4 * 2.0 ** -24 * np.abs(lse_ref[fine])
    eo = np.abs(go[fine] - o_ref[fine])
    bound = (2.0 ** -8 * (np.abs(o_ref) + mag) * 1.01 + 2 * tol[..., None] * mag)[fine]
    log("  o %.2e of its bound, lse %.2e of %.2e" % ((eo / np.maximum(bound, 1e-30)).max(), el.max(), tol[fine].max()))
    assert (eo <= bound).all() and (el <= tol[fine]).all()


CASES = [  # lens, news, Hq, Hkv, D, page, pad
    ([1], [1], 1, 1, 64, 1, 0), ([2], [2], 1, 1, 128, 16, 1), ([31], [1], 4, 2, 64, 8, 0), ([32], [1], 8, 1, 128, 32, 0),
    ([33, 1, 0, 64, 65, 7], [1, 1, 0, 1, 1, 1], 8, 2, 128, 16, 3), ([0, 0, 5], [0, 0, 1], 2, 2, 64, 4, 0),
    ([1000, 3, 517], [1, 3, 32], 12, 4, 128, 64, 0), ([2049, 100], [8, 5], 28, 4, 128, 128, 2),
    ([700], [32], 32, 1, 64, 1024, 0), ([5000, 4999, 17], [1, 2, 17], 32, 8, 128, 16, 0),
    ([300] * 40, [1] * 40, 16, 16, 64, 32, 0), ([40, 9] * 36, [1, 2] * 36, 32, 16, 64, 16, 0),
    ([70, 1, 0, 12] * 250, [1, 1, 0, 3] * 250, 3, 1, 128, 4, 1), ([260] * 3, [32, 1, 9], 80, 40, 64, 8, 0), ([3333], [3], 40, 8, 64, 2, 0), ([129, 64], [1, 1], 64, 1, 128, 8, 0)]


# Tables as wide as the requests need (short ones are done in one launch), and wide enough for 70000
# keys (shares of all tiles and a second launch).
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, e4m3, wide):
    lens, news, Hq, Hkv, D, page, pad = CASES[case]
    log("paged attention %s e4m3=%d wide=%d" % (CASES[case], e4m3, wide))
    s = make(case, lens, news, Hq, Hkv, D, page, e4m3, pad, extra_cols=70000 // page if wide else 1)
    check(s, *call(s, max(max(news), 1)))


def test_one_row_a_request_without_offsets():
    lens = [40, 1, 333, 0]
    s = make(50, lens, [1] * 4, 8, 2, 64, 16, False, pad=2)
    o, lse = call(s, 1, cu=False)
    check(s, o, lse)


def test_rows_that_see_no_key():
    """A request of fewer cached tokens than rows, one of negative length, one whose pages are all
    outside the cache; and a request longer than its table has columns."""
    s = make(51, [3, 0, 40, 112], [5, 2, 1, 1], 4, 4, 64, 16, False, extra_cols=0)
    s["table_np"][2] = [-1, 1 << 30, -(1 << 30), 10 ** 6, s["k"].shape[0], -7, 99]
    s["lens_np"] = np.array([3, -9, 40, 500])
    s["table"], s["lens"] = (torch.tensor(s[k], dtype=torch.int32, device="cuda") for k in ("table_np", "lens_np"))
    check(s, *call(s, 5))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_bad_pages_in_the_middle_count_for_nothing(D, e4m3):
    s = make(52 + D, [700, 90], [2, 4], 8, 2, D, 8, e4m3)
    n_pages = s["k"].shape[0]
    for j, bad in ((0, -1), (3, n_pages), (4, 2 ** 31 - 1), (40, -2 ** 31)):
        s["table_np"][0, j] = bad
    s["table_np"][1, 5] = -1
    s["table"] = torch.tensor(s["table_np"], dtype=torch.int32, device="cuda")
    # page 0 of the cache belongs to nobody now and holds what must not be read as a value
    check(s, *call(s, 4))


@pytest.mark.parametrize("lens,cols", [((100, 260), 1), ((100, 260), 3000), ((30, 17), 1)])
def test_values_a_mask_hides_do_not_spread(lens, cols):
    """Infinite and NaN keys and values of a later new token reach that token and those after it,
    no earlier one; of an ordinary token everybody."""
    for e4m3 in (False, True):
        s = make(53, list(lens), [6, 3], 8, 2, 128, 16, e4m3, extra_cols=cols)

        def put(r, p, h, what):
            i = s["table_np"][r, p // 16]
            for t in ("k", "v") if what == "nan" else ("v",):
                if e4m3:
                    s[t].view(torch.uint8)[i, p % 16, h, 5] = 0x7f
                else:
                    s[t][i, p % 16, h, 5] = float(what)

        put(0, lens[0] - 3, 1, "nan")  # the fourth new token of request 0, key head 1
        put(1, lens[1] - 1, 0, "inf")  # the last of request 1, key head 0
        o, lse = call(s, 6)
        go = np64(o)
        assert np.isnan(go[3:6, 4:]).all() and np.isfinite(go[:3]).all() and np.isfinite(go[3:6, :4]).all()
        assert not np.isfinite(go[8, :4, 5]).any() and np.isfinite(go[6:8]).all() and np.isfinite(go[8, 4:]).all()
        assert np.isfinite(np.delete(go[8], 5, axis=-1)).all()
        # s["ref"] is from before: the rows that see none of it are as they were
        ref, _, mag = OS.attention(np64(s["q"]), *s["ref"], s["table_np"], s["lens_np"], s["cu_np"])
        for rows in (slice(0, 3), slice(6, 8)):
            assert (np.abs(go - ref) <= 2.0 ** -8 * 1.01 * (np.abs(ref) + mag) + 1e-4 * mag)[rows].all()


@pytest.mark.parametrize("cols", [1, 5000])
def test_scores_of_minus_infinity_and_nan(cols):
    """-inf scores weigh nothing; a row of nothing else has o = 0, lse = -inf; NaN spreads."""
    s = make(54, [50, 40], [1, 1], 2, 1, 64, 16, False, extra_cols=cols)
    s["q"][:] = 1.0
    for r, keys in ((0, range(10)), (1, range(40))):
        for p in keys:
            s["k"][s["table_np"][r, p // 16], p % 16, 0, 0] = float("-inf")
    o, lse = call(s, 1)
    s["ref"] = (OS.cached(np64(s["k"])), s["ref"][1])
    ref, lref, mag = OS.attention(np64(s["q"]), *s["ref"], s["table_np"], s["lens_np"], s["cu_np"])
    assert (np.abs(np64(o)[0] - ref[0]) <= 2.0 ** -8 * 1.01 * (np.abs(ref[0]) + mag[0]) + 1e-4 * mag[0]).all()
    assert np.abs(np64(lse)[0] - lref[0]).max() <= 1e-4
    assert (np64(o)[1] == 0).all() and np.isneginf(np64(lse)[1]).all()
    s["k"][s["table_np"][1, 0], 3, 0, 1] = float("nan")
    o, lse = call(s, 1)
    assert np.isnan(np64(o)[1]).all() and np.isnan(np64(lse)[1]).all() and np.isfinite(np64(o)[0]).all()


def test_large_scores():
    """Scores of thousands: the running maximum carries them."""
    s = make(55, [900, 77], [1, 7], 4, 2, 128, 32, False)
    s["q"] *= 64
    check(s, *call(s, 7))


def test_long_cache_past_32_bit_offsets():
    """A cache of 4.5 GB a side whose last pages a request uses: byte and element offsets past 2^32
    and 2^31."""
    D, Hkv, page = 128, 32, 256
    n_pages = 2200
    k = torch.zeros((n_pages, page, Hkv, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    ids = [2199, 1100, 2198, 0]
    s = make(56, [900, 3], [1, 1], 32, Hkv, D, page, False)
    pos = {int(i): j for i, j in zip(s["table_np"][0], ids)}
    pos[int(s["table_np"][1, 0])] = 2190
    for a, b in pos.items():
        if a >= 0:
            k[b], v[b] = s["k"][a], s["v"][a]
    table = np.array([[pos.get(int(x), -1) if x >= 0 else -1 for x in row] for row in s["table_np"]])
    small = dict(s)
    s["k"], s["v"], s["table"] = k, v, torch.tensor(table, dtype=torch.int32, device="cuda")
    o, lse = call(s, 1)
    o2, lse2 = call(small, 1)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    check(small, o2, lse2)


def test_workspace_streams_and_repeats():
    """A caller's workspace, whatever it held, and another stream give the same bits, call after call."""
    s = make(57, [4000, 9, 2500], [2, 1, 8], 16, 4, 128, 16, False)
    o, lse = call(s, 8)
    n = ra.paged_attn_workspace(3, 16, 4, 128, 8)
    ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")
    st = torch.cuda.Stream()
    for i in range(3):
        o2, lse2 = call(s, 8, workspace=ws)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        with torch.cuda.stream(st):
            o3, lse3 = call(s, 8, workspace=ws if i else None)
        assert torch.equal(o, o3) and torch.equal(lse, lse3)
    if n > 16:
        with pytest.raises(ra.RingAttnError):
            call(s, 8, workspace=ws[:n - 16])
    with pytest.raises(ValueError):
        ra.paged_attn_decode(s["q"], s["k"], s["v"], s["table"], s["lens"][:2], s["cu"], o, lse, 8)
    with pytest.raises(TypeError):
        ra.paged_attn_decode(s["q"], s["k"].half(), s["v"].half(), s["table"], s["lens"], s["cu"], o, lse, 8)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_more_heads_than_waves_a_team(D, e4m3):
    """As many key heads as the library takes: one team of waves for all requests."""
    s = make(60 + D, [70, 3, 0, 41], [2, 1, 0, 3], 1024, 1024, D, 8, e4m3, extra_cols=9000)
    check(s, *call(s, 3))
    s = make(61 + D, [90, 20], [1, 1], 900, 900, D, 16, e4m3, extra_cols=9000)
    check(s, *call(s, 1))


@pytest.mark.parametrize("cols", [1, 3000])
@pytest.mark.parametrize("max_new", [1, 2])
def test_keys_of_rows_past_max_new_do_not_spread(max_new, cols):
    """Requests of more rows than max_new: the rows that are computed see none of the later tokens,
    whatever those hold; the others are left as they are."""
    for e4m3 in (False, True):
        s = make(70 + max_new, [60, 300], [5, 7], 8, 2, 128, 16, e4m3, extra_cols=cols)
        for r, n in ((0, 5), (1, 7)):
            for p in range(s["lens_np"][r] - n + max_new, s["lens_np"][r]):
                i = s["table_np"][r, p // 16]
                for t in ("k", "v"):
                    if e4m3:
                        s[t].view(torch.uint8)[i, p % 16] = 0x7f
                    else:
                        s[t][i, p % 16] = float("inf" if t == "v" else "nan")
        check(s, *call(s, max_new), max_new)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D,keys", [(128, 500), (64, 900), (128, 1100)])
def test_many_requests_of_middling_length(D, keys, e4m3):
    """512 groups of requests and key heads: four waves a group for tables of up to 768 keys, shares
    beyond."""
    lens = [keys - (keys * i) // 70 for i in range(64)]
    news = [1 + i % 3 for i in range(64)]
    s = make(80 + D, lens, news, 16, 8, D, 16, e4m3)
    check(s, *call(s, 3))
