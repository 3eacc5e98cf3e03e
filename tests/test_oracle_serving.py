"""Pins of the serving oracle that need no GPU: the page plan against its invariants, the 8-bit
and 4-bit roundings against torch and brute force, attention over pages against the plain one,
and what it does with empty rows, bad pages and values that a mask hides."""
import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import serving as OS


def _gen(seed):
    return np.random.default_rng(seed)


@pytest.mark.parametrize("R,page,T", [(1, 16, 5), (7, 8, 40), (40, 1, 200), (33, 128, 64)])
def test_plan_hands_out_every_slot_once(R, page, T):
    g = _gen(R)
    lens, n_new = g.integers(0, 60, R), g.integers(0, 4, R)
    n_pages = 4096
    ids = g.permutation(n_pages)
    table = np.full((R, 128), -1)
    at = 0
    for r in range(R):
        h = -(-lens[r] // page)
        table[r, :h] = ids[at:at + h]
        at += h
    out, cu, new_lens, slots, pos, counts = OS.plan(lens, n_new, ids[at:], 0, table, page, n_pages, T)
    rows = cu[-1]
    assert rows == min(T, n_new.sum()) and (slots[rows:] == -1).all() and (pos[rows:] == -1).all()
    assert len(set(slots[:rows])) == rows and (slots[:rows] >= 0).all()
    for r in range(R):
        for i in range(cu[r], cu[r + 1]):
            assert pos[i] == lens[r] + i - cu[r]
            assert slots[i] == out[r, pos[i] // page] * page + pos[i] % page
        assert new_lens[r] == lens[r] + cu[r + 1] - cu[r]
    assert counts[3] == (OS.FLAG_ROWS if n_new.sum() > T else 0)
    assert (out[table >= 0] == table[table >= 0]).all()


def test_plan_flags():
    t = np.full((2, 2), -1)
    out, _, new_lens, slots, _, counts = OS.plan([0, 7], [5, 3], [3, 99], 0, np.array([[-1, -1], [1, 2]]), 4, 8, 10)
    assert counts.tolist() == [8, 2, 2, OS.FLAG_CAPACITY]  # 10 tokens of request 1 in 2 pages of 4
    assert out.tolist() == [[3, -1], [1, 2]] and slots[4] == -1 and slots[5] == 2 * 4 + 3 and slots[6] == -1
    assert new_lens.tolist() == [5, 10]
    assert OS.plan([0, 0], [4, 4], [3], 0, t, 4, 8, 10)[5].tolist() == [8, 1, 1, OS.FLAG_PAGES]
    assert OS.plan([-1, 0], [1, -2], [3], -4, t, 4, 8, 10)[5].tolist() == [1, 1, 1, OS.FLAG_BAD]


def test_e4m3_matches_torch():
    g = _gen(5)
    for scale in (1e-30, 1e-3, 1.0, 700.0, 1e30):
        x = torch.from_numpy(g.standard_normal(128) * scale).to(torch.bfloat16)
        vals, e = OS.e4m3(x.double().numpy())
        want = (x.double() * 2.0 ** -e).float().to(torch.float8_e4m3fn).double() * 2.0 ** e
        assert np.array_equal(vals, want.numpy())
        top = float(x.double().abs().max())
        assert top <= 448 * 2.0 ** e and top > 448 * 2.0 ** (e - 1)
    vals, e = OS.e4m3([np.inf, -3.0, np.nan, 448.0])
    assert np.isnan(vals[[0, 2]]).all() and vals[1] == -3 and vals[3] == 448 and e == 0


def test_mx4_codes_are_the_nearest():
    g = _gen(6)
    w = g.standard_normal((160, 21)) * np.exp(g.standard_normal((160, 21)))
    w[32:64, 3] = 0
    w[:32, 4] = np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -6.0], 4)  # ties
    w4, scales = OS.mx4_pack(w)
    got = OS.mx4_values(w4, scales, 160, 21)
    assert got[:8, 4].tolist() == [0, 1, 1, 2, 2, 4, 4, -6] and (got[32:64, 3] == 0).all()
    for n in range(21):
        for k0 in range(0, 160, 32):
            x, y = w[k0:k0 + 32, n], got[k0:k0 + 32, n]
            s = 2.0 ** (float(scales[n // 16, k0 // 128, n % 16, k0 // 32 % 4]) - 127)
            grid = np.concatenate([-OS.E2M1, OS.E2M1]) * s
            best = np.abs(grid[None] - x[:, None]).min(axis=1)
            assert np.allclose(np.abs(y - x), best, rtol=0, atol=1e-12 * s) and np.abs(x).max() <= 6 * s


def _cache(g, n_pages, page, Hkv, D):
    return g.standard_normal((n_pages, page, Hkv, D)), g.standard_normal((n_pages, page, Hkv, D))


def test_attention_is_the_plain_one_where_a_request_fills_its_pages():
    g = _gen(7)
    k, v = _cache(g, 6, 8, 2, 16)
    n, S = 5, 48
    q = g.standard_normal((n, 4, 16))
    table = g.permutation(6)[None]
    o, lse, _ = OS.attention(q, k, v, table, [S], [0, n])
    kf, vf = (x[table[0]].reshape(1, S, 2, 16).repeat(2, axis=2) for x in (k, v))
    qf = np.concatenate([np.zeros((1, S - n, 4, 16)), q[None]], axis=1)
    o_ref, lse_ref = OA.attention_fwd(qf, kf, vf, causal=True)[:2]
    assert np.allclose(o, o_ref[0, S - n:], atol=1e-12)
    assert np.allclose(lse, np.asarray(lse_ref)[0, :, S - n:].T, atol=1e-12)


def test_attention_empty_rows_and_bad_pages():
    g = _gen(8)
    k, v = _cache(g, 4, 4, 1, 8)
    q = g.standard_normal((5, 2, 8))
    k[3], v[3] = np.nan, np.inf  # a page no table lists
    v[1, 2:] = np.nan            # rows past the end of request 0
    table = np.array([[0, 1, -1], [2, 7, 2], [-1, 4, 9]])
    o, lse, _ = OS.attention(q, k, v, table, [6, 10, 9], [0, 1, 3, 4])
    assert np.isfinite(o[:3]).all() and np.isfinite(lse[:3]).all()
    assert (o[3] == 0).all() and np.isneginf(lse[3]).all()  # no page of request 2 is valid
    assert np.isnan(o[4]).all()                              # no request's row
    both = OS.attention(q[1:3], k, v, np.array([[2, 2]]), [6], [0, 2])[0]
    assert np.allclose(o[1:3], both)                         # the bad page in between counts for nothing
