"""paged_plan against the oracle's allocator: every output equal, canaries past them untouched."""
import numpy as np
import pytest
import torch

import paper_2310_01889_amd as ra
from oracle import serving as OS
from tests.gpu_util import log

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _run(lens, n_new, free, head, table, page, n_pages, T):
    R = len(lens)
    out = [torch.full((n + 3,), -77, dtype=torch.int32, device="cuda") for n in (R + 1, R, T, T, 4)]
    cu, new_lens, slots, positions, counts = (t[:-3] for t in out)
    td = _i32(table)
    for _ in range(2):  # again with the same inputs: the same outputs
        ra.paged_plan(_i32(lens), _i32(n_new), _i32(free), None if head is None else _i32([head]), td, cu, new_lens,
                      slots, positions, counts, page, n_pages)
    torch.cuda.synchronize()
    assert all((t[-3:] == -77).all() for t in out)
    return [x.cpu().numpy() for x in (td, cu, new_lens, slots, positions, counts)]


def _check(*args):
    got = _run(*args)
    lens, n_new, free, head, table, page, n_pages, T = args
    want = OS.plan(lens, n_new, free, head or 0, table, page, n_pages, T)
    for name, g, w in zip(("table", "cu_rows", "new_lens", "slots", "positions", "counts"), got, want):
        assert np.array_equal(g, w), (name, g, w)
    return want


@pytest.mark.parametrize("R,page,max_len,max_new,pad", [
    (1, 16, 0, 1, 0), (1, 1, 9, 40, 3), (3, 1024, 5000, 1, 1), (64, 16, 400, 1, 0), (65, 8, 100, 0, 7),
    (255, 32, 900, 5, 2), (257, 64, 300, 30, 1000), (1000, 16, 200, 3, 5), (4096, 2, 20, 2, 1), (9, 128, 2000, 900, 100)])
def test_plan(R, page, max_len, max_new, pad):
    log("plan R=%d page=%d max_len=%d max_new=%d pad=%d" % (R, page, max_len, max_new, pad))
    g = np.random.default_rng(R * page + max_new)
    lens, n_new = g.integers(0, max_len + 1, R), g.integers(0, max_new + 1, R)
    lens[0], n_new[-1] = max_len, max_new
    held = -(-lens // page)
    need = -(-(lens + n_new) // page) - held
    max_pages = int((held + need).max()) + 1
    n_pages = int((held + need).sum()) + 4
    ids = g.permutation(n_pages)
    table = np.full((R, max_pages), -5)  # entries past a request's pages are left as they are
    at = 0
    for r in range(R):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    T = max(1, int(n_new.sum()) + pad)
    free = np.concatenate([[n_pages + 9, -3], ids[at:]])  # two used up before
    want = _check(lens, n_new, free, 2, table, page, n_pages, T)
    assert want[5][3] == 0
    # too few free pages; too few rows; too few columns; a head past the list; a head below zero
    if need.sum() > 1:
        assert _check(lens, n_new, free[:2 + int(need.sum()) // 2], 2, table, page, n_pages, T)[5][3] == ra.PLAN_PAGES
    if n_new.sum() > 1:
        assert _check(lens, n_new, free, 2, table, page, n_pages, int(n_new.sum()) // 2)[5][3] == ra.PLAN_ROWS
        _check(lens, n_new, free, 2, np.ascontiguousarray(table[:, :max(1, max_pages // 2)]), page, n_pages, T)
    _check(lens, n_new, free, len(free) + 5, table, page, n_pages, T)
    assert _check(lens, n_new, free, -1, table, page, n_pages, T)[5][3] & ra.PLAN_BAD_INPUT


def test_plan_bad_integers():
    """Negative and huge lengths, ids outside the cache in the list and in entries held."""
    big = 2 ** 31 - 1
    table = np.array([[0, -1, -1, -1], [99, 2, -1, -1], [3, -9, 4, -1], [-1] * 4, [5, 6, 7, 8]])
    _check([3, 6, 9, -4, big], [2, 1, 1, 3, 2], [11, 200, -1, 9], None, table, 4, 12, 16)
    _check([3, 6, 9, 0, 0], [big, -1, big, big, 0], [11, 200, -1, 9], 0, table, 4, 12, 5)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_slots_and_positions_off_a_16_byte_boundary(shift):
    lens, n_new, page, T = np.array([5, 0, 17, 40]), np.array([3, 9, 0, 6]), 8, 23
    free, table = np.arange(30, 60), np.arange(24).reshape(4, 6)
    want = OS.plan(lens, n_new, free, 0, table, page, 64, T)
    buf = torch.full((2, T + 8), -77, dtype=torch.int32, device="cuda")
    slots, pos = buf[0, shift:shift + T], buf[1, shift:shift + T]
    td, cu, nl, counts = _i32(table), _i32([0] * 5), _i32([0] * 4), _i32([0] * 4)
    ra.paged_plan(_i32(lens), _i32(n_new), _i32(free), None, td, cu, nl, slots, pos, counts, page, 64)
    assert np.array_equal(slots.cpu().numpy(), want[3]) and np.array_equal(pos.cpu().numpy(), want[4])
    assert (buf[:, :shift] == -77).all() and (buf[:, shift + T:] == -77).all()


def test_positions_past_31_bits():
    """Positions end at 2^31 - 1; slots go by what they would be."""
    page, cols = 1024, (1 << 21) + 2
    table = np.full((1, cols), 3)
    _check(np.array([2 ** 31 - 2]), np.array([1027]), np.array([7, 5]), None, table, page, 9, 1030)
