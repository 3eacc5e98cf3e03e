"""paged_append against the oracle: rotation, 8-bit rows, strided inputs, slots left alone.

Tolerances.  An angle's turns have double error, sine and cosine float32 error of a few units of
2^-24, the rotation three roundings: 2^-20 of the pair's size in all.  bf16 outputs add half a
step, 2^-8 of the value.  8-bit outputs are e4m3: half a step, 2^-4 of the value, or half the
smallest step, 2^-10 of the scale; without rotation the input is exact and so are the bits."""
import numpy as np
import pytest
import torch

import paper_2310_01889_amd as ra
from oracle import serving as OS
from tests.gpu_util import log, np64

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def _inputs(T, Hq, Hkv, D, fused, seed):
    g = torch.Generator().manual_seed(seed)
    if fused:
        w = torch.randn(T, Hq + 2 * Hkv + 1, D, generator=g).to(torch.bfloat16).cuda()
        return w[:, :Hq], w[:, Hq:Hq + Hkv], w[:, Hq + Hkv:Hq + 2 * Hkv]
    return tuple(torch.randn(T, h, D, generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))


def _pages(n_pages, page, Hkv, D, e4m3):
    if not e4m3:
        return [torch.full((n_pages, page, Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)] + [None] * 2
    return ([torch.full((n_pages, page, Hkv, D), 7, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
            + [torch.full((n_pages, page, Hkv), 9, dtype=torch.uint8, device="cuda") for _ in range(2)])


def _values(pages, scales):
    return OS.cached(np64(pages.cpu()), None if scales is None else scales.cpu().numpy())


@pytest.mark.parametrize("T,Hq,Hkv,D,page,e4m3,fused", [
    (1, 1, 1, 64, 1, False, False), (1, 32, 8, 128, 16, True, True), (5, 7, 7, 64, 8, True, False),
    (33, 16, 2, 128, 16, False, True), (64, 3, 1, 128, 1024, True, True), (257, 12, 4, 64, 32, False, True),
    (300, 8, 8, 128, 64, True, False), (19, 1024, 1, 64, 4, False, False)])
def test_append(T, Hq, Hkv, D, page, e4m3, fused):
    log("append T=%d Hq=%d Hkv=%d D=%d page=%d e4m3=%d fused=%d" % (T, Hq, Hkv, D, page, e4m3, fused))
    q, k, v = _inputs(T, Hq, Hkv, D, fused, T + Hq)
    rng = np.random.default_rng(T)
    n_pages = -(-T // page) + 2
    slots = rng.permutation(n_pages * page)[:T]
    positions = rng.integers(0, 1 << 20, T)
    positions[0] = 2 ** 31 - 1
    if T > 4:
        slots[1], slots[2], positions[3] = -1, n_pages * page, -1  # not stored, not stored, left out
    kp, vp, ks, vs = _pages(n_pages, page, Hkv, D, e4m3)
    q_out = torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    ra.paged_append(q, k, v, q_out, kp, vp, i32(slots), i32(positions), ks, vs)
    torch.cuda.synchronize()
    keep = positions >= 0
    q_ref, k_ref = OS.rope(np64(q), positions), OS.rope(np64(k), positions)
    pair = lambda x: np.repeat(np.hypot(x[..., 0::2], x[..., 1::2]), 2, axis=-1)
    # positions near 2^31: a double angle of 3e8 turns is off by 2^-25 of a turn
    far = 2.0 ** -20 + np.abs(positions)[:, None, None] * 2.0 ** -50
    got = np64(q_out)
    assert (np.abs(got - q_ref) <= 2.0 ** -8 * np.abs(q_ref) + far * pair(np64(q)))[keep].all()
    assert (got[~keep] == 7).all()
    stored = keep & (slots >= 0) & (slots < n_pages * page)
    for pages, scales, ref, noise in ((kp, ks, k_ref, far * pair(np64(k))), (vp, vs, np64(v), 0 * far)):
        flat = _values(pages, scales).reshape(-1, Hkv, D)
        at, ref, noise = slots[stored], ref[stored], np.broadcast_to(noise, ref.shape)[stored]
        if e4m3:
            step = 2.0 ** (scales.cpu().numpy().reshape(-1, Hkv)[at].astype(float) - 127)[..., None]
            top = np.abs(ref).max(axis=-1, keepdims=True)
            # the smallest scale, up to noise at the border
            assert (top <= 448 * step * (1 + 1e-6)).all() and (top > 224 * step * (1 - 1e-6)).all()
            assert (np.abs(flat[at] - ref) <= 2.0 ** -4 * np.abs(ref) + 2.0 ** -10 * step + noise * 1.1).all()
            if noise.max() == 0:  # not rotated: bit for bit
                for i in range(min(len(at), 8)):
                    for h in range(Hkv):
                        assert np.array_equal(flat[at[i], h], OS.e4m3(ref[i, h])[0])
        else:
            assert (np.abs(flat[at] - ref) <= 2.0 ** -8 * np.abs(ref) + noise).all()
        rest = np.setdiff1d(np.arange(n_pages * page), at)
        raw = pages.view(torch.uint8) if e4m3 else pages
        assert (raw.view(n_pages * page, -1)[torch.tensor(rest, device="cuda")].float() == 7).all()
        if e4m3:
            assert (scales.view(-1, Hkv)[torch.tensor(rest, device="cuda")] == 9).all()


def test_append_in_place_without_rotation_and_keys_alone():
    T, H, D, page = 6, 2, 64, 4
    q, k, v = _inputs(T, H, H, D, False, 3)
    kp, vp, _, _ = _pages(2, page, H, D, False)
    slots = torch.tensor([7, 6, 5, 4, 3, 2], dtype=torch.int32, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    q0 = q.clone()
    ra.paged_append(q, k, v, q, kp, vp, slots, pos, rotate=False)
    assert torch.equal(q, q0) and torch.equal(kp.view(-1, H, D)[slots.long()], k)
    assert torch.equal(vp.view(-1, H, D)[slots.long()], v)
    out = torch.empty_like(q)
    ra.paged_append(q, k, v, out, kp, vp, slots, pos)
    want = kp.clone()
    ra.paged_append(q, k, v, q, kp, vp, slots, pos)  # q in place
    assert torch.equal(q, out)
    kp.zero_()
    ra.paged_append(None, k, v, None, kp, vp, slots, pos)
    torch.cuda.synchronize()
    assert torch.equal(kp.view(-1, H, D)[slots.long()], want.view(-1, H, D)[slots.long()])


def test_append_e4m3_values_at_the_edges():
    """Infinities and NaN are stored as NaN and leave the scale to the others; zero rows; the
    largest and smallest bf16 numbers; rounding ties."""
    D = 64
    x = torch.zeros(6, 1, D)
    x[0, 0, :3] = torch.tensor([float("inf"), -3.0, float("nan")])
    x[2, 0, :4] = torch.tensor([3.3e38, -1.0, 1e38, 2e37])
    x[3, 0, :4] = torch.tensor([1e-39, -1e-40, 5e-39, 0.0])
    x[4, 0, :6] = torch.tensor([448.0, 17.0, 19.0, -21.0, 0.0009765625, 0.0029296875])
    x[5] = float("-inf")
    x = x.to(torch.bfloat16).cuda()
    kp, vp, ks, vs = _pages(6, 1, 1, D, True)
    idx = torch.arange(6, dtype=torch.int32, device="cuda")
    ra.paged_append(None, x, x, None, kp, vp, idx, idx, ks, vs, rotate=False)
    torch.cuda.synchronize()
    for pages, scales in ((kp, ks), (vp, vs)):
        got = _values(pages, scales)
        for i in range(6):
            want, e = OS.e4m3(np64(x)[i, 0])
            assert np.array_equal(got[i, 0, 0], want, equal_nan=True), i
            assert int(scales[i, 0, 0]) == e + 127
