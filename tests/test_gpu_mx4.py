"""mx4_pack and mx4_linear against the oracle.

Packing is exact.  Tolerance of the product: float32 sums of d_in terms, each term rounded by at
most 2^-24 of the running sum, bounded by d_in 2^-24 of the sum of the terms' sizes (products of a
bf16 and an e2m1 number are exact in float32); then the residual's addition, 2^-24, and half a
bf16 step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

import paper_2310_01889_amd as ra
from oracle import serving as OS
from tests.gpu_util import log, np64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K,N", [(32, 1), (64, 16), (96, 17), (128, 40), (416, 300), (1056, 33)])
def test_pack(K, N):
    log("mx4 pack %d x %d" % (K, N))
    g = torch.Generator().manual_seed(K + N)
    w = torch.randn(K, N, generator=g) * torch.exp(2 * torch.randn(K, N, generator=g))
    w[:32, 0] = 0
    if N > 4:
        w[:32, 1] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -6.0] * 4)
        w[3, 2], w[40, 3] = float("inf"), float("nan")
        w[:32, 4] *= 1e-38
    w = w.to(torch.bfloat16)
    w4, scales = ra.mx4_weights(w.cuda())
    torch.cuda.synchronize()
    w4_ref, s_ref = OS.mx4_pack(np64(w))
    assert np.array_equal(scales.cpu().numpy(), s_ref)
    got = OS.mx4_values(w4.cpu().numpy(), scales.cpu().numpy(), K, N)
    want = OS.mx4_values(w4_ref, s_ref, K, N)
    assert np.array_equal(got, want, equal_nan=True) and np.isnan(want).sum() == 32 * (s_ref == 255).sum()
    # no codes past the ends
    full = OS.mx4_values(w4.cpu().numpy(), np.full_like(s_ref, 127), 128 * w4.shape[1], 16 * w4.shape[0])
    assert (full[K:] == 0).all() and (full[:, N:] == 0).all()


@pytest.mark.parametrize("T,K,N,residual", [
    (1, 32, 1, False), (1, 4096, 64, True), (2, 96, 17, True), (3, 1056, 300, False), (16, 256, 48, True),
    (17, 416, 100, False), (31, 2080, 130, True), (33, 128, 16, True), (64, 512, 65, False), (65, 160, 20, True),
    (130, 288, 33, True), (512, 64, 50, False), (5, 11008, 40, True)])
def test_linear(T, K, N, residual):
    log("mx4 linear T=%d K=%d N=%d residual=%d" % (T, K, N, residual))
    g = torch.Generator().manual_seed(T * K + N)
    w = (0.02 * torch.randn(K, N, generator=g)).to(torch.bfloat16).cuda()
    x = (torch.randn(T, K, generator=g) + 0.5).to(torch.bfloat16).cuda()
    res = torch.randn(T, N, generator=g).to(torch.bfloat16).cuda() if residual else None
    w4, scales = ra.mx4_weights(w)
    guard = torch.full((T * N + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
    y = guard[:T * N].view(T, N)
    ra.mx4_linear(x, w4, scales, res, y)
    torch.cuda.synchronize()
    wv = OS.mx4_values(w4.cpu().numpy(), scales.cpu().numpy(), K, N)
    ref = np64(x) @ wv
    size = np.abs(np64(x)) @ np.abs(wv)
    if residual:
        ref, size = ref + np64(res), size + np.abs(np64(res))
    err, bound = np.abs(np64(y) - ref), 2.0 ** -8 * np.abs(ref) + (K + 1) * 2.0 ** -24 * size
    log("  %.2e of its bound" % (err / bound).max())
    assert (err <= bound).all() and (guard[T * N:] == 7).all()


@pytest.mark.parametrize("T,K,N", [
    (1, 2208, 9005), (1, 2208, 4100), (2, 1184, 14000), (5, 1184, 20000), (7, 2208, 5003), (8, 1184, 11000),
    (9, 4256, 1000), (12, 1184, 20000), (16, 2208, 8190), (11, 2208, 9005), (20, 2208, 6001), (20, 416, 20000),
    (31, 1184, 11000), (70, 416, 9005), (40, 1184, 12001), (90, 1056, 11000), (60, 1184, 9005), (200, 416, 8190),
    (6, 1184, 13001), (15, 1184, 14000), (23, 1184, 7000), (18, 1184, 13000), (66, 416, 13003), (45, 416, 15999)])
def test_linear_in_every_shape_of_workgroup(T, K, N):
    """Rows and outputs that take each number of row tiles and output blocks a workgroup, with a
    ragged end each; more inputs than the waves of one take at a time."""
    log("mx4 linear T=%d K=%d N=%d" % (T, K, N))
    g = torch.Generator(device="cuda").manual_seed(T + K + N)
    w4, scales = ra.mx4_weights((0.02 * torch.randn(K, N, generator=g, device="cuda")).to(torch.bfloat16))
    x = torch.randn(T, K, generator=g, device="cuda").to(torch.bfloat16)
    res = torch.randn(T, N, generator=g, device="cuda").to(torch.bfloat16)
    guard = torch.full((T * N + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
    y = guard[:T * N].view(T, N)
    ra.mx4_linear(x, w4, scales, res, y)
    torch.cuda.synchronize()
    wv = OS.mx4_values(w4.cpu().numpy(), scales.cpu().numpy(), K, N)
    ref = np64(x) @ wv + np64(res)
    size = np.abs(np64(x)) @ np.abs(wv) + np.abs(np64(res))
    err, bound = np.abs(np64(y) - ref), 2.0 ** -8 * np.abs(ref) + (K + 1) * 2.0 ** -24 * size
    log("  %.2e of its bound" % (err / bound).max())
    assert (err <= bound).all() and (guard[T * N:] == 7).all()
    again = torch.empty_like(y)
    ra.mx4_linear(x, w4, scales, res, again)
    assert torch.equal(y, again)


def test_every_code_and_scale():
    """Each of the 16 codes under scales from 2^-126 to 2^127, and a NaN scale, read by a product
    that picks one input out."""
    K, N = 128, 256
    w4 = torch.zeros((16, 1, 64, 16), dtype=torch.uint8)
    code = torch.arange(64 * 16).view(64, 16) % 16
    w4[:, 0] = (code | (15 - code) << 4).to(torch.uint8)
    scales = torch.arange(1, 257).clamp(max=255).to(torch.uint8).view(16, 1, 16, 1).expand(16, 1, 16, 4).contiguous()
    x = torch.zeros(K, K)
    x[torch.arange(K), torch.arange(K)] = 1
    xs = x.to(torch.bfloat16).cuda()
    y = torch.empty(K, N, dtype=torch.bfloat16, device="cuda")
    ra.mx4_linear(xs, w4.cuda(), scales.cuda(), None, y)
    want = OS.mx4_values(w4.numpy(), scales.numpy(), K, N)
    with np.errstate(over="ignore"):
        want = torch.tensor(want).float().to(torch.bfloat16)  # 4 and 6 at 2^127 are past float32: infinite
    got = y.cpu()
    tiny = want.abs() < 2.0 ** -126  # subnormal products may be flushed
    assert torch.equal(torch.isnan(got), torch.isnan(want) | torch.isnan(got) & torch.isinf(want).any(0))
    ok = (got == want) | torch.isnan(want) | tiny & ((got == 0) | (got == want)) | torch.isinf(want).any(0)
    assert ok.all()


def test_nonfinite_inputs_reach_every_output_of_their_row():
    x = torch.ones(3, 64, dtype=torch.bfloat16)
    x[1, 5], x[2, 40] = float("nan"), float("inf")
    w = torch.ones(64, 20, dtype=torch.bfloat16).cuda()
    w4, scales = ra.mx4_weights(w)
    y = torch.empty(3, 20, dtype=torch.bfloat16, device="cuda")
    ra.mx4_linear(x.cuda(), w4, scales, None, y)
    assert (y[0] == 64).all() and torch.isnan(y[1]).all() and (y[2] == float("inf")).all()
