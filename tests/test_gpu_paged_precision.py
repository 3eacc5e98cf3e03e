"""paged_attn_decode where the sums nearly cancel: values of +1 and -1 under probabilities that are
nearly equal, so that o is small and neither its storage in bf16 nor the mean of |v| = 1 hides how
exactly the probabilities enter the products.

Tolerance.  Scores are below 2^-8 in size, the sums of their D terms below 2^-6: off by D 2^-24 2^-6
at most (times log2(e), and its own rounding).  A probability is the hardware's 2^x, off by a unit
in the last place (2^-23 of it) and by what its argument is off; its product with a value is exact.
Numerator and denominator add n terms of at most 1 each in float32, in any order: n 2^-24 of their
number each at most.  The quotient and its weights where parts are joined: 2^-22.  So o is off by
at most 2 (D 2^-30 log2(e) + 2^-23 + n 2^-24) + 2^-22 beside its own rounding, 2^-8 of the value."""
import numpy as np
import pytest
import torch

from oracle import serving as OS
from tests.gpu_util import log, np64
from tests.test_gpu_paged_attention import E4M3, call, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_probabilities_enter_the_products_as_they_are(D, e4m3, wide):
    lens = [2, 3, 5, 8] * 6
    s = make(90 + D, lens, [1] * len(lens), 16, 4, D, 16, e4m3, extra_cols=5000 if wide else 1)
    g = torch.Generator().manual_seed(91)
    shape = tuple(s["k"].shape)
    k = torch.randn(shape, generator=g).clamp(-4, 4) * 64
    sign = torch.randint(0, 2, shape, generator=g) * 2.0 - 1
    if e4m3:
        s["k"], s["v"] = k.to(E4M3).cuda(), sign.to(E4M3).cuda()
        s["ks"].fill_(127 - 18)
        s["vs"].fill_(127)
        s["ref"] = (np64(s["k"]) * 2.0 ** -18, np64(s["v"]))
    else:
        s["k"], s["v"] = (k * 2.0 ** -18).to(torch.bfloat16).cuda(), sign.to(torch.bfloat16).cuda()
        s["ref"] = (np64(s["k"]), np64(s["v"]))
    o, lse = call(s, 1)
    ref, lref, mag = OS.attention(np64(s["q"]), *s["ref"], s["table_np"], s["lens_np"], s["cu_np"])
    assert (mag <= 1 + 1e-9).all()
    n = np.array(lens)[:, None, None]
    bound = 2.0 ** -8 * np.abs(ref) + 2 * (D * 2.0 ** -30 * 1.4427 + 2.0 ** -23 + n * 2.0 ** -24) + 2.0 ** -22
    err = np.abs(np64(o) - ref)
    log("  o %.2e of its bound; smallest |o| %.1e" % ((err / bound).max(), np.abs(ref).min()))
    assert (err <= bound).all()
    # scores, their largest and the sum of n terms: as above, the logarithm of it 2^-22
    assert (np.abs(np64(lse) - lref) <= (D * 2.0 ** -30 + (n[..., 0] + 8) * 2.0 ** -24)).all()


@pytest.mark.parametrize("wide", [False, True])
def test_an_infinite_value_of_small_probability(wide):
    """Scores that lie up to 118 (log2 units) below the largest: probabilities of 2^-118 are float32 and
    bf16 numbers, and an infinite value under them makes o infinite, not NaN."""
    D, n = 128, 40
    s = make(93, [n], [1], 1, 1, D, 16, False, extra_cols=5000 if wide else 1)
    s["q"].zero_()
    s["q"][0, 0, 0] = 8.0 * 2 ** 0.5 * 0.6875  # times k / sqrt(128): 0.6875 k nats, 0.99 k in log2 units
    for p in range(n):
        i = s["table_np"][0, p // 16]
        s["k"][i, p % 16, 0, 0] = -3.0 * p
        s["v"][i, p % 16, 0] = 1.0
        s["v"][i, p % 16, 0, p] = float("inf")
        s["v"][i, p % 16, 0, 64 + p] = float("-inf")
    o, lse = call(s, 1)
    assert (o[0, 0, :n] == float("inf")).all() and (o[0, 0, 64:64 + n] == float("-inf")).all()
    assert (o[0, 0, n:64] == 1).all()


def test_a_huge_value_of_small_probability():
    """Zeros but for one value of 2^127 under a probability of 2^-106 to 2^-119: o is their product to bf16's
    precision, as no part of a probability is moved by more than 2^-132: 2^-13 of it.

    Scores are 0 and one product of two bf16 numbers, so the probability is 2^x with x rounded at 120:
    2^-18 in x, 2^-18 ln 2 of the value, and the hardware's own 2^-23."""
    D = 64
    ks = [-range_ / 8 for range_ in range(108 * 8, 118 * 8)]
    s = make(94, [2] * len(ks), [1] * len(ks), 1, 1, D, 16, False)
    s["q"].zero_()
    s["k"].zero_()
    s["v"].zero_()
    s["q"][:, 0, 0] = 8.0
    for r, x in enumerate(ks):
        i = s["table_np"][r, 0]
        s["k"][i, 1, 0, 0] = x * 0.6931  # times 8 / sqrt(64)
        s["v"][i, 1, 0, 3] = 2.0 ** 127
    o, lse = call(s, 1)
    k = np64(torch.stack([s["k"][s["table_np"][r, 0], 1, 0, 0] for r in range(len(ks))]))
    want = np.exp(k) * 2.0 ** 127
    assert (np.exp(k) > 2.0 ** -119).all() and (np.exp(k) < 2.0 ** -106).all()
    err = np.abs(np64(o)[:, 0, 3] / want - 1)
    log("  relative error %.2e, bf16 rounds by up to %.2e" % (err.max(), 2.0 ** -8))
    assert (err <= 2.0 ** -8 + 2.0 ** -13 + 2.0 ** -18 + 2.0 ** -22).all()
    assert (np64(o)[:, 0, :3] == 0).all()
