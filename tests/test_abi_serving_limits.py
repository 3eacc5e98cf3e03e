"""Sizes at the edge of what the serving calls' launches hold, refused without a GPU."""
import ctypes
import os

import pytest

import paper_2310_01889_amd as ra

RA_EUNSUPPORTED = 2
P, P2, P3, NULL = (ctypes.c_void_p(x) for x in (0x1000, 0x2000, 0x3000, 0))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ra.library_path()):
        pytest.skip("library not built")
    return ra.load()


def test_packing_grid(lib):
    """2^29 - 96 inputs and more are 2^22 blocks of 128, four workgroups of 256 threads each: 2^32
    threads, one more than a launch takes."""
    for d_in in ((1 << 29) - 32, (1 << 29) - 96):
        assert 4 * -(-d_in // 128) * 256 == 1 << 32
        assert lib.mx4_pack(P, P2, P3, d_in, 1, NULL) == RA_EUNSUPPORTED
        assert b"2^29" in lib.ring_attn_last_error()
        assert lib.mx4_linear(P, P2, P3, NULL, ctypes.c_void_p(0x4000), 1, d_in, 1, NULL) == RA_EUNSUPPORTED
