"""Arguments the serving entry points refuse, checked without a GPU: every call here fails
validation, so no pointer is used and nothing is enqueued."""
import ctypes
import os

import pytest
import torch

import paper_2310_01889_amd as ra

RA_EINVAL, RA_EUNSUPPORTED = 1, 2
P = ctypes.c_void_p(0x1000)
P2, P3 = ctypes.c_void_p(0x2000), ctypes.c_void_p(0x3000)
MIS = ctypes.c_void_p(0x1008)
MIS4 = ctypes.c_void_p(0x1002)
NULL = ctypes.c_void_p(0)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ra.library_path()):
        pytest.skip("library not built")
    return ra.load()


def test_plan_refusals(lib):
    def plan(*, lens=P, head=NULL, new_lens=P2, counts=P3, slots=P, R=4, page=16, mp=8, n_pages=64, n_free=9, T=4):
        return lib.paged_plan(lens, P, P, head, P, P, new_lens, slots, P, counts, R, page, mp, n_pages, n_free, T, NULL)
    assert plan(lens=NULL) == RA_EINVAL and plan(slots=NULL) == RA_EINVAL
    assert plan(slots=MIS4) == RA_EINVAL
    assert plan(new_lens=P) == RA_EINVAL                     # in place
    assert plan(head=ctypes.c_void_p(0x3008)) == RA_EINVAL   # inside counts
    for bad in (dict(R=0), dict(page=0), dict(mp=0), dict(n_pages=-1), dict(n_free=0), dict(T=0)):
        assert plan(**bad) == RA_EINVAL, bad
    for bad in (dict(page=24), dict(page=2048), dict(R=4097), dict(n_pages=1 << 27)):
        assert plan(**bad) == RA_EUNSUPPORTED, bad
    assert b"2^31" in lib.ring_attn_last_error()


def test_append_refusals(lib):
    def app(*, q=P, k=P, q_out=P2, ks=NULL, vs=NULL, T=4, Hq=8, Hkv=2, D=64, qs=512, kst=128, vst=128, n_pages=9,
            page=16, kv=0, rot=1):
        return lib.paged_append(q, k, P, q_out, P, P, ks, vs, P, P, T, Hq, Hkv, D, qs, kst, vst, n_pages, page, kv, rot,
                                NULL)
    assert app(k=NULL) == RA_EINVAL and app(q=NULL) == RA_EINVAL and app(q_out=NULL) == RA_EINVAL
    assert app(q=MIS) == RA_EINVAL
    assert app(kv=2) == RA_EINVAL and app(rot=2) == RA_EINVAL
    assert app(kv=1) == RA_EINVAL and b"scales" in lib.ring_attn_last_error()
    assert app(ks=P) == RA_EINVAL                       # a bf16 cache has none
    assert app(qs=504) == RA_EINVAL and app(kst=132) == RA_EINVAL and app(vst=64) == RA_EINVAL
    assert app(q=P, q_out=P, qs=1024) == RA_EINVAL      # in place, rows apart
    assert app(T=0) == RA_EINVAL and app(Hq=0) == RA_EINVAL and app(Hkv=0) == RA_EINVAL
    assert app(D=96, qs=768, kst=192, vst=192) == RA_EUNSUPPORTED
    assert app(page=48) == RA_EUNSUPPORTED
    assert app(T=1 << 24) == RA_EUNSUPPORTED
    assert app(Hq=1025, qs=65600) == RA_EUNSUPPORTED


def test_attention_refusals(lib):
    def att(*, q=P, ks=NULL, vs=NULL, cu=P, lse=P, ws=NULL, wsb=0, T=4, R=4, Hq=8, Hkv=2, D=64, n_pages=9, page=16,
            mp=4, max_new=1, kv=0):
        return lib.paged_attn_decode(q, P, P, ks, vs, P, P, cu, P2, lse, ws, wsb, T, R, Hq, Hkv, D, n_pages, page, mp,
                                     max_new, kv, NULL)
    assert att(q=NULL) == RA_EINVAL and att(lse=NULL) == RA_EINVAL and att(q=MIS) == RA_EINVAL
    assert att(lse=MIS4) == RA_EINVAL
    for bad in (dict(T=0), dict(R=0), dict(Hq=0), dict(Hkv=0), dict(mp=0), dict(max_new=0), dict(kv=7), dict(kv=1)):
        assert att(**bad) == RA_EINVAL, bad
    assert att(cu=NULL, T=3) == RA_EINVAL and att(cu=NULL, max_new=2) == RA_EINVAL
    assert att(ws=MIS, wsb=1 << 30) == RA_EINVAL
    for bad in (dict(D=32), dict(max_new=33), dict(Hq=9), dict(R=4097, T=5000), dict(page=3), dict(mp=1 << 27)):
        assert att(**bad) == RA_EUNSUPPORTED, bad
    n = ctypes.c_size_t(0)
    assert lib.paged_attn_workspace(4, 8, 2, 64, 1, NULL) == RA_EINVAL
    assert lib.paged_attn_workspace(4, 8, 3, 64, 1, ctypes.byref(n)) == RA_EUNSUPPORTED
    assert lib.paged_attn_workspace(0, 8, 2, 64, 1, ctypes.byref(n)) == RA_EINVAL


def test_mx4_refusals(lib):
    assert lib.mx4_pack(NULL, P, P, 64, 64, NULL) == RA_EINVAL
    assert lib.mx4_pack(P, P, P, 0, 64, NULL) == RA_EINVAL
    assert lib.mx4_pack(P, P, P, 48, 64, NULL) == RA_EUNSUPPORTED
    assert lib.mx4_pack(P, P, P, 1 << 16, 1 << 15, NULL) == RA_EUNSUPPORTED
    f = lib.mx4_linear
    assert f(P, P, P, NULL, NULL, 1, 64, 64, NULL) == RA_EINVAL
    assert f(P, MIS, P, NULL, P2, 1, 64, 64, NULL) == RA_EINVAL
    assert f(P, P, MIS4, NULL, P2, 1, 64, 64, NULL) == RA_EINVAL
    assert f(P, P, P, NULL, P2, 0, 64, 64, NULL) == RA_EINVAL
    assert f(P, P, P, NULL, P2, 1, 33, 64, NULL) == RA_EUNSUPPORTED
    assert f(P, P, P, NULL, P2, 513, 64, 64, NULL) == RA_EUNSUPPORTED
    assert b"512" in lib.ring_attn_last_error()


def test_binding_checks_tensors_before_calling():
    bf = torch.bfloat16
    with pytest.raises(ValueError):  # not on the GPU
        ra._arg(torch.zeros(3, dtype=bf), "x", bf, 0, (3,))
    with pytest.raises(ValueError):
        ra._cache(torch.zeros(2, 4, 8), torch.zeros(2, 4, 8), None, None, 0)
    with pytest.raises(TypeError):
        ra._cache(torch.zeros(2, 4, 1, 64), torch.zeros(2, 4, 1, 64), None, None, 0)
    with pytest.raises(ValueError):
        ra._rows(torch.zeros(2, 1, 64, dtype=bf), "q", 2, 1, 64, 0)
    with pytest.raises(ValueError):
        ra._rows(torch.zeros(2, 1, 64, dtype=bf), "q", 3, 1, 64, 0)
    with pytest.raises(ValueError):
        ra._rows(torch.zeros(2, 64, 2, dtype=bf).transpose(1, 2), "q", 2, 2, 64, 0)


def test_outputs_over_inputs_and_far_rows(lib):
    assert lib.mx4_pack(P, P2, P3, 1 << 29, 1, NULL) == RA_EUNSUPPORTED
    assert lib.mx4_linear(P, P2, P3, NULL, P, 1, 64, 64, NULL) == RA_EINVAL
    assert b"y must not be x" in lib.ring_attn_last_error()
    with pytest.raises(ValueError, match="apart"):
        ra._rows(torch.empty((2, 1, 64), dtype=torch.bfloat16, device="meta").as_strided((2, 1, 64), (1 << 31, 64, 1)),
                 "q", 2, 1, 64, -1)
