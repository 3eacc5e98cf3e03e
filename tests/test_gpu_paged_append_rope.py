"""paged_append rotates as rope_apply does: the same bits.

Both form angles in double and round sine and cosine to float32 once, so they differ only where the
two angles' last bits (10^-16 of up to 10^6 radians) lie on both sides of a float32 border, one in a
thousand at the farthest positions here, and an output only where that last bit of float32 crosses a
border of bf16, one in 2^15 of those: less than one in a hundred runs over other inputs would show a
differing element.  Sines good to 22 bits alone show seven to twenty-three each."""
import pytest
import torch

import paper_2310_01889_amd as ra
from tests.gpu_util import log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pos0", [0, 70001, 1000003])
def test_append_is_rope_apply(D, pos0):
    T, Hq, Hkv, page = 512, 4, 2, 16
    g = torch.Generator().manual_seed(D + pos0)
    q, k, v = (torch.randn(T, h, D, generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))
    kp, vp = (torch.zeros(T // page, page, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots = torch.arange(T, dtype=torch.int32, device="cuda")
    q_out = torch.empty_like(q)
    ra.paged_append(q, k, v, q_out, kp, vp, slots, slots + pos0)
    want_q, want_k = q.clone(), k.clone()
    ra.rope_apply(want_q, pos0)
    ra.rope_apply(want_k, pos0)
    torch.cuda.synchronize()
    differ = int((q_out != want_q).sum()) + int((kp.view(T, Hkv, D) != want_k).sum())
    log("  D=%d from position %d: %d of %d elements differ" % (D, pos0, differ, T * (Hq + Hkv) * D))
    assert differ == 0
    assert torch.equal(vp.view(T, Hkv, D), v)
