"""What paged_attn_decode allocates where the caller gives no workspace: nothing for short requests,
which one launch does, and for others no more than the waves of their type need."""
import pytest
import torch

import paper_2310_01889_amd as ra
from tests.gpu_util import log
from tests.test_gpu_paged_attention import call, make

pytestmark = pytest.mark.gpu


def _taken(s, max_new):
    """Bytes of device memory that a call leaves with the library."""
    workspace = torch.empty(ra.paged_attn_workspace(s["lens"].numel(), 8, 1, 128, max_new), dtype=torch.uint8, device="cuda")
    call(s, max_new, workspace=workspace)  # what the runtime allocates for a kernel's first launch
    call(s, max_new)
    ra.release_workspace()
    out = [torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")]
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    ra.paged_attn_decode(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"], *out, max_new, s["ks"], s["vs"])
    torch.cuda.synchronize()
    taken = free - torch.cuda.mem_get_info()[0]
    ra.release_workspace()
    return taken


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("lens", [[30, 9], [300, 70, 411]])  # one wave a group; four
def test_short_requests_take_no_workspace(lens, e4m3):
    s = make(95, lens, [4] * len(lens), 8, 1, 128, 16, e4m3)
    taken = _taken(s, 4)
    log("  %d bytes" % taken)
    assert taken <= 0


@pytest.mark.parametrize("e4m3", [False, True])
def test_others_take_what_their_waves_need(e4m3):
    """32 query slots of 128 + 2 floats, two sets a wave, and an entry of 24 bytes; 1024 waves for bf16
    pages and 1792 for 8 bits, sizes rounded up by an eighth and to the driver's 2 MiB."""
    s = make(96, [5000, 70], [4, 4], 8, 1, 128, 16, e4m3)
    taken, bytes_ = _taken(s, 4), (1792 if e4m3 else 1024) * (2 * 32 * 130 * 4 + 24)
    log("  %d bytes of %d" % (taken, bytes_))
    assert 0 < taken <= bytes_ * 9 // 8 + (4 << 20)
