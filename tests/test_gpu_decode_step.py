"""The serving operators together, as a program uses them: an attention block of a LLaMA-style layer
decodes a batch of requests over a paged cache, step after step (prompts first, then a token or a
few each), with RMSNorm, 4-bit projections, the page plan, the append and the attention; against
the fp64 oracle working on what each call was given, and against ring_attn_decode, and captured in
a HIP graph.

Tolerances: each call's own (see its tests), its inputs being taken as the previous call left
them."""
import math

import numpy as np
import pytest
import torch

import paper_2310_01889_amd as ra
from oracle import llama as OL
from oracle import serving as OS
from tests.gpu_util import log, np64
from tests.test_gpu_paged_attention import E4M3

pytestmark = pytest.mark.gpu

DM, HQ, HKV, D, PAGE = 512, 8, 2, 64, 16


class Step:
    """A program's weights, cache and buffers."""

    def __init__(self, R, T, max_len, e4m3, seed=0):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g)
        self.R, self.T, self.cols = R, T, -(-max_len // PAGE)
        self.gain = (1 + 0.1 * rnd(DM)).to(torch.bfloat16).cuda()
        w_qkv = (rnd(DM, (HQ + 2 * HKV) * D) / math.sqrt(DM)).to(torch.bfloat16)
        w_o = (rnd(HQ * D, DM) / math.sqrt(HQ * D)).to(torch.bfloat16)
        self.w_qkv, self.w_o = ra.mx4_weights(w_qkv.cuda()), ra.mx4_weights(w_o.cuda())
        self.n_pages = R * self.cols + 1
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        shape = (self.n_pages, PAGE, HKV, D)
        if e4m3:
            self.cache = [torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
            self.scales = [torch.full(shape[:3], 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
        else:
            self.cache = [torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            self.scales = [None, None]
        self.free = torch.randperm(self.n_pages, generator=g).to(torch.int32).cuda()
        self.table = torch.full((R, self.cols), -1, dtype=torch.int32, device="cuda")
        self.lens, self.lens2, self.head, self.counts = i32(R), i32(R), i32(1), i32(4)
        self.n_new, self.cu, self.slots, self.pos = i32(R), i32(R + 1), i32(T), i32(T)
        bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
        self.x, self.n1, self.qkv = bf(T, DM), bf(T, DM), bf(T, (HQ + 2 * HKV) * D)
        self.q, self.o, self.z = bf(T, HQ, D), bf(T, HQ, D), bf(T, DM)
        self.lse = torch.zeros(T, HQ, device="cuda")
        self.ws = torch.zeros(ra.paged_attn_workspace(R, HQ, HKV, D, 32), dtype=torch.uint8, device="cuda")

    def launch(self):
        ra.rms_norm_fwd(self.x, self.gain, self.n1)
        ra.mx4_linear(self.n1, *self.w_qkv, None, self.qkv)
        ra.paged_plan(self.lens, self.n_new, self.free, self.head, self.table, self.cu, self.lens2, self.slots, self.pos,
                      self.counts, PAGE, self.n_pages)
        h = self.qkv.view(self.T, HQ + 2 * HKV, D)
        ra.paged_append(h[:, :HQ], h[:, HQ:HQ + HKV], h[:, HQ + HKV:], self.q, *self.cache, self.slots, self.pos,
                        *self.scales)
        ra.paged_attn_decode(self.q, *self.cache, self.table, self.lens2, self.cu, self.o, self.lse, 32, *self.scales,
                             workspace=self.ws)
        ra.mx4_linear(self.o.view(self.T, HQ * D), *self.w_o, self.x, self.z)

    def advance(self):
        self.lens.copy_(self.lens2)
        self.head.copy_(self.counts[2:3])


@pytest.mark.parametrize("e4m3", [False, True])
def test_steps_against_the_oracle(e4m3):
    R, T = 5, 70
    s = Step(R, T, 200, e4m3)
    rng, g = np.random.default_rng(1), torch.Generator().manual_seed(1)
    table, lens, head = np.full((R, s.cols), -1), np.zeros(R, int), 0
    wq, wo = (OS.mx4_values(w[0].cpu().numpy(), w[1].cpu().numpy(), k, n)
              for w, k, n in ((s.w_qkv, DM, (HQ + 2 * HKV) * D), (s.w_o, HQ * D, DM)))
    for step, n_new in enumerate([[17, 0, 32, 1, 5], [16, 1, 1, 1, 8], [1] * 5, [0, 3, 30, 2, 32], [1, 1, 0, 1, 1]]):
        log("step %d: %s" % (step, n_new))
        s.x.copy_(torch.randn(T, DM, generator=g))
        s.n_new.copy_(torch.tensor(n_new, dtype=torch.int32))
        s.launch()
        torch.cuda.synchronize()
        table, cu, lens2, slots, pos, counts = OS.plan(lens, n_new, s.free.cpu().numpy(), head, table, PAGE, s.n_pages, T)
        for got, want in ((s.table, table), (s.cu, cu), (s.lens2, lens2), (s.slots, slots), (s.pos, pos), (s.counts, counts)):
            assert np.array_equal(got.cpu().numpy(), want)
        assert counts[3] == 0
        rows = cu[-1]
        n1 = np64(s.n1)
        ref = OL.rmsnorm_fwd(np64(s.x), np64(s.gain))[0]
        assert (np.abs(n1 - ref) <= 2.0 ** -8 * 1.01 * np.abs(ref) + 1e-6).all()
        qkv = np64(s.qkv)
        assert (np.abs(qkv - n1 @ wq) <= 2.0 ** -8 * np.abs(n1 @ wq) + (DM + 1) * 2.0 ** -24 * (np.abs(n1) @ np.abs(wq))).all()
        h = qkv.reshape(T, HQ + 2 * HKV, D)
        q_ref = OS.rope(h[:rows, :HQ], pos[:rows])
        assert (np.abs(np64(s.q)[:rows] - q_ref) <= 2.0 ** -8 * np.abs(q_ref) + 1e-4).all()
        cache = [OS.cached(np64(c.cpu()), None if sc is None else sc.cpu().numpy()) for c, sc in zip(s.cache, s.scales)]
        k_ref = OS.rope(h[:rows, HQ:HQ + HKV], pos[:rows])
        for c, ref in zip(cache, (k_ref, h[:rows, HQ + HKV:])):
            got = c.reshape(-1, HKV, D)[slots[:rows]]
            top = np.abs(ref).max(-1, keepdims=True)
            tol = 2.0 ** -4 * np.abs(ref) + 2.0 ** -10 * top / 224 if e4m3 else 2.0 ** -8 * np.abs(ref)
            assert (np.abs(got - ref) <= tol + 1e-4).all()
        o, lse, mag = OS.attention(np64(s.q), *cache, table, lens2, cu)
        o, lse, mag = o[:rows], lse[:rows], mag[:rows]
        assert (np.abs(np64(s.o)[:rows] - o) <= 2.0 ** -8 * 1.01 * (np.abs(o) + mag) + 1e-4 * mag).all()
        assert np.abs(np64(s.lse)[:rows] - lse).max() <= 1e-4
        ov, x = np64(s.o).reshape(T, HQ * D), np64(s.x)
        z = x + ov @ wo
        assert (np.abs(np64(s.z) - z) <= 2.0 ** -8 * np.abs(z) + (HQ * D + 2) * 2.0 ** -24 * (np.abs(x) + np.abs(ov) @ np.abs(wo))).all()
        s.advance()
        lens, head = lens2, counts[2]


def test_paged_and_contiguous_decode_agree():
    """The same cache through ring_attn_decode (one head of keys a query head, one length)."""
    B, S, H, Tq = 2, 1024, 4, 5
    g = torch.Generator().manual_seed(7)
    q, k, v = (torch.randn(B, n, H, 128, generator=g).to(torch.bfloat16).cuda() for n in (Tq, S, S))
    o, lse = ra.attention_decode(q, k, v, 4, True)
    page = 32
    ids = torch.randperm(B * S // page, generator=g).to(torch.int32)
    kp, vp = (torch.empty(B * S // page, page, H, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kp[ids.long().cuda()], vp[ids.long().cuda()] = k.view(-1, page, H, 128), v.view(-1, page, H, 128)
    table = ids.view(B, -1).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    op, lp = ra.paged_attention(q.view(B * Tq, H, 128), kp, vp, table, i32([S, S]), i32([0, Tq, 2 * Tq]), Tq)
    torch.cuda.synchronize()
    # both within 2^-8 (|o| + mean |v|) of the exact result; mean |v| below 1
    assert (op.view_as(o).float() - o.float()).abs().max() <= 2 * 2.0 ** -8 * (o.float().abs().max() + 1)
    # ring_attn_decode may sum probabilities rounded to bf16 in its denominator, each off by up to
    # 2^-8 of itself, so the sum by 2^-8 of it and its logarithm by -ln(1 - 2^-8) < 2^-8 + 2^-16;
    # float32 sums of 1024 terms (1024 x 2^-24 < 1e-4) on both sides
    assert (lp.view(B, Tq, H).permute(0, 2, 1) - lse).abs().max() <= 2.0 ** -8 + 2.0 ** -16 + 2e-4


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_captured_step_replays_as_the_eager_one(e4m3):
    """Six steps of one captured graph, eager work and synchronisation between, against the same
    steps run eagerly by a second program: every buffer equal, bit for bit."""
    R, T = 9, 9
    a, b = Step(R, T, 160, e4m3), Step(R, T, 160, e4m3)
    g = torch.Generator().manual_seed(3)
    st = torch.cuda.Stream()
    for s in (a, b):
        s.lens.fill_(100)
        s.lens2.fill_(100)
        s.table.copy_(s.free[:R * 7].view(R, 7).repeat(1, 2)[:, :s.cols])
        s.table[:, 7:] = -1
        s.head.fill_(R * 7)
        for c in s.cache:
            c.copy_(torch.randn(c.shape, generator=torch.Generator().manual_seed(5)).to(c.dtype))
        for sc in s.scales:
            if sc is not None:
                sc.fill_(125)
        s.n_new.fill_(1)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        a.launch()  # a warm-up on the capture stream: the first step's outputs, written again by its replay
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        a.launch()
    for step in range(6):
        x = torch.randn(T, DM, generator=g)
        for s in (a, b):
            s.x.copy_(x)
            s.z.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        b.launch()
        torch.cuda.synchronize()
        for name in ("qkv", "q", "o", "lse", "z", "table", "cu", "lens2", "slots", "pos", "counts"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (step, name)
        for c, d in zip(a.cache, b.cache):
            assert torch.equal(c.view(torch.uint8), d.view(torch.uint8))
        assert int(b.counts[3]) == 0 and bool(torch.isfinite(b.z.float()).all())
        for s in (a, b):
            s.advance()
    log("  six steps: bit-identical")
