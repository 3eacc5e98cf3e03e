"""Performance cases of the serving operators: a decode step over a paged key/value cache.

A serving program runs, for every step of a batch of requests of different lengths,
  plan     ``paged_plan``: pages for the new tokens, row offsets, cache slots and positions
  append   ``paged_append``: rotary embedding of q and k, keys and values into their pages
  attend   ``paged_attn_decode``: the new tokens' attention over their pages
  linear   ``mx4_linear``: a projection of the few rows of a step, weights in 4 bits
``run`` computes one of them in its plain form, elementary torch operations in 32 bits, or,
where ``own`` is true, by the library's entry points.  ``exact`` gives the same outputs from
the definitions in 64 bits.  Lengths of a batch are spread evenly over their range (``work``
depends on nothing else) and dealt to the requests by the seed.
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
BF16 = torch.bfloat16
ROPE_BASE = 10000.0


# ---------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------
def _plan(name, R, page, max_len, max_new):
    c = dict(kind="plan", R=R, page=page, max_len=max_len, max_new=max_new)
    return dict(c, name=name) if name else c


def _append(name, T, Hq, Hkv, D, page, kv, fused, max_pos):
    c = dict(kind="append", T=T, Hq=Hq, Hkv=Hkv, D=D, page=page, kv=kv, fused=fused, max_pos=max_pos)
    return dict(c, name=name) if name else c


def _attend(name, R, Hq, Hkv, D, page, kv, min_len, max_len, max_new):
    c = dict(kind="attend", R=R, Hq=Hq, Hkv=Hkv, D=D, page=page, kv=kv, min_len=min_len, max_len=max_len,
             max_new=max_new)
    return dict(c, name=name) if name else c


def _linear(name, T, d_in, d_out, residual):
    c = dict(kind="linear", T=T, d_in=d_in, d_out=d_out, residual=residual)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decode step of a handful of chats: latency alone
        _plan("plan_step_8", 8, 16, 4096, 1),
        # prompts of a large batch enter the cache at once
        _plan("plan_prefill_512", 512, 64, 32768, 1024),
        # one decode step of 64 chats, grouped heads, q, k and v three parts of one projection
        _append("append_step_64", 64, 32, 8, 128, 16, "bf16", True, 16384),
        # a chunk of prompts in an 8-bit cache, an odd number of rows
        _append("append_chunk_e4m3", 4099, 32, 8, 128, 64, "e4m3", True, 131072),
        # a long prompt, one key head a query head
        _append("append_prompt_16k", 16384, 32, 32, 128, 64, "bf16", False, 16384),
        # a few short chats with 64-wide heads: latency alone
        _attend("attend_short", 6, 16, 16, 64, 16, "bf16", 1, 301, 1),
        # an ordinary batch, lengths from nothing to 8192, grouped heads
        _attend("attend_batch_64", 64, 32, 8, 128, 16, "bf16", 0, 8192, 1),
        # up to eight drafted tokens a request checked at once, 8-bit cache
        _attend("attend_draft_e4m3", 24, 32, 8, 128, 64, "e4m3", 700, 16001, 8),
        # one very long context, one key head a query head
        _attend("attend_262k", 1, 32, 32, 128, 64, "bf16", 262144, 262144, 1),
        # the attention's projections for one token
        _linear("linear_1x4096x4096", 1, 4096, 4096, False),
        # a feed-forward product for a few tokens
        _linear("linear_7x4096x11008", 7, 4096, 11008, False),
        # and back, for the rows of a larger batch, added to the residual
        _linear("linear_48x11008x4096", 48, 11008, 4096, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "append", "attend", "attend", "attend", "linear", "linear"])
    page = rng.choice([8, 16, 32, 64, 128])
    Hkv, G = rng.choice([(1, 8), (2, 8), (4, 4), (8, 4), (8, 1), (16, 1), (4, 7), (32, 1)])
    D, kv = rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "e4m3"])
    if kind == "plan":
        R = _log_int(rng, 1, 2048)
        return _plan(None, R, page, _log_int(rng, 16, 32768), _log_int(rng, 1, max(1, min(2048, (1 << 18) // R))))
    if kind == "append":
        return _append(None, _log_int(rng, 1, 8192), Hkv * G, Hkv, D, page, kv, rng.random() < 0.5,
                       _log_int(rng, 8192, 262144))
    if kind == "attend":
        R = _log_int(rng, 1, 128)
        most = min(131072, (1 << 28) // (R * Hkv * D))
        hi = _log_int(rng, 32, max(64, most))
        return _attend(None, R, Hkv * G, Hkv, D, page, kv, rng.randrange(hi + 1), hi,
                       rng.choice([1, 1, 1, 2, 4, 8, 16]))
    return _linear(None, _log_int(rng, 1, 96), 32 * _log_int(rng, 8, 344), _log_int(rng, 200, 12000),
                   rng.random() < 0.5)


def _spread(n, lo, hi):
    """n whole numbers spread evenly from lo to hi, the largest always among them."""
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _lengths(c):
    """(cache length, new tokens) of the requests, before they are dealt."""
    lens = _spread(c["R"], c.get("min_len", 0), c["max_len"])
    news = _spread(c["R"], 1, c["max_new"])
    if c["kind"] == "attend":  # the new tokens are part of the length; a request of none has none
        news = [min(a, b) for a, b in zip(lens, news)]
    return list(zip(lens, news))


# ---------------------------------------------------------------------------------------
# What a program has in hand
# ---------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _dealt(c, g):
    pairs = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
    pairs = pairs[torch.randperm(c["R"], generator=g, device="cuda")]
    return pairs[:, 0].contiguous(), pairs[:, 1].contiguous()


def _ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


def _pages(c, n_pages, g, filled):
    """k_pages, v_pages, k_scales, v_scales (None for bf16)."""
    shape = (n_pages, c["page"], c["Hkv"], c["D"])
    if c["kv"] == "bf16":
        if filled:
            return (torch.randn(shape, generator=g, device="cuda", dtype=BF16),
                    torch.randn(shape, generator=g, device="cuda", dtype=BF16), None, None)
        return tuple(torch.zeros(shape, device="cuda", dtype=BF16) for _ in range(2)) + (None, None)
    if filled:
        codes = [torch.randn(shape, generator=g, device="cuda", dtype=BF16).mul_(96).clamp_(-448, 448).to(E4M3)
                 for _ in range(2)]
        # magnitudes of a few units: 2^-8 to 2^-5 a step
        return tuple(codes) + tuple(torch.randint(119, 123, shape[:3], generator=g, device="cuda", dtype=torch.uint8)
                                    for _ in range(2))
    return (tuple(torch.zeros(shape, device="cuda", dtype=BF16).to(E4M3) for _ in range(2))
            + tuple(torch.full(shape[:3], 127, device="cuda", dtype=torch.uint8) for _ in range(2)))


def prepare(case, seed):
    c, g = case, _gen(seed)
    if c["kind"] == "plan":
        R, P = c["R"], c["page"]
        pairs = _lengths(c)
        max_pages = -(-max(a + b for a, b in pairs) // P)
        held = sum(-(-a // P) for a, b in pairs)
        need = sum(-(-(a + b) // P) for a, b in pairs) - held
        n_pages, T = held + need + 5, sum(b for _, b in pairs) + 3
        lens, n_new = _dealt(c, g)
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        have = (lens.long() + P - 1) // P
        first = torch.cumsum(have, 0) - have
        col = torch.arange(max_pages, device="cuda")
        table = order[(first[:, None] + col).clamp(max=n_pages - 1)]
        table = torch.where(col < have[:, None], table, -1).to(torch.int32).contiguous()
        return dict(c=c, lens=lens, n_new=n_new, free=order[held:].contiguous(), head=_ints(1), table=table,
                    cu=_ints(R + 1), new_lens=_ints(R), slots=_ints(T), positions=_ints(T), counts=_ints(4),
                    n_pages=n_pages)
    if c["kind"] == "append":
        T, Hq, Hkv, D, P = c["T"], c["Hq"], c["Hkv"], c["D"], c["page"]
        if c["fused"]:
            qkv = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device="cuda", dtype=BF16)
            q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        else:
            q, k, v = (torch.randn((T, h, D), generator=g, device="cuda", dtype=BF16) for h in (Hq, Hkv, Hkv))
        n_pages = -(-T // P) + 4
        page = torch.randperm(n_pages, generator=g, device="cuda")
        i = torch.arange(T, device="cuda")
        start = torch.randint(0, max(1, c["max_pos"] - T + 1), (1,), generator=g, device="cuda")
        kp, vp, ks, vs = _pages(c, n_pages, g, False)
        return dict(c=c, q=q, k=k, v=v, slots=(page[i // P] * P + i % P).to(torch.int32),
                    positions=((start + i) % c["max_pos"]).to(torch.int32),
                    q_out=torch.zeros((T, Hq, D), device="cuda", dtype=BF16), kp=kp, vp=vp, ks=ks, vs=vs)
    if c["kind"] == "attend":
        P = c["page"]
        pairs = _lengths(c)
        n_pages = sum(-(-a // P) for a, _ in pairs) + 3
        max_pages = -(-c["max_len"] // P) + 1
        T = sum(b for _, b in pairs)
        lens, n_new = _dealt(c, g)
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        have = (lens.long() + P - 1) // P
        first = torch.cumsum(have, 0) - have
        col = torch.arange(max_pages, device="cuda")
        table = torch.where(col < have[:, None], order[(first[:, None] + col).clamp(max=n_pages - 1)], -1)
        kp, vp, ks, vs = _pages(c, n_pages, g, True)
        cu = _ints(c["R"] + 1)
        cu[1:] = torch.cumsum(n_new, 0)
        s = dict(c=c, q=torch.randn((T, c["Hq"], c["D"]), generator=g, device="cuda", dtype=BF16), kp=kp, vp=vp, ks=ks,
                 vs=vs, table=table.to(torch.int32).contiguous(), lens=lens, cu=cu)
        s["o"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros((T, c["Hq"]), device="cuda")
        return s
    T, K, N = c["T"], c["d_in"], c["d_out"]
    nb, kb = -(-N // 16), -(-K // 128)
    s = dict(c=c, x=torch.randn((T, K), generator=g, device="cuda", dtype=BF16),
             w4=torch.randint(0, 256, (nb, kb, 64, 16), generator=g, device="cuda", dtype=torch.uint8),
             ws=torch.randint(118, 122, (nb, kb, 16, 4), generator=g, device="cuda", dtype=torch.uint8),
             res=torch.randn((T, N), generator=g, device="cuda", dtype=BF16) if c["residual"] else None,
             y=torch.zeros((T, N), device="cuda", dtype=BF16))
    # blocks past the ends of the product hold no weights: zeros
    s["w4"].view(nb, kb, 4, 16, 4, 4)[:, -1, :, :, (K - 128 * (kb - 1)) // 32:] = 0
    if N % 16:
        s["w4"].view(nb, kb, 4, 16, 16)[-1, :, :, N % 16:] = 0
    return s


# ---------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------
def run(state):
    return _RUN[state["c"]["kind"]](state)


def _run_plan(s):
    c = s["c"]
    if own:
        import paper_2310_01889_amd as ra
        ra.paged_plan(s["lens"], s["n_new"], s["free"], s["head"], s["table"], s["cu"], s["new_lens"], s["slots"],
                      s["positions"], s["counts"], c["page"], s["n_pages"])
        return [s[k] for k in ("table", "cu", "new_lens", "slots", "positions", "counts")]
    P, T, i32 = c["page"], s["slots"].shape[0], torch.int32
    lens, n_new, table, free = s["lens"].long(), s["n_new"].long(), s["table"], s["free"]
    have = (lens + P - 1) // P
    need = (lens + n_new + P - 1) // P - have
    cu = torch.cat([torch.zeros_like(n_new[:1]), torch.cumsum(n_new, 0)])
    taken = torch.cumsum(need, 0)
    first = taken - need + s["head"]
    col = torch.arange(table.shape[1], device=table.device)
    nth = col - have[:, None]
    fresh = (nth >= 0) & (nth < need[:, None])
    at = first[:, None] + nth
    page = torch.where(at < free.shape[0], free[at.clamp(0, free.shape[0] - 1)], -1)
    table = torch.where(fresh, page, table)
    i = torch.arange(T, device=table.device)
    r = (torch.searchsorted(cu, i, right=True) - 1).clamp(max=c["R"] - 1)
    real = i < cu[-1]
    pos = torch.where(real, lens[r] + i - cu[r], -1)
    entry = table[r, pos.clamp(min=0) // P]
    slots = torch.where(real & (entry >= 0), entry * P + pos % P, -1)
    short = (s["head"] + taken[-1:] > free.shape[0]).long()
    took = torch.minimum(taken[-1:], free.shape[0] - s["head"])
    counts = torch.cat([cu[-1:], took, s["head"] + took, short])
    return [table, cu.to(i32), (lens + n_new).to(i32), slots.to(i32), pos.to(i32), counts.to(i32)]


def _run_append(s):
    c = s["c"]
    if own:
        import paper_2310_01889_amd as ra
        ra.paged_append(s["q"], s["k"], s["v"], s["q_out"], s["kp"], s["vp"], s["slots"], s["positions"], s["ks"],
                        s["vs"])
        return [s["q_out"], s["kp"], s["vp"]] + _scale_values(s)
    D = c["D"]
    freq = ROPE_BASE ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
    angle = s["positions"].double()[:, None] * freq
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def rotated(x):
        a, b = x[..., 0::2].float(), x[..., 1::2].float()
        return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)

    slots = s["slots"].long()
    for x, pages, scales in ((rotated(s["k"]), s["kp"], s["ks"]), (s["v"].float(), s["vp"], s["vs"])):
        if scales is not None:
            m, e = torch.frexp(x.abs().amax(-1))
            e = torch.where(m > 0, e - 9 + (m > 0.875), 0).clamp(min=-126)
            x = torch.ldexp(x, -e[..., None])
            scales.view(-1, c["Hkv"])[slots] = (e + 127).to(torch.uint8)
            pages.view(torch.uint8).view(-1, c["Hkv"], D)[slots] = x.to(E4M3).view(torch.uint8)
        else:
            pages.view(-1, c["Hkv"], D)[slots] = x.to(BF16)
    return [rotated(s["q"]).to(BF16), s["kp"], s["vp"]] + _scale_values(s)


def _scale_values(s):
    """The powers of two that the scales' bytes stand for."""
    return [] if s["ks"] is None else [s[k].view(torch.float8_e8m0fnu) for k in ("ks", "vs")]


def _run_attend(s):
    c = s["c"]
    if own:
        import paper_2310_01889_amd as ra
        ra.paged_attn_decode(s["q"], s["kp"], s["vp"], s["table"], s["lens"], s["cu"], s["o"], s["lse"], c["max_new"],
                             s["ks"], s["vs"])
        return [s["o"], s["lse"]]
    R, Hq, Hkv, D, n = c["R"], c["Hq"], c["Hkv"], c["D"], c["max_new"]
    G, T = Hq // Hkv, s["q"].shape[0]
    table = s["table"].long().clamp(min=0)
    S = table.shape[1] * c["page"]

    def cached(pages, scales):  # [R, Hkv, S, D]
        x = pages[table].float() if scales is None else pages.view(torch.uint8)[table].view(E4M3).float()
        if scales is not None:
            x = x * torch.exp2(scales[table].float() - 127)[..., None]
        return x.view(R, S, Hkv, D).transpose(1, 2)

    cu, lens = s["cu"].long(), s["lens"].long()
    t = torch.arange(n, device="cuda")
    q = s["q"].float()[(cu[:-1, None] + t).clamp(max=T - 1)]  # [R, n, Hq, D]
    q = q.view(R, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(R, Hkv, n * G, D)
    x = (q @ cached(s["kp"], s["ks"]).transpose(2, 3)).view(R, Hkv, n, G, S) * (1.0 / math.sqrt(D))
    pos = lens[:, None] - (cu[1:] - cu[:-1])[:, None] + t  # [R, n]
    key = torch.arange(S, device="cuda")
    seen = ((key <= pos[..., None]) & (key < lens[:, None, None]))[:, None, :, None]
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    v = torch.where((key < lens[:, None])[:, None, :, None], cached(s["vp"], s["vs"]), 0)
    o = (p.view(R, Hkv, n * G, S) @ v).view(R, Hkv, n, G, D) / total.clamp(min=1e-30)
    lse = (top + torch.log(total))[..., 0]
    i = torch.arange(T, device="cuda")
    r = (torch.searchsorted(cu, i, right=True) - 1).clamp(max=R - 1)
    at = (i - cu[r]).clamp(0, n - 1)
    return [o.permute(0, 2, 1, 3, 4).reshape(R, n, Hq, D)[r, at].to(BF16),
            lse.permute(0, 2, 1, 3).reshape(R, n, Hq)[r, at]]


def _run_linear(s):
    c = s["c"]
    if own:
        import paper_2310_01889_amd as ra
        ra.mx4_linear(s["x"], s["w4"], s["ws"], s["res"], s["y"])
        return [s["y"]]
    nb, kb = s["w4"].shape[:2]
    codes = torch.stack([s["w4"] & 15, s["w4"] >> 4], -1).view(nb, kb, 4, 16, 4, 4, 2)
    codes = codes.permute(0, 3, 1, 4, 2, 5, 6).reshape(nb * 16, kb * 4, 32).int()
    values = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    scale = torch.exp2(s["ws"].float() - 127).permute(0, 2, 1, 3).reshape(nb * 16, kb * 4, 1)
    w = (values[codes] * scale).view(nb * 16, kb * 128)[:c["d_out"], :c["d_in"]]
    y = s["x"].float() @ w.t()
    return [(y + s["res"].float() if c["residual"] else y).to(BF16)]


_RUN = dict(plan=_run_plan, append=_run_append, attend=_run_attend, linear=_run_linear)


# ---------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "plan":
        pairs, P = _lengths(c), c["page"]
        need = sum(-(-(a + b) // P) - -(-a // P) for a, b in pairs)
        rows = sum(b for _, b in pairs)
        # lengths in and out, offsets, pages from the list to the table, an entry held before, slots, positions
        return dict(bytes=4 * (4 * c["R"] + 2 * need + c["R"] + 2 * rows), flops=0)
    if c["kind"] == "append":
        row_in, kv = (c["Hq"] + 2 * c["Hkv"]) * c["D"] * 2, 2 * c["Hkv"] * c["D"]
        out = c["Hq"] * c["D"] * 2 + (2 * kv if c["kv"] == "bf16" else kv + 2 * c["Hkv"])
        return dict(bytes=c["T"] * (row_in + out + 8), flops=3 * c["T"] * (c["Hq"] + c["Hkv"]) * c["D"])
    if c["kind"] == "attend":
        pairs = _lengths(c)
        token = 2 * c["Hkv"] * (2 * c["D"] if c["kv"] == "bf16" else c["D"] + 1)
        rows = sum(b for _, b in pairs)
        pages = sum(-(-a // c["page"]) for a, _ in pairs)
        return dict(bytes=sum(a for a, _ in pairs) * token + rows * c["Hq"] * (4 * c["D"] + 4) + 4 * pages,
                    flops=4 * c["Hq"] * c["D"] * sum(b * a - b * (b - 1) // 2 for a, b in pairs))
    T, K, N = c["T"], c["d_in"], c["d_out"]
    rows = 2 * T * K + 2 * T * N * (2 if c["residual"] else 1)
    return dict(bytes=K * N // 2 + K * N // 32 + rows, flops=2 * T * K * N)


# ---------------------------------------------------------------------------------------
# The same outputs from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["kind"]](s)


def _exact_plan(s):
    """Request by request and token by token, as an allocator would."""
    P, table, free = s["c"]["page"], s["table"].tolist(), s["free"].tolist()
    cu, after, slots, positions, taken = [0], [], [], [], s["head"].item()
    for r, (n, m) in enumerate(zip(s["lens"].tolist(), s["n_new"].tolist())):
        for pos in range(n, n + m):
            if pos % P == 0:
                table[r][pos // P] = free[taken]
                taken += 1
            slots.append(table[r][pos // P] * P + pos % P)
            positions.append(pos)
        cu.append(cu[-1] + m)
        after.append(n + m)
    rest = [-1] * (s["slots"].shape[0] - cu[-1])
    counts = [cu[-1], taken - s["head"].item(), taken, 0]
    return [torch.tensor(x) for x in (table, cu, after, slots + rest, positions + rest, counts)]


def _exact_append(s):
    c = s["c"]
    D, slots = c["D"], s["slots"].long()
    freq = torch.exp(torch.arange(D // 2, device="cuda").double() * (-2 * math.log(ROPE_BASE) / D))
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(s["positions"].double(), freq))

    def spun(x):
        z = torch.view_as_complex(x.double().reshape(x.shape[0], x.shape[1], D // 2, 2).contiguous())
        return torch.view_as_real(z * turn[:, None]).reshape(x.shape)

    out = [spun(s["q"])]
    if c["kv"] != "bf16":
        return out + [None] * 4  # what the 8 bits hold
    for x, pages in ((spun(s["k"]), s["kp"]), (s["v"].double(), s["vp"])):
        full = pages.double().view(-1, c["Hkv"], D)
        full[slots] = x
        out.append(full.view(pages.shape))
    return out


def _exact_attend(s):
    c = s["c"]
    D, Hkv, G = c["D"], c["Hkv"], c["Hq"] // c["Hkv"]
    if (c["R"] + s["q"].shape[0]) * Hkv > 16000:
        return [None, None]  # one row of one head at a time: too long
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    lens, cu, table = s["lens"].tolist(), s["cu"].tolist(), s["table"].long()
    for r, n in enumerate(lens):
        rows = range(cu[r], cu[r + 1])
        if not rows:
            continue
        ids = table[r, :-(-n // c["page"])]
        for h in range(Hkv):
            k, v = (p[ids, :, h].double().reshape(-1, D)[:n] if sc is None else
                    p.view(torch.uint8)[ids, :, h].view(E4M3).double().reshape(-1, D)[:n]
                    * 2.0 ** (sc[ids, :, h].double().reshape(-1, 1)[:n] - 127)
                    for p, sc in ((s["kp"], s["ks"]), (s["vp"], s["vs"])))
            for i in rows:
                m = n - (cu[r + 1] - 1 - i)  # keys up to the row's own
                hs = slice(h * G, (h + 1) * G)
                x = s["q"][i, hs].double() @ k[:m].t() / math.sqrt(D)
                lse[i, hs] = torch.logsumexp(x, -1)
                o[i, hs] = torch.exp(x - lse[i, hs, None]) @ v[:m]
    return [o, lse]


def _exact_linear(s):
    c = s["c"]
    n = torch.arange(c["d_out"], device="cuda")[:, None]
    k = torch.arange(c["d_in"], device="cuda")[None]
    kb = s["w4"].shape[1]
    block, lane = n // 16 * kb + k // 128, k // 8 % 4 * 16 + n % 16
    byte = s["w4"].flatten()[(block * 64 + lane) * 16 + k // 32 % 4 * 4 + k // 2 % 4]
    code = torch.where(k % 2 == 1, byte >> 4, byte & 15).double()
    sign, m = torch.where(code >= 8, -1.0, 1.0), code % 8
    e = torch.floor(m / 2)
    w = sign * torch.where(m < 2, m / 2, (1 + m % 2 / 2) * 2.0 ** (e - 1))
    w = w * 2.0 ** (s["ws"].flatten()[(block * 16 + n % 16) * 4 + k // 32 % 4].double() - 127)
    y = s["x"].double() @ w.t()
    return [y + s["res"].double() if c["residual"] else y]


_EXACT = dict(plan=_exact_plan, append=_exact_append, attend=_exact_attend, linear=_exact_linear)
