"""What is measured: the operators that serve a batch of unequal requests over a paged K/V cache with a
shared prefix, through the library's public entry points.

Four operators make up such a step: the plan (block tables, slots and positions from the requests'
lengths), the norm of queries and keys with the position rotation (K and V written to their slots), the
attention over the shared prefix and each request's own pages, and the processing of the logits
(penalties, biases, grammar masks) with the decision taken from them.

`run` computes an operator in plain torch where `own` is false, and calls the library where it is true.
Lengths are part of a case (`mix` seeds them), so that its work is known; the values, the order of the
pages and the token ids come from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

# (query heads, K/V heads, head dim) of this repository's configurations and tests
SHAPES = {"llada": (32, 32, 128), "dream": (28, 4, 128), "tiny": (4, 4, 64), "small": (16, 4, 64)}
VOCAB = {"llada": 126464, "dream": 152064, "tiny": 1024}
THETA = {"llada": 500000.0, "dream": 1000000.0, "tiny": 10000.0, "small": 10000.0}
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-5
MASKED = float("-inf")


def listed():
    return [
        # A step's plan for 16 requests with windows of 32 tokens: launch latency and nothing else.
        _plan("plan_windows", "llada", B=16, q=(32, 32), own=(0, 900), page=64, mix=1),
        # Continuous batching: prompts and single tokens of a thousand requests in small pages, a
        # third of which end and make room for others at every step.
        _plan("plan_prompts", "dream", B=1000, q=(1, 700), own=(0, 3000), page=16, mix=2),
        # One 32-token window straight from the fp32 output of the projection.
        _norm("norm_window", "llada", N=32, dtype="bf16", src="f32", page=64, pos=600),
        # An odd number of rows, grouped heads, in f16, far into a long context.
        _norm("norm_f16", "dream", N=1201, dtype="f16", src="f16", page=16, pos=100000),
        # Prompts of a whole batch: bandwidth.
        _norm("norm_prompts", "llada", N=16384, dtype="bf16", src="bf16", page=64, pos=4096),
        # One request that decodes a single token after a short prefix.
        _attn("attn_one_token", "dream", B=1, q=(1, 1), own=(40, 40), P=300, page=16, mix=3),
        # Denoising windows of a batch under one long prompt.
        _attn("attn_windows", "llada", B=16, q=(32, 32), own=(0, 1000), P=4096, page=64, mix=4),
        # Single tokens of many requests, grouped heads, f16, small pages, an odd prefix.
        _attn("attn_tokens_f16", "dream", B=96, q=(1, 1), own=(1, 1500), P=8001, page=16, mix=5, dtype="f16"),
        # New prompts behind a shared prefix, causal.
        _attn("attn_prompts_causal", "dream", B=5, q=(200, 1100), own=(0, 0), P=2000, page=32, mix=6, causal=True),
        # One row of logits: latency.
        _logits("logits_one", "llada", N=1, T=1, hist=500, dtype="f32", out=True),
        # The windows of a batch, the decision alone (penalties of a request hold for its 32 rows).
        _logits("logits_windows", "llada", N=512, T=32, hist=2000, dtype="f32", out=False),
        # Single tokens of a batch with long histories in bf16, the processed logits kept.
        _logits("logits_bf16", "dream", N=96, T=1, hist=5000, dtype="bf16", out=True),
    ]


def _plan(name, shape, B, q, own, page, mix):
    return dict(name=name, kind="plan", shape=shape, B=B, q0=q[0], q1=q[1], own0=own[0], own1=own[1], page=page, mix=mix)


def _norm(name, shape, N, dtype, src, page, pos):
    return dict(name=name, kind="norm", shape=shape, N=N, dtype=dtype, src=src, page=page, pos=pos)


def _attn(name, shape, B, q, own, P, page, mix, dtype="bf16", causal=False):
    return dict(name=name, kind="attn", shape=shape, B=B, q0=q[0], q1=q[1], own0=own[0], own1=own[1], P=P, page=page,
                mix=mix, dtype=dtype, causal=causal)


def _logits(name, shape, N, T, hist, dtype, out):
    return dict(name=name, kind="logits", shape=shape, N=N, T=T, hist=hist, dtype=dtype, out=out)


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3072 else n


def _seconds(case):
    w = work(case)
    return w["bytes"] / 6.8e12 + w["flops"] / 1.9e15


def draw(rng):
    most = max(_seconds(c) for c in listed())
    while True:
        kind = rng.choice(["plan", "norm", "attn", "attn", "attn", "logits", "logits"])
        shape = rng.choice(["llada", "dream", "tiny", "small"])
        page, mix = rng.choice([16, 32, 64, 128]), rng.randrange(1 << 20)
        if kind == "plan":
            B, hi = _log(rng, 1, 2000), _log(rng, 1, 1500)
            if B * hi > 1 << 20:
                continue
            c = _plan("", shape, B, (rng.randint(0, hi), hi), (0, _log(rng, 1, 4000)), page, mix)
        elif kind == "norm":
            dtype = rng.choice(["bf16", "bf16", "f16"])
            c = _norm("", shape, _log(rng, 1, 16384), dtype, rng.choice([dtype, dtype, "f32"]), page,
                      _log(rng, 100, 200000))
        elif kind == "attn":
            form = rng.choice(["tokens", "windows", "windows", "prompts"])
            P = 0 if rng.random() < 0.1 else _log(rng, 16, 16384)
            causal = form == "prompts" and rng.random() < 0.7
            if form == "tokens":
                B, q, hi = _log(rng, 1, 256), (1, 1), _log(rng, 1, 2000)
            elif form == "windows":
                T = _log(rng, 2, 160)
                B, q, hi = max(1, min(_log(rng, 1, 64), 4096 // T)), (rng.choice([T, 1]), T), _log(rng, 1, 2000)
            else:
                B, hi = rng.randint(1, 6), _log(rng, 1, 500)
                q = (_log(rng, 1, 300), _log(rng, 300, 1200))
            c = _attn("", shape, B, q, (0, hi), P, page, mix, dtype=rng.choice(["bf16", "bf16", "f16"]), causal=causal)
            if B * q[1] * SHAPES[shape][0] * (P + hi + q[1]) > 1.5e9:  # scores of the plain form
                continue
        else:
            shape = rng.choice(["llada", "dream", "tiny"])
            T = rng.choice([1, 1, _log(rng, 2, 64)])
            N = T * _log(rng, 1, 512 // T)
            c = _logits("", shape, N, T, _log(rng, 1, 20000), rng.choice(["f32", "f32", "bf16"]), rng.random() < 0.6)
        del c["name"]
        if _seconds(c) <= most:
            return c


# ------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """(own lengths, new tokens) of the requests."""
    r = random.Random(case["mix"])
    L = [r.randint(case["own0"], case["own1"]) for _ in range(case["B"])]
    Q = [r.randint(case["q0"], case["q1"]) for _ in range(case["B"])]
    return L, Q


def _next_lengths(case):
    """The step after: what was new is cached, a third of the requests have ended and others took their place."""
    L, Q = _lengths(case)
    r = random.Random(case["mix"] + 1)
    ended = [r.random() < 1 / 3 for _ in L]
    return ([0 if e else l + q for l, q, e in zip(L, Q, ended)],
            [r.randint(case["q0"], case["q1"]) if e else min(q, 1) for q, e in zip(Q, ended)])


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pages(L, page):
    return [-(-n // page) for n in L]


def _theta(case):
    hd = SHAPES[case["shape"]][2]
    j = torch.arange(0, hd, 2, dtype=torch.float64)
    return (THETA[case["shape"]] ** (-j / hd)).to(torch.float32).cuda()


def _handle(case, B, rows, n_pages, max_pages, dtype="bf16"):
    from paper_2606_13740_gb300 import serve

    H, Hkv, hd = SHAPES[case["shape"]]
    return serve.Serve(serve.ServeConfig(max_batch=B, max_rows=max(1, rows), page=case["page"], n_pages=n_pages,
                                         max_pages=max_pages, n_heads=H, n_kv_heads=Hkv, head_dim=hd, dtype=dtype))


def prepare(case, seed):
    return {"plan": _prepare_plan, "norm": _prepare_norm, "attn": _prepare_attn, "logits": _prepare_logits}[case["kind"]](
        case, seed)


def _prepare_plan(case, seed):
    """Requests that hold the pages of their own lengths, a pool with a third to spare, pages in random order; two
    steps' lengths, which the passes take in turn."""
    steps = [_lengths(case), _next_lengths(case)]
    held = _pages(steps[0][0], case["page"])
    need = max(sum(_pages([a + b for a, b in zip(L, Q)], case["page"])) for L, Q in steps)
    n_pages = (need * 4 + 2) // 3 + sum(held) + 4
    max_pages = max(max(_pages([a + b for a, b in zip(L, Q)], case["page"])) for L, Q in steps) + 2
    rows = max(sum(Q) for _, Q in steps)
    g = _generator(seed)
    order = torch.randperm(n_pages, device="cuda", generator=g, dtype=torch.int32)
    h = _ints(held)
    first = torch.cumsum(h, 0) - h
    col = torch.arange(max_pages, device="cuda", dtype=torch.int32)[None]
    table = torch.where(col < h[:, None], order[(first[:, None] + col).clamp(max=n_pages - 1).long()], -1).to(torch.int32)
    used = int(sum(held))
    ring = torch.cat([order[used:], torch.zeros(used, device="cuda", dtype=torch.int32)]).to(torch.int32)
    s = {"case": dict(case), "turn": 0, "rows": [sum(Q) for _, Q in steps], "table": table.contiguous(), "held": h,
         "ring": ring, "ring_pos": _ints([0, n_pages - used]), "steps": [(_ints(L), _ints(Q)) for L, Q in steps],
         "prefix": 1000}
    if own:
        s["handle"] = k = _handle(case, case["B"], rows, n_pages, max_pages)
        k.table.copy_(table), k.held.copy_(h), k.ring.copy_(ring), k.ring_pos.copy_(s["ring_pos"])
    return s


def _prepare_norm(case, seed):
    """The packed output of a projection, and a cache whose slots the rows get in random order; some rows are padding."""
    H, Hkv, hd = SHAPES[case["shape"]]
    N, page = case["N"], case["page"]
    g = _generator(seed)
    qkv = torch.randn(N, (H + 2 * Hkv) * hd, device="cuda", generator=g).mul_(1.7).to(DTYPE[case["src"]])
    n_pages = -(-N // page) + 1
    slot = torch.randperm(n_pages * page, device="cuda", generator=g, dtype=torch.int32)[:N].contiguous()
    slot[torch.rand(N, device="cuda", generator=g) < 0.02] = -1
    pos = torch.randint(0, case["pos"], (N,), device="cuda", generator=g, dtype=torch.int32)
    gains = [1 + 0.1 * torch.randn(hd, device="cuda", generator=g) for _ in range(2)]
    kc, vc = (torch.zeros(n_pages, Hkv, page, hd, device="cuda", dtype=DTYPE[case["dtype"]]) for _ in range(2))
    s = {"case": dict(case), "qkv": qkv, "slot": slot, "pos": pos, "gains": gains, "theta": _theta(case), "kc": kc, "vc": vc}
    if own:
        s["handle"] = k = _handle(case, 1, N, n_pages, n_pages, case["dtype"])
        k.slot[:N].copy_(slot), k.pos[:N].copy_(pos)
    return s


def _prepare_attn(case, seed):
    """The requests' pages in random order over a full pool, and the plan of the step (made once for all its layers)."""
    H, Hkv, hd = SHAPES[case["shape"]]
    page, P, B = case["page"], case["P"], case["B"]
    L, Q = _lengths(case)
    held = _pages([a + b for a, b in zip(L, Q)], page)
    n_prefix = -(-P // page)
    n_pages, max_pages = sum(held) + n_prefix + 1, max(max(held), 1)
    g = _generator(seed)
    order = torch.randperm(n_pages, device="cuda", generator=g, dtype=torch.int32)
    h = _ints(held)
    first = torch.cumsum(h, 0) - h + n_prefix
    col = torch.arange(max_pages, device="cuda", dtype=torch.int32)[None]
    table = torch.where(col < h[:, None], order[(first[:, None] + col).clamp(max=n_pages - 1).long()], -1).to(torch.int32)
    dt = DTYPE[case["dtype"]]
    q = torch.randn(sum(Q), H, hd, device="cuda", generator=g).to(dt)
    kc, vc = (torch.randn(n_pages, Hkv, page, hd, device="cuda", generator=g).to(dt) for _ in range(2))
    s = {"case": dict(case), "q": q, "kc": kc, "vc": vc, "prefix_pages": order[:n_prefix].contiguous(),
         "table": table.contiguous(), "len": _ints(L), "q_len": _ints(Q)}
    if own:
        s["handle"] = k = _handle(case, B, sum(Q), n_pages, max_pages, case["dtype"])
        k.table.copy_(table), k.held.copy_(h), k.ring_pos.zero_()
        k.dllm_serve_plan(s["len"], s["q_len"], sum(Q), prefix_len=P, causal=case["causal"])
    return s


def _prepare_logits(case, seed):
    """Logits of random spread, Zipf histories of unequal length, a few biases a request, a third of the rows under
    a grammar that allows some of the vocabulary."""
    V, N, T = VOCAB[case["shape"]], case["N"], case["T"]
    R = N // T
    g = _generator(seed)
    z = torch.randn(N, V, device="cuda", generator=g).mul_(2.5).to(DTYPE[case["dtype"]])
    u = torch.rand(R, case["hist"], device="cuda", generator=g)
    hist = torch.exp(u * math.log(V - 1)).to(torch.int32).clamp(max=V - 2) - 1
    hist_len = torch.randint(case["hist"] // 2, case["hist"] + 1, (R,), device="cuda", generator=g, dtype=torch.int32)
    nb = 48
    grammar = torch.zeros(8, (V + 31) // 32, device="cuda", dtype=torch.int32)
    for k in range(8):  # bit v % 32 of word v / 32: id v is allowed
        bits = torch.rand(grammar.shape[1] * 32, device="cuda", generator=g) < 0.02 * (k + 1)
        w = bits.view(-1, 32).to(torch.int64) << torch.arange(32, device="cuda")
        w = w.sum(1)
        grammar[k] = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)
    row = torch.randint(0, 24, (N,), device="cuda", generator=g, dtype=torch.int32)
    return {"case": dict(case), "z": z, "hist": hist, "hist_len": hist_len, "V": V,
            "req": (torch.arange(N, device="cuda", dtype=torch.int32) // T).to(torch.int32),
            "rep": 1 + 0.3 * torch.rand(R, device="cuda", generator=g),
            "freq": 0.5 * torch.rand(R, device="cuda", generator=g),
            "pres": 0.5 * torch.rand(R, device="cuda", generator=g),
            "bias_ids": torch.randint(0, V, (R, nb), device="cuda", generator=g, dtype=torch.int32),
            "bias": 2 * torch.randn(R, nb, device="cuda", generator=g),
            "bias_len": torch.randint(0, nb + 1, (R,), device="cuda", generator=g, dtype=torch.int32),
            "grammar": grammar, "grammar_row": torch.where(row < 8, row, -1).to(torch.int32),
            "cur": torch.randint(0, V, (N,), device="cuda", generator=g, dtype=torch.int32)}


# ------------------------------------------------------------------------------------ one pass
def run(state):
    kind = state["case"]["kind"]
    if kind == "plan":
        turn, state["turn"] = state["turn"], 1 - state["turn"]  # the two steps in turn
        return (_own_plan if own else _plain_plan)(state, turn)
    if own:
        return {"norm": _own_norm, "attn": _own_attn, "logits": _own_logits}[kind](state)
    return {"norm": _plain_norm, "attn": _plain_attn, "logits": _plain_logits}[kind](state)


def _own_plan(s, turn):
    k, rows, B = s["handle"], s["rows"][turn], s["case"]["B"]
    L, Q = s["steps"][turn]
    k.dllm_serve_plan(L, Q, rows, prefix_len=s["prefix"])
    return {"table": k.table, "held": k.held, "ring": k.ring, "ring_pos": k.ring_pos, "row_start": k.row_start,
            "n_keys": k.n_keys, "slot": k.slot[:rows], "pos": k.pos[:rows], "req": k.req[:rows]}


def _plain_plan(s, turn):
    page, rows = s["case"]["page"], s["rows"][turn]
    table, held, ring, ring_pos = s["table"], s["held"], s["ring"], s["ring_pos"]
    L, Q = s["steps"][turn]
    n_pages, max_pages = ring.shape[0], table.shape[1]
    need = (L + Q + page - 1) // page
    bad = (L < 0) | (Q < 0) | (need > max_pages)
    grow = torch.where(bad, 0, (need - held).clamp(min=0))
    shrink = torch.where(bad, 0, (held - need).clamp(min=0))
    cum = torch.cumsum(grow, 0)
    head, count = ring_pos[0], ring_pos[1]
    refused = bad | ((grow > 0) & (cum > count))
    taken = torch.where(refused, 0, cum).amax()
    col = torch.arange(max_pages, device=table.device, dtype=torch.int32)[None]
    new = (col >= held[:, None]) & (col < need[:, None]) & ~refused[:, None]
    old = (col >= need[:, None]) & (col < held[:, None]) & ~bad[:, None]
    src = (head + (cum - grow)[:, None] + col - held[:, None]) % n_pages
    dst = (head + count + (torch.cumsum(shrink, 0) - shrink)[:, None] + col - need[:, None]) % n_pages
    given = ring[src.clamp(min=0).long()]
    ring[dst[old].long()] = table[old]
    table.copy_(torch.where(new, given, torch.where(old, -1, table)))
    held.copy_(torch.where(refused, held, need))
    ring_pos.copy_(torch.stack([(head + taken) % n_pages, count - taken + shrink.sum()]))
    row_start = torch.cat([torch.zeros(1, device=table.device, dtype=torch.int64), torch.cumsum(Q.clamp(min=0), 0)])
    r = torch.arange(rows, device=table.device)
    b = torch.searchsorted(row_start[1:], r, right=True).clamp(max=Q.shape[0] - 1)
    ok = (r < row_start[-1]) & ~refused[b]
    at = (L[b] + r - row_start[b]).clamp(min=0)
    slot = table[b, torch.where(ok, at // page, 0)] * page + at % page
    return {"table": table, "held": held, "ring": ring, "ring_pos": ring_pos, "row_start": row_start.to(torch.int32),
            "n_keys": torch.where(refused, 0, L + Q), "slot": torch.where(ok, slot, -1).to(torch.int32),
            "pos": torch.where(ok, s["prefix"] + at, 0).to(torch.int32),
            "req": torch.where(r < row_start[-1], b, -1).to(torch.int32)}


def _heads(s):
    H, Hkv, hd = SHAPES[s["case"]["shape"]]
    x = s["qkv"]
    return x[:, :H * hd], x[:, H * hd:(H + Hkv) * hd], x[:, (H + Hkv) * hd:], H, Hkv, hd


def _own_norm(s):
    q, k, v, _, _, _ = _heads(s)
    out = s["handle"].dllm_serve_qk_norm_rope(q, k, v, s["theta"], s["kc"], s["vc"], q_gain=s["gains"][0],
                                              k_gain=s["gains"][1], eps=EPS)
    return {"q": out, "k": s["kc"], "v": s["vc"]}


def _plain_norm(s):
    q, k, v, H, Hkv, hd = _heads(s)
    N, page, dt = s["case"]["N"], s["case"]["page"], DTYPE[s["case"]["dtype"]]
    angle = s["pos"].float()[:, None] * s["theta"]
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

    def turned(x, n, gain):
        x = x.float().reshape(N, n, hd)
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
        a, b = x[..., :hd // 2], x[..., hd // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(dt)

    live = s["slot"] >= 0
    at = s["slot"][live].long()
    s["kc"][at // page, :, at % page] = turned(k, Hkv, s["gains"][1])[live]
    s["vc"][at // page, :, at % page] = v.float().reshape(N, Hkv, hd)[live].to(dt)
    return {"q": turned(q, H, s["gains"][0]), "k": s["kc"], "v": s["vc"]}


def _own_attn(s):
    return s["handle"].dllm_serve_attention(s["q"], s["kc"], s["vc"], s["prefix_pages"])


def _plain_attn(s):
    c = s["case"]
    H, Hkv, hd = SHAPES[c["shape"]]
    B, P, G, q = c["B"], c["P"], H // Hkv, s["q"]
    L, Q = s["len"].long(), s["q_len"].long()
    N, T, K = q.shape[0], c["q1"], s["table"].shape[1] * c["page"]
    start = torch.cumsum(Q, 0) - Q
    row = torch.arange(N, device=q.device)
    req = torch.searchsorted(torch.cumsum(Q, 0), row, right=True)
    t = torch.arange(T, device=q.device)
    # queries [B][Hkv][T * G][hd], keys and values of the prefix [Hkv][P][hd] and of each request [B][Hkv][K][hd]
    x = q[(start[:, None] + t).clamp(max=N - 1)].float().view(B, T, Hkv, G, hd).permute(0, 2, 1, 3, 4)
    x = x.reshape(B, Hkv, T * G, hd) / math.sqrt(hd)
    pages, mine = s["prefix_pages"].long(), s["table"].clamp(min=0).long()
    kp, vp = (m[pages].float().transpose(0, 1).reshape(Hkv, -1, hd)[:, :P] for m in (s["kc"], s["vc"]))
    ko, vo = (m[mine].float().transpose(1, 2).reshape(B, Hkv, K, hd) for m in (s["kc"], s["vc"]))
    n_keys = L + Q
    key = torch.arange(K, device=q.device)
    vo = torch.where((key < n_keys[:, None])[:, None, :, None], vo, 0.0)
    last = n_keys[:, None] if not c["causal"] else L[:, None] + t + 1
    seen = (key < last.expand(B, T)[..., None])[:, None, :, None].expand(B, 1, T, G, K).reshape(B, 1, T * G, K)
    sp = torch.matmul(x, kp.transpose(1, 2))
    so = torch.where(seen, torch.matmul(x, ko.transpose(2, 3)), MASKED)
    m = so.amax(-1, keepdim=True)
    if P:
        m = torch.maximum(m, sp.amax(-1, keepdim=True))
    m = torch.where(m == MASKED, 0.0, m)
    sp, so = torch.exp(sp - m), torch.exp(so - m)
    total = sp.sum(-1, keepdim=True) + so.sum(-1, keepdim=True)
    o = (torch.matmul(sp, vp) + torch.matmul(so, vo)) / torch.where(total > 0, total, 1.0)
    o = o.view(B, Hkv, T, G, hd).permute(0, 2, 1, 3, 4)[req, row - start[req]]
    return o.reshape(N, H * hd).to(q.dtype)


def _own_logits(s):
    from paper_2606_13740_gb300 import serve

    out = torch.empty_like(s["z"]) if s["case"]["out"] else None
    x0, conf, tokconf = serve.dllm_serve_logits(
        s["z"], s["V"] - 1, req=s["req"], hist=s["hist"], hist_len=s["hist_len"], rep=s["rep"], freq=s["freq"],
        pres=s["pres"], bias_ids=s["bias_ids"], bias=s["bias"], bias_len=s["bias_len"], grammar=s["grammar"],
        grammar_row=s["grammar_row"], cur=s["cur"], out=out)
    return {"x0": x0, "conf": conf, "tokconf": tokconf, **({} if out is None else {"z": out})}


def _plain_logits(s):
    V, req, R = s["V"], s["req"].long(), s["hist"].shape[0]
    z = s["z"].float()
    there = torch.arange(s["hist"].shape[1], device=z.device) < s["hist_len"][:, None]
    count = torch.zeros(R, V, device=z.device).scatter_add_(1, s["hist"].long(), there.float())[req]
    rep, freq, pres = (s[k][req][:, None] for k in ("rep", "freq", "pres"))
    z = torch.where(count > 0, torch.where(z > 0, z / rep, z * rep) - (freq * count + pres), z)
    # of an id that a request's biases name twice, the last one counts
    nb = s["bias"].shape[1]
    nth = torch.arange(1, nb + 1, device=z.device)
    nth = torch.where(nth <= s["bias_len"][:, None], nth, 0)
    which = torch.zeros(R, V, device=z.device, dtype=torch.int64).scatter_reduce_(1, s["bias_ids"].long(), nth, "amax")
    bias = torch.where(which > 0, torch.gather(s["bias"], 1, (which - 1).clamp(min=0)), 0.0)
    z = torch.where(which[req] > 0, z + bias[req], z)
    ids = torch.arange(V, device=z.device)
    allowed = (s["grammar"][:, ids // 32] >> (ids % 32).to(torch.int32)) & 1 > 0
    row = s["grammar_row"].long()
    z = torch.where((row < 0)[:, None] | allowed[row.clamp(min=0)], z, MASKED)
    out = {"z": z.to(s["z"].dtype)} if s["case"]["out"] else {}
    z = torch.where(ids == V - 1, MASKED, z)  # the mask id is no answer
    top = z.amax(1, keepdim=True)
    x0 = torch.where((z == top) & (top > MASKED), ids, V).amin(1)
    e = torch.exp(z - torch.where(top > MASKED, top, 0.0))
    total = e.sum(1)
    cur = s["cur"].long()
    tok = torch.gather(e, 1, cur[:, None])[:, 0]
    some = total > 0
    return {"x0": torch.where(x0 < V, x0, -1).to(torch.int32), "conf": torch.where(some, 1 / total, 0.0),
            "tokconf": torch.where(some, tok / total, 0.0), **out}


# ------------------------------------------------------------------------------------ work
def work(case):
    if case["kind"] == "plan":
        b = 0.0
        steps = [_lengths(case), _next_lengths(case)]
        held = [_pages([x + y for x, y in zip(*s)], case["page"]) for s in steps]
        moved = sum(abs(x - y) for x, y in zip(*held))
        for L, Q in steps:  # lengths, pages held, row starts and key counts; slot, position and request of each row
            b += 24.0 * len(L) + 12.0 * sum(Q)
        return {"bytes": b / 2 + 8.0 * moved, "flops": 0.0}
    H, Hkv, hd = SHAPES[case["shape"]]
    size = {"f32": 4.0, "bf16": 2.0, "f16": 2.0}
    if case["kind"] == "norm":
        N, n = case["N"], (H + 2 * Hkv) * hd
        return {"bytes": N * n * (size[case["src"]] + size[case["dtype"]]) + 8.0 * N, "flops": 10.0 * N * (H + Hkv) * hd}
    if case["kind"] == "attn":
        L, Q = _lengths(case)
        pairs = sum(q * case["P"] + (q * l + q * (q + 1) / 2 if case["causal"] else q * (l + q)) for l, q in zip(L, Q))
        return {"bytes": 4.0 * sum(Q) * H * hd + 4.0 * (case["P"] + sum(L) + sum(Q)) * Hkv * hd, "flops": 4.0 * hd * H * pairs}
    V, N = VOCAB[case["shape"]], case["N"]
    hist = 0.75 * case["hist"] * (N // case["T"])  # histories lie between half of hist and hist
    return {"bytes": N * V * size[case["dtype"]] * (2 if case["out"] else 1) + N * V / 24.0 + 4.0 * hist, "flops": 5.0 * N * V}


# ------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """From the operators' definitions: angles, sums and softmaxes in 64 bits, request by request."""
    if case["kind"] == "plan":
        return None  # whole numbers only
    return {"norm": _exact_norm, "attn": _exact_attn, "logits": _exact_logits}[case["kind"]](case, seed)


def _exact_norm(case, seed):
    s = _prepare_norm(case, seed)
    H, Hkv, hd = SHAPES[case["shape"]]
    page = case["page"]
    qkv = s["qkv"].double().view(case["N"], H + 2 * Hkv, hd)
    turn = torch.polar(torch.ones((), device="cuda", dtype=torch.float64),
                       s["pos"].double().outer(s["theta"].double()))  # e^(i position theta)
    gain = torch.cat([s["gains"][0].double().expand(H, hd), s["gains"][1].double().expand(Hkv, hd)])
    x = qkv[:, :H + Hkv]
    x = x / (x.square().sum(-1, keepdim=True) / hd + EPS).sqrt() * gain
    w = torch.complex(x[..., :hd // 2], x[..., hd // 2:]) * turn[:, None]
    x = torch.cat([w.real, w.imag], -1)
    kc, vc = (torch.zeros(s["kc"].shape, device="cuda", dtype=torch.float64) for _ in range(2))
    rows = torch.nonzero(s["slot"] >= 0)[:, 0]
    at = s["slot"][rows].long()
    kc[at.div(page, rounding_mode="floor"), :, at.remainder(page)] = x[rows, H:]
    vc[at.div(page, rounding_mode="floor"), :, at.remainder(page)] = qkv[rows, H + Hkv:]
    return {"q": x[:, :H], "k": kc, "v": vc}


def _exact_attn(case, seed):
    s = _prepare_attn(case, seed)
    H, Hkv, hd = SHAPES[case["shape"]]
    page, P, G = case["page"], case["P"], H // Hkv
    L, Q = _lengths(case)
    if 4.0 * hd * sum(q * (P + l + q) for l, q in zip(L, Q)) * H > 6e12:
        return None
    outs, at = [], 0
    pre = s["prefix_pages"].long()
    for b, (l, q) in enumerate(zip(L, Q)):
        mine = s["table"][b, :-(-(l + q) // page)].long()
        x = s["q"][at:at + q].double()
        at += q
        ids = torch.cat([(pre[:, None] * page + torch.arange(page, device="cuda")).flatten()[:P],
                         (mine[:, None] * page + torch.arange(page, device="cuda")).flatten()[:l + q]])
        o = torch.zeros(q, H, hd, device="cuda", dtype=torch.float64)
        if len(ids) and q:
            for h in range(Hkv):
                k, v = (m[ids // page, h, ids % page].double() for m in (s["kc"], s["vc"]))
                score = torch.einsum("tgd,kd->gtk", x[:, h * G:(h + 1) * G], k) * hd ** -0.5
                if case["causal"]:
                    ahead = torch.arange(len(ids), device="cuda")[None] - (P + l) > torch.arange(q, device="cuda")[:, None]
                    score.masked_fill_(ahead, MASKED)
                o[:, h * G:(h + 1) * G] = torch.einsum("gtk,kd->tgd", torch.softmax(score, -1), v)
        outs.append(o.reshape(q, H * hd))
    return torch.cat(outs)


def _exact_logits(case, seed):
    s = _prepare_logits(case, seed)
    V, N = s["V"], case["N"]
    conf, tok, kept = np.zeros(N), np.zeros(N), []
    grammar = s["grammar"].cpu().numpy().view(np.uint8)
    allowed = torch.from_numpy(np.unpackbits(grammar, axis=1, bitorder="little")[:, :V].astype(bool)).cuda()
    lists = {k: s[k].cpu().numpy() for k in ("hist", "hist_len", "rep", "freq", "pres", "bias_ids", "bias", "bias_len",
                                             "grammar_row", "cur", "req")}
    for n in range(N):
        r = lists["req"][n]
        z = s["z"][n].double()
        if n == 0 or r != lists["req"][n - 1]:
            ids, times = np.unique(lists["hist"][r, :lists["hist_len"][r]], return_counts=True)
            ids_d, times_d = torch.from_numpy(ids).long().cuda(), torch.from_numpy(times).double().cuda()
            bias = {int(i): float(v) for i, v in zip(lists["bias_ids"][r, :lists["bias_len"][r]], lists["bias"][r])}
            at = torch.tensor(list(bias), dtype=torch.long, device="cuda")
            add = torch.tensor(list(bias.values()), dtype=torch.float64, device="cuda")
        rep, freq, pres = (float(lists[k][r]) for k in ("rep", "freq", "pres"))
        w = z[ids_d]
        z[ids_d] = torch.where(w > 0, w / rep, w * rep) - freq * times_d - pres
        z[at] += add
        if lists["grammar_row"][n] >= 0:
            z[~allowed[lists["grammar_row"][n]]] = MASKED
        if case["out"]:
            kept.append(z.clone())
        z[V - 1] = MASKED
        p = torch.softmax(z, 0)
        conf[n], tok[n] = float(p.max()), float(p[lists["cur"][n]])
    return {"x0": None, "conf": conf, "tokconf": tok, **({"z": torch.stack(kept)} if case["out"] else {})}
