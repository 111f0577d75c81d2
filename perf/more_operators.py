"""What is measured: the operators that decode from drafts over the paged K/V cache of the serving operators,
through the library's public entry points.

A step takes for every request a tree of drafted tokens behind the token it decided on last.  `tree` makes the
tokens' positions and the bits that say which of them each one sees, `attn` is the attention of the rows with such
bits over the shared prefix and the own pages, `logprobs` gives log probabilities of given tokens, the entropy and the
best alternatives from the logits, `keep` finds the path of the tree that the decisions bear out and moves its keys and
values together in all layers (or drops tokens of a long cache), `fork` lets requests continue others: full
pages are shared, the last one is copied, and what nobody holds any more is given back.

`run` computes an operator in plain torch where `own` is false, and calls the library where it is true.
Lengths, trees and choices are part of a case (`mix` seeds them), so that its work is known; the values, the order of
the pages and the token ids come from the seed.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

# (query heads, K/V heads, head dim, layers) of this repository's configurations and tests
SHAPES = {"llada": (32, 32, 128, 32), "dream": (28, 4, 128, 28), "tiny": (4, 4, 64, 2), "small": (16, 4, 64, 4)}
VOCAB = {"llada": 126464, "dream": 152064, "tiny": 1024}
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
MASKED = float("-inf")
PREFIX = 1000  # positions before the own ones, where a case does not say


def listed():
    return [
        # One request's tree of 26 drafts: launch latency and nothing else.
        _tree("tree_one", B=1, q=(26, 26), words=2, mix=1),
        # Trees of unequal sizes of a large batch, some requests without one.
        _tree("tree_many", B=800, q=(0, 64), words=2, mix=2),
        # One request checks a small tree after a short prompt.
        _attn("attn_tree_one", "dream", B=1, q=(26, 26), own=(120, 120), P=200, page=16, mix=3),
        # A batch checks trees of 48 under a system prompt.
        _attn("attn_tree_batch", "llada", B=16, q=(48, 48), own=(0, 1000), P=2048, page=64, mix=4),
        # Ragged trees and single tokens of many requests, grouped heads, f16, small pages, nothing shared.
        _attn("attn_tree_f16", "dream", B=64, q=(1, 61), own=(1, 2500), P=0, page=16, mix=5, dtype="f16"),
        # The token decided on and five alternatives: latency.
        _logprobs("logprobs_one", "llada", N=1, dtype="f32", tokens=1, top=5),
        # A batch's windows with twenty alternatives a row.
        _logprobs("logprobs_windows", "llada", N=512, dtype="f32", tokens=1, top=20),
        # A prompt is scored: its own tokens and the entropy, in bf16.
        _logprobs("logprobs_prompt", "dream", N=1501, dtype="bf16", tokens=1, top=0),
        # The accepted paths of a batch's trees, in all layers.
        _keep("keep_paths", "dream", "tree", B=32, q=(1, 61), own=(1, 500), page=16, mix=6),
        # Long requests drop a third of what they hold.
        _keep("keep_evicted", "dream", "evict", B=6, q=(0, 0), own=(500, 2000), page=64, mix=7),
        # Four beams of one small request: latency.
        _fork("fork_one", "tiny", groups=1, beams=4, own=(70, 70), page=16, mix=8),
        # Beams of a batch, in all layers.
        _fork("fork_beams", "dream", groups=16, beams=6, own=(100, 700), page=64, mix=9),
    ]


def _tree(name, B, q, words, mix):
    return dict(name=name, kind="tree", B=B, q0=q[0], q1=q[1], words=words, mix=mix)


def _attn(name, shape, B, q, own, P, page, mix, dtype="bf16", form="tree"):
    return dict(name=name, kind="attn", shape=shape, B=B, q0=q[0], q1=q[1], own0=own[0], own1=own[1], P=P, page=page,
                mix=mix, dtype=dtype, form=form)


def _logprobs(name, shape, N, dtype, tokens, top):
    return dict(name=name, kind="logprobs", shape=shape, N=N, dtype=dtype, tokens=tokens, top=top)


def _keep(name, shape, form, B, q, own, page, mix, dtype="bf16"):
    return dict(name=name, kind="keep", shape=shape, form=form, B=B, q0=q[0], q1=q[1], own0=own[0], own1=own[1], page=page,
                mix=mix, dtype=dtype)


def _fork(name, shape, groups, beams, own, page, mix, dtype="bf16"):
    return dict(name=name, kind="fork", shape=shape, groups=groups, beams=beams, own0=own[0], own1=own[1], page=page,
                mix=mix, dtype=dtype)


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _seconds(case):
    w = work(case)
    return w["bytes"] / 6.8e12 + w["flops"] / 1.9e15


def draw(rng):
    most = max(_seconds(c) for c in listed())
    while True:
        kind = rng.choice(["tree", "attn", "attn", "attn", "logprobs", "logprobs", "keep", "keep", "fork"])
        shape = rng.choice(["llada", "dream", "tiny", "small"])
        page, mix, dtype = rng.choice([16, 32, 64, 128]), rng.randrange(1 << 20), rng.choice(["bf16", "bf16", "f16"])
        if kind == "tree":
            hi = _log(rng, 1, 500)
            B = _log(rng, 1, max(1, min(2000, 60000 // hi)))
            c = _tree("", B, (rng.choice([0, 1, hi]), hi), -(-hi // 32) + rng.choice([0, 0, 1]), mix)
        elif kind == "attn":
            T = _log(rng, 1, 300)
            B, hi = max(1, min(_log(rng, 1, 100), 3000 // T)), _log(rng, 1, 4000)
            P = 0 if rng.random() < 0.5 else _log(rng, 16, 8000)
            form = rng.choice(["tree", "tree", "any"])
            c = _attn("", shape, B, (rng.choice([T, 1]), T), (rng.choice([0, hi]), hi), P, page, mix, dtype, form)
            if B * T * SHAPES[shape][0] * (P + hi + T) > 1.2e9:  # scores of the plain form
                continue
        elif kind == "logprobs":
            shape = rng.choice(["llada", "dream", "tiny"])
            c = _logprobs("", shape, _log(rng, 1, 1500), rng.choice(["f32", "bf16", "f16"]),
                          rng.choice([0, 1, 1, rng.randint(2, 9)]), rng.choice([0, 1, rng.randint(2, 32), 20]))
        else:
            form = rng.choice(["tree", "evict"]) if kind == "keep" else ""
            hi = _log(rng, 1, 3000)
            if kind == "fork":
                c = _fork("", shape, _log(rng, 1, 40), rng.randint(1, 9), (rng.choice([1, hi]), hi), page, mix, dtype)
            else:
                T = _log(rng, 1, 120) if form == "tree" else 0
                c = _keep("", shape, form, _log(rng, 1, 60), (min(1, T), T), (rng.choice([0, hi]), hi), page, mix, dtype)
            H, Hkv, hd, layers = SHAPES[shape]
            if _n_pages(c) * page * Hkv * hd * layers * 4 > 1.6e9:
                continue
        del c["name"]
        if _seconds(c) <= most:
            return c


# ------------------------------------------------------------------------------------ what `mix` decides
def _lengths(case):
    """(own lengths, new tokens) of the requests."""
    r = random.Random(case["mix"])
    own_lo, own_hi = case.get("own0", 0), case.get("own1", 0)
    if case["kind"] == "fork":
        L = [n for n in (r.randint(own_lo, own_hi) for _ in range(case["groups"])) for _ in range(case["beams"])]
        return L, [0] * len(L)
    return ([r.randint(own_lo, own_hi) for _ in range(case["B"])], [r.randint(case["q0"], case["q1"]) for _ in range(case["B"])])


def _parents(case):
    """The trees: for each new token the one that it follows, an earlier one among the last eight (the first: -1)."""
    r = random.Random(case["mix"] + 1)
    return [[-1 if i == 0 else r.randint(max(0, i - 8), i - 1) for i in range(q)] for q in _lengths(case)[1]]


def _drafts(case):
    """Drafted ids and decisions of the trees' tokens (small numbers; siblings may draft the same): four decisions of
    five name a child."""
    r = random.Random(case["mix"] + 2)
    ids, decided = [], []
    for tree in _parents(case):
        mine = [r.randrange(40) for _ in tree]
        children = [[] for _ in tree]
        for c, p in enumerate(tree):
            if p >= 0:
                children[p].append(c)
        ids.append(mine)
        decided.append([mine[r.choice(c)] if c and r.random() < 0.8 else r.randrange(40) for c in children])
    return ids, decided


DEPTH = 16  # tokens of a path that are kept at most


def _kept(case):
    """The places, among the own ones from a first on, that are kept of each request."""
    if case["form"] == "evict":
        r = np.random.RandomState(case["mix"])
        return [np.sort(r.permutation(n)[:n - n // 3]).tolist() for n in _lengths(case)[0]]
    out = []
    for tree, ids, decided in zip(_parents(case), *_drafts(case)):
        path = [0] if tree else []
        while path and len(path) < DEPTH:
            nxt = [c for c in range(path[-1] + 1, len(tree)) if tree[c] == path[-1] and ids[c] == decided[path[-1]]]
            if not nxt:
                break
            path.append(nxt[0])
        out.append(path)
    return out


def _beams(case):
    """Which request each request continues: one of its group."""
    r, K = random.Random(case["mix"] + 3), case["beams"]
    return [g * K + r.randrange(K) for g in range(case["groups"]) for _ in range(K)]


def _pages(L, page):
    return [-(-n // page) for n in L]


def _n_pages(case):
    L, Q = _lengths(case)
    if case["kind"] == "fork":  # full pages of a group once, the last of each beam, and as many to spare
        return sum(n // case["page"] for n in L[::case["beams"]]) + 2 * len(L) + 1
    return sum(_pages([a + b for a, b in zip(L, Q)], case["page"])) + _pages([case.get("P", 0)], case["page"])[0] + 1


# ------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _flat(v):
    return _ints([x for row in v for x in row])


def _handle(case, B, rows, n_pages, max_pages):
    from paper_2606_13740_gb300 import serve

    H, Hkv, hd, _ = SHAPES[case.get("shape", "tiny")]
    return serve.Serve(serve.ServeConfig(max_batch=B, max_rows=max(1, rows), page=case.get("page", 64), n_pages=n_pages,
                                         max_pages=max_pages, n_heads=H, n_kv_heads=Hkv, head_dim=hd,
                                         dtype=case.get("dtype", "bf16")))


def prepare(case, seed):
    return {"tree": _prepare_tree, "attn": _prepare_attn, "logprobs": _prepare_logprobs, "keep": _prepare_keep,
            "fork": _prepare_fork}[case["kind"]](case, seed)


def _prepare_tree(case, seed):
    """The step's plan, and the trees in their packed order; the requests' lengths come from the seed."""
    _, Q = _lengths(case)
    g = _generator(seed)
    L = torch.randint(0, 1000, (case["B"],), device="cuda", generator=g, dtype=torch.int32)
    rows = sum(Q)
    s = {"case": dict(case), "parent": _flat(_parents(case)), "q_len": _ints(Q), "len": L, "rows": rows}
    if own:
        most = -(-(1000 + case["q1"]) // 64)
        s["handle"] = k = _handle(case, case["B"], rows, case["B"] * most, most)
        k.dllm_serve_plan(L, s["q_len"], rows, prefix_len=PREFIX)
    return s


def _tables(case, seed, need, taken):
    """Pages in random order: `taken` of them apart, then the requests' own; (order, table, held)."""
    g = _generator(seed)
    n_pages, max_pages = _n_pages(case), max(need + [1])
    order = torch.randperm(n_pages, device="cuda", generator=g, dtype=torch.int32)
    h = _ints(need)
    first = torch.cumsum(h, 0) - h + taken
    col = torch.arange(max_pages, device="cuda", dtype=torch.int32)[None]
    table = torch.where(col < h[:, None], order[(first[:, None] + col).clamp(max=n_pages - 1).long()], -1).to(torch.int32)
    return g, order, table.contiguous(), h


def _prepare_attn(case, seed):
    """The requests' pages in random order over a full pool, the plan of the step and the bits of its rows (made once
    for all its layers)."""
    H, Hkv, hd, _ = SHAPES[case["shape"]]
    page, P, B = case["page"], case["P"], case["B"]
    L, Q = _lengths(case)
    n_prefix = -(-P // page)
    g, order, table, h = _tables(case, seed, _pages([a + b for a, b in zip(L, Q)], page), n_prefix)
    dt, N, words = DTYPE[case["dtype"]], sum(Q), -(-case["q1"] // 32)
    q = torch.randn(N, H, hd, device="cuda", generator=g).to(dt)
    kc, vc = (torch.randn(order.numel(), Hkv, page, hd, device="cuda", generator=g).to(dt) for _ in range(2))
    if case["form"] == "tree":
        rows = []
        for tree in _parents(case):
            seen = []
            for i, p in enumerate(tree):
                seen.append((seen[p] if p >= 0 else 0) | 1 << i)
            rows += seen
        mask = np.frombuffer(b"".join(x.to_bytes(4 * words, "little") for x in rows), np.int32).reshape(N, words)
        mask = torch.from_numpy(mask.copy()).cuda()
    else:  # any bits, those past the tokens that there are as well; one row of twenty sees no new token
        mask = torch.randint(-(1 << 31), 1 << 31, (N, words), device="cuda", generator=g, dtype=torch.int64).to(torch.int32)
        mask *= (torch.rand(N, 1, device="cuda", generator=g) < 0.95).to(torch.int32)
    s = {"case": dict(case), "q": q, "kc": kc, "vc": vc, "prefix_pages": order[:n_prefix].contiguous(), "table": table,
         "len": _ints(L), "q_len": _ints(Q), "mask": mask}
    if own:
        s["handle"] = k = _handle(case, B, N, order.numel(), table.shape[1])
        k.table.copy_(table), k.held.copy_(h), k.ring_pos.zero_()
        k.dllm_serve_plan(s["len"], s["q_len"], N, prefix_len=P)
    return s


def _prepare_logprobs(case, seed):
    """Logits from flat to peaked; in a fifth of the rows a grammar has left one id of ten."""
    V, N = VOCAB[case["shape"]], case["N"]
    g = _generator(seed)
    z = torch.randn(N, V, device="cuda", generator=g)
    z *= 0.5 + 4 * torch.rand(N, 1, device="cuda", generator=g)
    for n in torch.nonzero(torch.rand(N, device="cuda", generator=g) < 0.2)[:, 0].tolist():
        z[n, torch.rand(V, device="cuda", generator=g) < 0.9] = MASKED
    z = z.to(DTYPE[case["dtype"]])
    tokens = torch.randint(0, V - 1, (N, case["tokens"]), device="cuda", generator=g, dtype=torch.int32)
    best = z[:, :V - 1].argmax(1, keepdim=True).to(torch.int32)
    there = torch.gather(z, 1, tokens.long()) > MASKED
    tokens = torch.where(there & (torch.rand(N, case["tokens"], device="cuda", generator=g) < 0.5), tokens, best)
    return {"case": dict(case), "z": z, "tokens": tokens.contiguous() if case["tokens"] else None, "V": V}


def _caches(case, g, n_pages):
    _, Hkv, hd, layers = SHAPES[case["shape"]]
    shape, dt = (layers, n_pages, Hkv, case["page"], hd), DTYPE[case["dtype"]]
    return [torch.empty(shape, device="cuda", dtype=dt).normal_(generator=g) for _ in range(2)]


def _prepare_keep(case, seed):
    """The requests' caches in all layers, with the trees' drafts and decisions, or the places that are kept."""
    L, Q = _lengths(case)
    g, order, table, h = _tables(case, seed, _pages([a + b for a, b in zip(L, Q)], case["page"]), 0)
    kc, vc = _caches(case, g, order.numel())
    s = {"case": dict(case), "table": table, "kc": kc, "vc": vc, "len": _ints(L), "q_len": _ints(Q)}
    if case["form"] == "tree":
        ids, decided = _drafts(case)
        off = int(torch.randint(0, 100000, (1,), device="cuda", generator=g))
        s["parent"], s["ids"], s["x0"] = _flat(_parents(case)), _flat(ids) + off, _flat(decided) + off
    else:
        kept = _kept(case)
        most = max(max(map(len, kept)), 1)
        s["keep"], s["keep_len"] = _ints([k + [-1] * (most - len(k)) for k in kept]), _ints([len(k) for k in kept])
        s["first"] = torch.zeros_like(s["len"])
    if own:
        s["handle"] = k = _handle(case, case["B"], sum(Q), order.numel(), table.shape[1])
        k.table.copy_(table), k.held.copy_(h), k.ring_pos.zero_()
        k.dllm_serve_plan(s["len"], s["q_len"], sum(Q))
        s["layers"] = k.layers(kc, vc)
    return s


def _prepare_fork(case, seed):
    """Beams that share their group's full pages, each with a last page of its own; the free pages."""
    L, _ = _lengths(case)
    K, page, B = case["beams"], case["page"], len(L)
    n_pages, max_pages = _n_pages(case), max(_pages(L, page) + [1]) + 1
    order = torch.randperm(n_pages, device="cuda", generator=_generator(seed), dtype=torch.int32)
    at, pick = 0, []
    for g in range(case["groups"]):
        full = L[g * K] // page
        shared = list(range(at, at + full))
        at += full
        for b in range(K):
            mine = shared + ([at] if L[g * K] % page else [])
            at += len(mine) - full
            pick.append(mine + [-1] * (max_pages - len(mine)))
    pick = _ints(pick)
    table = torch.where(pick >= 0, order[pick.clamp(min=0).long()], -1).to(torch.int32).contiguous()
    ring = torch.cat([order[at:], torch.zeros(at, device="cuda", dtype=torch.int32)]).contiguous()
    kc, vc = _caches(case, _generator(seed + 1), n_pages)
    held = (table >= 0).sum(1).to(torch.int32)
    s = {"case": dict(case), "table": table, "held": held, "ring": ring, "ring_pos": _ints([0, n_pages - at]), "kc": kc,
         "vc": vc, "src": _ints(_beams(case)), "len": _ints(L)}
    if own:
        s["handle"] = k = _handle(case, B, 1, n_pages, max_pages)
        k.table.copy_(table), k.held.copy_(held), k.ring.copy_(ring), k.ring_pos.copy_(s["ring_pos"])
        s["layers"] = k.layers(kc, vc)
    return s


# ------------------------------------------------------------------------------------ one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"tree": _own_tree, "attn": _own_attn, "logprobs": _own_logprobs, "keep": _own_keep, "fork": _own_fork}[kind](state)
    return {"tree": _plain_tree, "attn": _plain_attn, "logprobs": _plain_logprobs, "keep": _plain_keep,
            "fork": _plain_fork}[kind](state)


def _own_tree(s):
    k = s["handle"]
    return {"mask": k.dllm_serve_tree(s["parent"], 32 * s["case"]["words"]), "pos": k.pos}


def _rows(s):
    """Rows of the packed arrays as [batch][longest]: (row of each place, whether there is one)."""
    Q, T = s["q_len"].long(), s["case"]["q1"]
    t = torch.arange(T, device="cuda")
    return ((torch.cumsum(Q, 0) - Q)[:, None] + t), t < Q[:, None]


def _plain_tree(s):
    B, T, N, words = s["case"]["B"], s["case"]["q1"], s["rows"], s["case"]["words"]
    if N == 0:
        return {"mask": torch.zeros(0, words, dtype=torch.int32, device="cuda"), "pos": torch.zeros(1, dtype=torch.int32, device="cuda")}
    row, there = _rows(s)
    parent = torch.where(there, s["parent"][row.clamp(max=N - 1)].long(), -1)
    t = torch.arange(T, device="cuda")
    seen = ((parent[..., None] == t) | (t[:, None] == t)).float()
    n = 1
    while n < T:  # who is reached within twice as many steps
        seen = (torch.matmul(seen, seen) > 0).float()
        n *= 2
    depth = seen.sum(-1).long() - 1
    bits = torch.zeros(B, T, 32 * words, dtype=torch.int64, device="cuda")
    bits[..., :T] = seen.long()
    w = (bits.view(B, T, words, 32) << torch.arange(32, device="cuda")).sum(-1)
    w = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)
    pos = PREFIX + s["len"][:, None].long() + depth
    return {"mask": w[there], "pos": pos[there].to(torch.int32)}


def _own_attn(s):
    return s["handle"].dllm_serve_tree_attention(s["q"], s["kc"], s["vc"], s["mask"], s["prefix_pages"])


def _plain_attn(s):
    c = s["case"]
    H, Hkv, hd, _ = SHAPES[c["shape"]]
    B, P, G, q = c["B"], c["P"], H // Hkv, s["q"]
    L, Q = s["len"].long(), s["q_len"].long()
    N, T, K = q.shape[0], c["q1"], s["table"].shape[1] * c["page"]
    row, there = _rows(s)
    row = row.clamp(max=N - 1)
    # queries [B][Hkv][T * G][hd], keys and values of the prefix [Hkv][P][hd] and of each request [B][Hkv][K][hd]
    x = q[row].float().view(B, T, Hkv, G, hd).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, hd) / math.sqrt(hd)
    pages, mine = s["prefix_pages"].long(), s["table"].clamp(min=0).long()
    kp, vp = (m[pages].float().transpose(0, 1).reshape(Hkv, -1, hd)[:, :P] for m in (s["kc"], s["vc"]))
    ko, vo = (m[mine].float().transpose(1, 2).reshape(B, Hkv, K, hd) for m in (s["kc"], s["vc"]))
    key = torch.arange(K, device="cuda")
    vo = torch.where((key < (L + Q)[:, None])[:, None, :, None], vo, 0.0)
    new = key - L[:, None]  # [B][K]: which new token a key is
    word = torch.gather(s["mask"][row], 2, (new // 32).clamp(0, s["mask"].shape[1] - 1)[:, None].expand(B, T, K))
    bit = (word >> (new % 32).to(torch.int32)[:, None]) & 1 > 0
    seen = (new < 0)[:, None] | (bit & (new < Q[:, None])[:, None])
    seen = seen[:, None, :, None].expand(B, 1, T, G, K).reshape(B, 1, T * G, K)
    sp = torch.matmul(x, kp.transpose(1, 2))
    so = torch.where(seen, torch.matmul(x, ko.transpose(2, 3)), MASKED)
    m = so.amax(-1, keepdim=True)
    if P:
        m = torch.maximum(m, sp.amax(-1, keepdim=True))
    m = torch.where(m == MASKED, 0.0, m)
    sp, so = torch.exp(sp - m), torch.exp(so - m)
    total = sp.sum(-1, keepdim=True) + so.sum(-1, keepdim=True)
    o = (torch.matmul(sp, vp) + torch.matmul(so, vo)) / torch.where(total > 0, total, 1.0)
    return o.view(B, Hkv, T, G, hd).permute(0, 2, 1, 3, 4)[there].reshape(N, H * hd).to(q.dtype)


def _own_logprobs(s):
    from paper_2606_13740_gb300 import serve

    lp, entropy, top_ids, top_lp, lse = serve.dllm_serve_logprobs(s["z"], s["tokens"], s["V"] - 1, top=s["case"]["top"])
    out = {"entropy": entropy, "lse": lse}
    if lp is not None:
        out["lp"] = lp
    if top_ids is not None:
        out["top_ids"], out["top_lp"] = top_ids, top_lp
    return out


def _plain_logprobs(s):
    V = s["V"]
    ids = torch.arange(V, device="cuda")
    z = torch.where(ids == V - 1, MASKED, s["z"].float())  # the mask id is no answer
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    out = {"lse": lse[:, 0], "entropy": torch.where(e > 0, e * (lse - z), 0.0).sum(1) / total[:, 0]}
    if s["tokens"] is not None:
        out["lp"] = torch.gather(z, 1, s["tokens"].long()) - lse
    tops = []
    for _ in range(s["case"]["top"]):
        top = torch.where(z == z.amax(1, keepdim=True), ids, V).amin(1, keepdim=True)
        tops.append((top, torch.gather(z, 1, top)))
        z = torch.where(ids == top, MASKED, z)
    if tops:
        out["top_ids"] = torch.cat([t for t, _ in tops], 1).to(torch.int32)
        out["top_lp"] = torch.cat([v for _, v in tops], 1) - lse
    return out


def _own_keep(s):
    k, out = s["handle"], {"k": s["kc"], "v": s["vc"]}
    if s["case"]["form"] == "tree":
        keep, n, nxt = k.dllm_serve_accept(s["parent"], s["ids"], s["x0"], s["case"]["B"], DEPTH)
        k.dllm_serve_compact(s["layers"], s["len"], keep, n)
        return {"keep": keep, "n": n, "next": nxt, **out}
    k.dllm_serve_compact(s["layers"], s["first"], s["keep"], s["keep_len"])
    return out


def _plain_keep(s):
    page, out = s["case"]["page"], {"k": s["kc"], "v": s["vc"]}
    if s["case"]["form"] == "tree":
        N = s["parent"].shape[0]
        row, there = _rows(s)
        parent, ids, x0 = (torch.where(there, s[k][row.clamp(max=max(N - 1, 0))], -2) for k in ("parent", "ids", "x0"))
        T = s["case"]["q1"]
        t = torch.arange(T, device="cuda")
        node = torch.where(there[:, 0], 0, T)  # T: no token
        nxt, path = torch.full_like(s["len"], -1), []
        for _ in range(DEPTH):
            path.append(torch.where(node < T, node, -1))
            want = torch.gather(x0, 1, node.clamp(max=T - 1)[:, None])
            nxt = torch.where(node < T, want[:, 0], nxt)
            child = (parent == node[:, None]) & (ids == want) & there
            node = torch.where(child, t, T).amin(1)
        keep = torch.stack(path, 1).to(torch.int32)
        n, first = (keep >= 0).sum(1).to(torch.int32), s["len"]
        out.update({"keep": keep, "n": n, "next": nxt})
    else:
        keep, n, first = s["keep"], s["keep_len"], s["first"]
    i = torch.arange(keep.shape[1], device="cuda")
    moved = (i < n[:, None]) & (keep != i)
    place = [torch.where(moved, first[:, None] + v, 0).long() for v in (keep, i)]
    src, dst = (torch.gather(s["table"], 1, p // page)[moved].long() * page + (p % page)[moved] for p in place)
    for c in (s["kc"], s["vc"]):
        c[:, dst // page, :, dst % page] = c[:, src // page, :, src % page]
    return out


def _own_fork(s):
    k = s["handle"]
    k.dllm_serve_fork(s["layers"], s["src"], s["len"])
    return {"table": k.table, "held": k.held, "ring": k.ring, "ring_pos": k.ring_pos, "k": s["kc"], "v": s["vc"]}


def _plain_fork(s):
    page, table, held, ring, ring_pos = s["case"]["page"], s["table"], s["held"], s["ring"], s["ring_pos"]
    n_pages, (B, M), L = ring.shape[0], table.shape, s["len"]
    col, page_ids = torch.arange(M, device="cuda"), torch.arange(n_pages, device="cuda")
    need, full, tail = (L + page - 1) // page, L // page, L % page
    new = torch.where(col < need[:, None], table[s["src"].long()], -1)

    def holders(t, of):
        return torch.zeros(n_pages + 1, dtype=torch.int64, device="cuda").scatter_add_(
            0, torch.where(of, t, n_pages).flatten().long(), torch.ones(t.numel(), dtype=torch.int64, device="cuda"))[:n_pages]

    count = holders(new, col < full[:, None])
    last = torch.gather(new, 1, full.clamp(max=M - 1)[:, None].long())[:, 0].long()  # the page that is written on
    b = torch.arange(B, device="cuda")
    writer = torch.full((n_pages + 1,), B, dtype=torch.int64, device="cuda").scatter_reduce_(
        0, torch.where(tail > 0, last, n_pages), b, "amin")
    at = last.clamp(min=0)
    copied = (tail > 0) & ((count[at] > 0) | (writer[at] != b))
    head, free = ring_pos[0], ring_pos[1]
    nth = torch.cumsum(copied, 0)
    given = ring[((head + nth - 1) % n_pages).clamp(min=0).long()]
    new = torch.where(copied[:, None] & (col == full[:, None]), given[:, None], new)
    back = (holders(table, col < held[:, None]) > 0) & (holders(new, col < need[:, None]) == 0)
    rank = torch.cumsum(back, 0) - 1
    ring[((head + free + rank) % n_pages)[back].long()] = page_ids[back].to(torch.int32)
    which = torch.nonzero(copied)[:, 0]
    there = torch.arange(page, device="cuda") < tail[which][:, None]
    for c in (s["kc"], s["vc"]):
        to, of = given[which].long(), last[which]
        c[:, to] = torch.where(there[:, None, :, None], c[:, of], c[:, to])
    taken = nth[-1]
    ring_pos.copy_(torch.stack([(head + taken) % n_pages, free - taken + back.sum()]))
    table.copy_(new), held.copy_(need)
    return {"table": table, "held": held, "ring": ring, "ring_pos": ring_pos, "k": s["kc"], "v": s["vc"]}


# ------------------------------------------------------------------------------------ work
def work(case):
    if case["kind"] == "tree":  # a parent and a position in, a position and the bits out
        return {"bytes": sum(_lengths(case)[1]) * (12.0 + 4.0 * case["words"]) + 8.0 * case["B"], "flops": 0.0}
    size = {"f32": 4.0, "bf16": 2.0, "f16": 2.0}[case["dtype"]]
    if case["kind"] == "logprobs":
        V, N = VOCAB[case["shape"]], case["N"]
        return {"bytes": N * (V * size + 8.0 * case["tokens"] + 8.0 * case["top"] + 8.0), "flops": 6.0 * N * V}
    H, Hkv, hd, layers = SHAPES[case["shape"]]
    if case["kind"] == "attn":
        L, Q = _lengths(case)
        if case["form"] == "tree":
            pairs = 0
            for tree in _parents(case):
                seen = []
                for p in tree:
                    seen.append(1 + (seen[p] if p >= 0 else 0))
                pairs += sum(seen)
        else:
            pairs = sum(0.475 * q * q for q in Q)
        pairs += sum(q * (case["P"] + l) for l, q in zip(L, Q))
        words = -(-case["q1"] // 32)
        return {"bytes": 4.0 * sum(Q) * (H * hd + words) + 4.0 * (case["P"] + sum(L) + sum(Q)) * Hkv * hd, "flops": 4.0 * hd * H * pairs}
    token = 2.0 * layers * Hkv * hd * size  # of keys and values
    if case["kind"] == "keep":
        kept = _kept(case)
        moved = sum(sum(k != i for i, k in enumerate(ks)) for ks in kept)
        lists = 12.0 * sum(_lengths(case)[1]) if case["form"] == "tree" else 4.0 * sum(map(len, kept))
        return {"bytes": 2.0 * moved * token + lists + 4.0 * case["B"], "flops": 0.0}
    L, _ = _lengths(case)
    src, b = _beams(case), 0.0
    for i, (s, n) in enumerate(zip(src, L)):
        if s in src[:i]:
            b += 2.0 * (n % case["page"]) * token
    return {"bytes": b + 16.0 * len(L) + 8.0 * sum(_pages(L, case["page"])), "flops": 0.0}


# ------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """From the operators' definitions, request by request or row by row (moved and counted things have no such value)."""
    if case["kind"] == "attn":
        return _exact_attn(case, seed)
    return _exact_logprobs(case, seed) if case["kind"] == "logprobs" else None


def _exact_attn(case, seed):
    s = _prepare_attn(case, seed)
    H, Hkv, hd, _ = SHAPES[case["shape"]]
    page, P, G = case["page"], case["P"], H // Hkv
    L, Q = _lengths(case)
    if 4.0 * hd * sum(q * (P + l + q) for l, q in zip(L, Q)) * H > 6e12:
        return None
    bits = np.unpackbits(s["mask"].cpu().numpy().view(np.uint8), axis=1, bitorder="little").astype(bool)
    outs, at = [], 0
    pre = s["prefix_pages"].long()
    place = functools.partial(torch.arange, device="cuda")
    for b, (l, q) in enumerate(zip(L, Q)):
        mine = s["table"][b, :-(-(l + q) // page)].long()
        x = s["q"][at:at + q].double()
        slots = torch.cat([(pre[:, None] * page + place(page)).flatten()[:P], (mine[:, None] * page + place(page)).flatten()[:l + q]])
        sees = np.ones((q, P + l + q), bool)
        sees[:, P + l:] = bits[at:at + q, :q]
        sees = torch.from_numpy(sees).cuda()
        at += q
        o = torch.zeros(q, H, hd, device="cuda", dtype=torch.float64)
        for h in range(Hkv):
            k, v = (m[slots // page, h, slots % page].double() for m in (s["kc"], s["vc"]))
            score = torch.einsum("tgd,kd->gtk", x[:, h * G:(h + 1) * G], k) * hd ** -0.5
            p = torch.softmax(score.masked_fill_(~sees, MASKED), -1)
            p = torch.where(sees.any(-1)[None, :, None], p, 0.0)  # a row that sees nothing: zeros
            o[:, h * G:(h + 1) * G] = torch.einsum("gtk,kd->tgd", p, v)
        outs.append(o.reshape(q, H * hd))
    return torch.cat(outs)


def _exact_logprobs(case, seed):
    s = _prepare_logprobs(case, seed)
    V, N, top = s["V"], case["N"], case["top"]
    rows = {"lse": [], "entropy": [], "lp": [], "top_lp": []}
    for n in range(N):
        z = s["z"][n].double()
        z[V - 1] = MASKED
        lp = torch.log_softmax(z, 0)
        rows["lse"].append(torch.logsumexp(z, 0))
        rows["entropy"].append(torch.special.entr(lp.exp()).sum())
        if case["tokens"]:
            rows["lp"].append(lp[s["tokens"][n].long()])
        if top:
            rows["top_lp"].append(torch.sort(lp, descending=True).values[:top])
    out = {k: torch.stack(v) for k, v in rows.items() if v}
    return {**out, "top_ids": None} if top else out
