"""The serving operators on the GPU against plain implementations in 64 bits (or, for whole numbers, in plain
Python): the plan over many steps, the norm and rotation, attention over pages, and the logits."""
import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# unit roundoff of a type
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_13740_gb300 as pkg
    pkg.lib()
    return torch.device("cuda:0")


def _serve(**kw):
    from paper_2606_13740_gb300 import serve
    return serve.Serve(serve.ServeConfig(**kw))


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ plan
class Pool:
    """The plan's definition in plain Python."""

    def __init__(self, B, page, n_pages, max_pages):
        self.page, self.n, self.most = page, n_pages, max_pages
        self.rows = [[] for _ in range(B)]
        self.free = list(range(n_pages))  # oldest first

    def plan(self, L, Q, rows, prefix):
        budget, asked, back, refused = len(self.free), 0, [], []
        for b, (l, q) in enumerate(zip(L, Q)):
            need = -(-(l + q) // self.page)
            bad = l < 0 or q < 0 or need > self.most
            grow = 0 if bad else max(0, need - len(self.rows[b]))
            asked += grow
            no = bad or (grow > 0 and asked > budget)
            refused.append(no)
            if no:
                continue
            for _ in range(grow):
                self.rows[b].append(self.free.pop(0))
            back += self.rows[b][need:]
            del self.rows[b][need:]
        self.free += back
        slot, pos, req, start = [], [], [], [0]
        for b, (l, q) in enumerate(zip(L, Q)):
            start.append(start[-1] + max(q, 0))
            for t in range(max(q, 0)):
                at = l + t
                slot.append(-1 if refused[b] else self.rows[b][at // self.page] * self.page + at % self.page)
                pos.append(0 if refused[b] else prefix + at)
                req.append(b)
        pad = max(0, rows - len(slot))
        return dict(row_start=start, n_keys=[0 if no else l + q for no, l, q in zip(refused, L, Q)],
                    slot=(slot + [-1] * pad)[:rows], pos=(pos + [0] * pad)[:rows], req=(req + [-1] * pad)[:rows],
                    refused=sum(refused), given=len(back))


def _same_plan(s, pool, want, B, rows):
    got = {k: getattr(s, k).cpu().tolist() for k in ("row_start", "n_keys", "slot", "pos", "req", "held", "ring", "ring_pos")}
    assert got["row_start"][:B + 1] == want["row_start"] and got["n_keys"][:B] == want["n_keys"]
    for k in ("slot", "pos", "req"):
        assert got[k][:rows] == want[k], k
    table = s.table.cpu().tolist()
    for b in range(B):
        n = len(pool.rows[b])
        assert got["held"][b] == n and table[b][:n] == pool.rows[b] and all(p == -1 for p in table[b][n:])
    head, count = got["ring_pos"]
    assert [got["ring"][(head + i) % pool.n] for i in range(count)] == pool.free
    assert s.status.cpu().tolist()[1] == want["refused"] and s.status.cpu().tolist()[3] == want["given"]


@pytest.mark.parametrize("B,page,n_pages,max_pages,q_most,steps", [
    (1, 64, 4, 4, 70, 12), (3, 16, 40, 12, 40, 30), (17, 32, 60, 9, 60, 30), (200, 16, 900, 20, 50, 8),
    (1025, 16, 3000, 8, 30, 5), (4096, 16, 9000, 6, 12, 4), (5, 128, 30, 9, 700, 12), (2, 256, 64, 40, 6000, 8),
])
def test_plan_matches_definition_over_steps(dev, B, page, n_pages, max_pages, q_most, steps):
    """Requests grow, end, shrink and are refused (pool empty, too many pages, negative lengths), step after step."""
    from paper_2606_13740_gb300 import DllmError
    r = random.Random(B * 31 + page)
    most = B * q_most + 64
    s = _serve(max_batch=B, max_rows=most, page=page, n_pages=n_pages, max_pages=max_pages, n_heads=4, n_kv_heads=2, head_dim=64)
    pool = Pool(B, page, n_pages, max_pages)
    own = [0] * B
    for step in range(steps):
        L, Q = [], []
        for b in range(B):
            kind = r.random()
            if kind < 0.15:
                own[b] = 0
            elif kind < 0.25:
                own[b] = r.randint(0, own[b])
            q = 0 if kind > 0.9 else r.randint(0, q_most) if r.random() < 0.5 else min(1, q_most)
            if kind > 0.98 and B > 1:  # lengths that make no sense
                L.append(r.choice([-1, -2 ** 31, 2 ** 31 - 1, max_pages * page]))
                Q.append(r.choice([1, 3]))
            else:
                L.append(own[b])
                Q.append(q)
        rows = min(most, sum(max(q, 0) for q in Q) + r.choice([0, 0, 5]))
        want = pool.plan(L, Q, rows, 7 * step)
        s.dllm_serve_plan(_i32(L), _i32(Q), rows, prefix_len=7 * step)
        _same_plan(s, pool, want, B, rows)
        own = [n if n else o for n, o in zip(want["n_keys"], own)]
        own = [min(o, len(p) * page) for o, p in zip(own, pool.rows)]
        bad = any(l < 0 or -(-(l + q) // page) > max_pages for l, q in zip(L, Q))
        if want["refused"]:
            with pytest.raises(DllmError) as e:
                s.dllm_serve_check()
            assert e.value.code == (-6 if want["refused"] and not bad else e.value.code) and e.value.code in (-1, -6)
        s.dllm_serve_check()  # clear again


def test_plan_rows_left_out_and_batch_below_its_limit(dev):
    """More tokens than rows: the last are left out and reported; requests past the batch keep their pages."""
    from paper_2606_13740_gb300 import DllmError
    s = _serve(max_batch=4, max_rows=50, page=16, n_pages=20, max_pages=8, n_heads=4, n_kv_heads=2, head_dim=64)
    s.dllm_serve_plan(_i32([0, 0, 0, 40]), _i32([0, 0, 0, 1]), 1)
    mine = s.table[3].cpu().tolist()
    s.dllm_serve_plan(_i32([0, 5]), _i32([30, 30]), 40)
    assert s.slot[:40].cpu().tolist()[-1] == s.table[1, 0].item() * 16 + 5 + 9
    assert s.table[3].cpu().tolist() == mine and s.held.cpu().tolist() == [2, 3, 0, 3]
    with pytest.raises(DllmError, match="status bits 8"):
        s.dllm_serve_check()
    s.dllm_serve_plan(_i32([0]), _i32([0]), 0)
    s.dllm_serve_check()
    s.dllm_serve_reset()
    assert s.held.cpu().tolist() == [0] * 4 and s.ring_pos.cpu().tolist() == [0, 20]


def test_plan_keeps_to_its_buffers_on_a_broken_state(dev):
    """A state no plan leaves (pages outside the pool, wild counts) is reported and refused, never followed."""
    from paper_2606_13740_gb300 import DllmError
    s = _serve(max_batch=4, max_rows=64, page=16, n_pages=8, max_pages=4, n_heads=4, n_kv_heads=2, head_dim=64)
    s.held.copy_(_i32([1 << 30, -5, 1, 2]))
    s.table[2:] = _i32([[99, -7, 5, 6]])
    s.dllm_serve_plan(_i32([3, 3, 3, 20]), _i32([1, 1, 1, 1]), 4)
    assert s.slot[:4].cpu().tolist() == [-1, -1, -1, -1] and s.n_keys.cpu().tolist()[:2] == [0, 0]
    with pytest.raises(DllmError, match="status bits 64"):
        s.dllm_serve_check()
    s.dllm_serve_reset()
    s.ring_pos.copy_(_i32([-3, 1 << 30]))
    s.dllm_serve_plan(_i32([0]), _i32([1]), 1)
    with pytest.raises(DllmError):
        s.dllm_serve_check()


# ------------------------------------------------------------------ norm and rotation
@pytest.mark.parametrize("H,Hkv,hd,N,page,src,dtype,packed,far", [
    (4, 4, 64, 1, 16, "bf16", "bf16", True, 100), (28, 4, 128, 37, 16, "f16", "f16", True, 131072),
    (32, 32, 128, 96, 64, "f32", "bf16", True, 1000), (5, 5, 64, 201, 32, "f32", "f16", False, 1 << 20),
    (16, 4, 64, 3000, 128, "bf16", "bf16", False, 70000), (3, 1, 128, 7, 256, "bf16", "bf16", True, 1 << 30),
    (28, 4, 128, 12000, 16, "bf16", "bf16", True, 5000), (128, 1, 128, 5, 16, "f16", "f16", False, 9),
])
def test_qk_norm_rope_matches_64_bits(dev, H, Hkv, hd, N, page, src, dtype, packed, far):
    g = torch.Generator(device="cuda").manual_seed(N + hd)
    n_pages = -(-N // page) + 2
    # pages farther apart than dense, in a cache where K and V share an allocation
    stride = 2 * Hkv * page * hd
    s = _serve(max_batch=1, max_rows=N, page=page, n_pages=n_pages, max_pages=4, n_heads=H, n_kv_heads=Hkv, head_dim=hd,
               dtype=dtype, page_stride=stride)
    both = torch.full((n_pages, 2, Hkv, page, hd), 3.0, device="cuda", dtype=DT[dtype])
    kc, vc = both[:, 0], both[:, 1]
    x = torch.randn(N, (H + 2 * Hkv) * hd, device="cuda", generator=g) * torch.exp(2 * torch.randn(N, 1, device="cuda", generator=g))
    x[N // 2] *= 1e-6  # a row where eps counts
    x = x.to(DT[src])
    if packed:
        q, k, v = x[:, :H * hd], x[:, H * hd:(H + Hkv) * hd], x[:, (H + Hkv) * hd:]
    else:
        q, k, v = (t.contiguous() for t in (x[:, :H * hd], x[:, H * hd:(H + Hkv) * hd], x[:, (H + Hkv) * hd:]))
        q = q.view(N, H, hd)
    slot = torch.randperm(n_pages * page, device="cuda", generator=g)[:N].to(torch.int32)
    slot[N // 3] = -1 if N > 1 else slot[0]
    pos = torch.randint(0, far, (N,), device="cuda", generator=g, dtype=torch.int32)
    s.slot.copy_(slot), s.pos.copy_(pos)
    theta = torch.tensor([10000.0 ** (-2 * j / hd) for j in range(hd // 2)], dtype=torch.float32, device="cuda")
    gains = [1 + 0.2 * torch.randn(hd, device="cuda", generator=g) for _ in range(2)]
    for gq, gk in ((gains[0], gains[1]), (None, None)):
        out = s.dllm_serve_qk_norm_rope(q, k, v, theta, kc, vc, q_gain=gq, k_gain=gk, eps=1e-5)
        s.dllm_serve_check()
        xd = x.double().view(N, H + 2 * Hkv, hd)
        ang = pos.double()[:, None] * theta.double()
        c, d = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        y = xd[:, :H + Hkv]
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-5)
        if gq is not None:
            y = y * torch.cat([gq.double().expand(H, hd), gk.double().expand(Hkv, hd)])
        a, b = y[..., :hd // 2], y[..., hd // 2:]
        want = torch.cat([a * c - b * d, b * c + a * d], -1)
        # one rounding to the type, and fp32: about ten roundings of the two products a value is a sum of
        size = torch.cat([a.abs() + b.abs()] * 2, -1)
        tol = U[dtype] * want.abs() + 2e-6 * size + 2.0 ** -25
        assert bool(((out.double() - want[:, :H]).abs() <= tol[:, :H]).all())
        rows = torch.nonzero(slot >= 0)[:, 0]
        at = slot[rows].long()
        gotk, gotv = kc[at // page, :, at % page].double(), vc[at // page, :, at % page]
        assert bool(((gotk - want[rows, H:]).abs() <= tol[rows, H:]).all())
        assert torch.equal(gotv, x.view(N, H + 2 * Hkv, hd)[rows, H + Hkv:].to(DT[dtype]))
        rest = torch.ones(n_pages, page, dtype=torch.bool, device="cuda")
        rest[at // page, at % page] = False
        assert bool((kc.transpose(1, 2)[rest] == 3.0).all()) and bool((vc.transpose(1, 2)[rest] == 3.0).all())


def test_qk_norm_rope_in_place_and_bad_slots(dev):
    """q_out = q, a row of zeros (eps carries it), a row of infinities, slots outside the pool skipped and reported."""
    from paper_2606_13740_gb300 import DllmError
    s = _serve(max_batch=1, max_rows=8, page=16, n_pages=2, max_pages=2, n_heads=4, n_kv_heads=2, head_dim=64)
    x = torch.randn(8, 8 * 64, device="cuda").to(torch.bfloat16)
    x[1] = 0
    x[2, :64] = float("inf")
    kc = torch.zeros(2, 2, 16, 64, device="cuda", dtype=torch.bfloat16)
    vc = torch.zeros_like(kc)
    s.slot.copy_(_i32([0, 1, 2, 3, 32, 1 << 30, -9, 31])), s.pos.copy_(_i32(list(range(8))))
    theta = torch.ones(32, device="cuda")
    apart = s.dllm_serve_qk_norm_rope(x[:, :256], x[:, 256:384], x[:, 384:], theta, kc, vc)
    k1 = kc.clone()
    with pytest.raises(DllmError, match="status bits 32"):
        s.dllm_serve_check()
    y = x.clone()
    s.dllm_serve_qk_norm_rope(y[:, :256], y[:, 256:384], y[:, 384:], theta, kc, vc, out=y[:, :256])
    assert torch.equal(y[:, :256].reshape(8, 4, 64).nan_to_num(7.0), apart.nan_to_num(7.0)) and torch.equal(kc, k1)
    assert torch.equal(y[:, 256:], x[:, 256:]) and bool((apart[1] == 0).all())
    assert bool(apart[2, 0].isnan().any()) and not bool(apart[2, 1:].isnan().any())
    used = torch.zeros(2, 16, dtype=torch.bool, device="cuda")
    for p in (0, 1, 2, 3, 31):
        used[p // 16, p % 16] = True
    assert bool((kc.transpose(1, 2)[~used] == 0).all()) and bool((kc[1, :, 15] != 0).any())


# ------------------------------------------------------------------ attention
class Paged:
    """A random batch over a pool whose unused places hold NaN and infinities."""

    def __init__(self, L, Q, P, page, H, Hkv, hd, dtype="bf16", causal=False, seed=0, spread=1.0, stride=0, pad=0,
                 refused=()):
        self.L, self.Q, self.P, self.page, self.H, self.Hkv, self.hd, self.causal = L, Q, P, page, H, Hkv, hd, causal
        g = torch.Generator(device="cuda").manual_seed(seed)
        need, npre = [-(-(a + b) // page) for a, b in zip(L, Q)], -(-P // page)
        n_pages = sum(need) + npre + 3
        N = sum(Q) + pad
        self.dtype = DT[dtype]
        self.s = _serve(max_batch=len(L), max_rows=max(N, 1), page=page, n_pages=n_pages, max_pages=max(need + [1]) + 1, n_heads=H,
                        n_kv_heads=Hkv, head_dim=hd, dtype=dtype, page_stride=stride)
        order = torch.randperm(n_pages, device="cuda", generator=g, dtype=torch.int32)
        self.s.ring.copy_(order)
        # the prefix's pages, taken off the ring by the program
        self.prefix = order[:npre].clone()
        self.s.ring_pos.copy_(_i32([npre, n_pages - npre]))
        dense = (Hkv * page * hd, page * hd, hd, 1)
        def cache():
            if stride:
                c = torch.empty(n_pages * stride, device="cuda", dtype=self.dtype).as_strided(
                    (n_pages, Hkv, page, hd), (stride,) + dense[1:])
            else:
                c = torch.empty(n_pages, Hkv, page, hd, device="cuda", dtype=self.dtype)
            c.fill_(float("nan"))
            return c
        self.kc, self.vc = cache(), cache()
        self.vc[:, :, 1::3] = float("inf")
        self.q = (torch.randn(N, H, hd, device="cuda", generator=g) * spread).to(self.dtype)
        self.s.dllm_serve_plan(_i32(L), _i32(Q), N, prefix_len=P, causal=causal)
        table = self.s.table.cpu().tolist()
        self.k, self.v = [], []  # own keys and values of a request [n][Hkv][hd]
        for b in range(-1, len(L)):
            n = P if b < 0 else L[b] + Q[b]
            k, v = (torch.randn(n, Hkv, hd, device="cuda", generator=g).to(self.dtype) for _ in range(2))
            pages = (self.prefix.cpu().tolist() if b < 0 else table[b])
            at = torch.tensor([pages[i // page] for i in range(n)], device="cuda", dtype=torch.long)
            off = torch.arange(n, device="cuda") % page
            self.kc[at, :, off], self.vc[at, :, off] = k, v
            self.k.append(k), self.v.append(v)

    def call(self, **kw):
        return self.s.dllm_serve_attention(self.q, self.kc, self.vc, self.prefix, **kw)

    def want(self, scale=None):
        """Output, sum of p |v| over the softmax, and lse, in 64 bits."""
        G, hd = self.H // self.Hkv, self.hd
        scale = hd ** -0.5 if scale is None else scale
        N = self.q.shape[0]
        out = torch.zeros(N, self.H, hd, dtype=torch.float64, device="cuda")
        size, lse = torch.zeros_like(out), torch.full((N, self.H), -math.inf, dtype=torch.float64, device="cuda")
        at = 0
        for b, (l, q) in enumerate(zip(self.L, self.Q)):
            k, v = (torch.cat([x[0], x[b + 1]]).double() for x in (self.k, self.v))
            if len(k) and q:
                k, v = (x.repeat_interleave(G, 1) for x in (k, v))
                z = torch.einsum("thd,khd->htk", self.q[at:at + q].double(), k) * scale
                if self.causal:
                    last = self.P + l + torch.arange(q, device="cuda")
                    z = z.masked_fill(torch.arange(len(k), device="cuda") > last[:, None], -math.inf)
                p = torch.softmax(z, -1)
                out[at:at + q] = torch.einsum("htk,khd->thd", p, v)
                size[at:at + q] = torch.einsum("htk,khd->thd", p, v.abs())
                lse[at:at + q] = torch.logsumexp(z, -1).T
            at += q
        return out.reshape(N, -1), size.reshape(N, -1), lse

    def check(self, **kw):
        out, lse = self.call(lse=True, **kw)
        self.s.dllm_serve_check()
        want, size, wlse = self.want(kw.get("scale"))
        u = U["bf16" if self.dtype == torch.bfloat16 else "f16"]
        keys = self.P + max([a + b for a, b in zip(self.L, self.Q)] + [0])
        # a rounding of the output, one of each probability (which in f16 lose what is below 2^-25 too), fp32 sums
        tol = u * want.abs() + (u + 2e-5) * size + (keys * 2.0 ** -25 if u < 2.0 ** -10 else 0.0)
        err = (out.double() - want).abs()
        assert bool((err <= tol).all()), float((err - tol).max())
        fin = torch.isfinite(wlse)
        assert torch.equal(fin, torch.isfinite(lse))
        assert bool(((lse.double() - wlse)[fin].abs() <= 2e-5 + 2e-6 * wlse[fin].abs()).all())
        # the mean error is that of roundings, not a bias
        if want.numel() > 1000:
            assert float(err.norm() / want.norm()) <= 1.2 * u
        return out


SHAPES = [(4, 4, 64), (28, 4, 128), (32, 32, 128), (16, 4, 64), (3, 1, 128), (128, 1, 64)]


@pytest.mark.parametrize("H,Hkv,hd", SHAPES)
@pytest.mark.parametrize("L,Q,P,page,causal", [
    ([0], [1], 0, 16, False),                          # one token that sees itself
    ([0, 0], [1, 0], 1, 16, False),                    # a prefix of one, a request without rows
    ([5], [1], 300, 64, False),
    ([0, 40, 63, 64, 65], [3, 1, 1, 1, 1], 100, 16, False),
    ([0, 100, 17], [32, 32, 32], 777, 32, False),      # windows
    ([130, 0, 2], [1, 200, 65], 64, 128, True),        # prompts and a token, causal
    ([700], [129], 0, 256, True),
    ([0] * 40, [1] * 40, 130, 16, False),              # many requests in one tile
])
def test_attention_matches_64_bits(dev, H, Hkv, hd, L, Q, P, page, causal):
    Paged(L, Q, P, page, H, Hkv, hd, causal=causal, seed=P + hd).check()


@pytest.mark.parametrize("dtype,spread", [("f16", 1.0), ("bf16", 12.0), ("f16", 12.0), ("bf16", 0.0)])
def test_attention_types_and_spreads(dev, dtype, spread):
    """f16, scores that leave one key standing, and equal ones."""
    Paged([900, 31, 0, 2000], [1, 32, 100, 7], 1500, 32, 28, 4, 128, dtype=dtype, seed=5, spread=spread).check()
    Paged([900, 31, 0], [1, 32, 100], 500, 16, 16, 4, 64, dtype=dtype, causal=True, seed=6, spread=spread).check()


def test_attention_long(dev):
    """Long prefixes and own contexts, split over many CTAs, in both directions of unevenness."""
    Paged([1, 9000, 20], [1, 1, 1], 20000, 64, 28, 4, 128, seed=7).check()
    Paged([30000], [1], 0, 16, 28, 4, 128, seed=8).check()
    Paged([0, 10], [900, 40], 6000, 64, 8, 8, 128, causal=True, seed=9).check()
    Paged([3] * 150, [2] * 150, 4097, 16, 16, 4, 64, seed=10).check()


def test_attention_rows_without_keys_and_padding(dev):
    """No prefix and a refused request: its rows see nothing; padding rows are zero; with a prefix a refused
    request sees that alone."""
    from paper_2606_13740_gb300 import DllmError
    for P in (0, 70):
        x = Paged([10, 0], [4, 6], P, 16, 4, 2, 64, pad=3, seed=11)
        x.s.ring_pos.copy_(_i32([0, 0]))
        x.s.held[1] = 0
        x.s.dllm_serve_plan(_i32([10, 0]), _i32([4, 6]), 13, prefix_len=P)
        with pytest.raises(DllmError):
            x.s.dllm_serve_check()
        x.k[2], x.v[2] = x.k[2][:0], x.v[2][:0]
        x.Q, x.L = [4, 6], [10, 0]
        out = x.check(out=torch.full((13, 256), 9.0, device="cuda", dtype=torch.bfloat16))
        assert bool((out[10:] == 0).all()) and (P > 0 or bool((out[4:10] == 0).all()))


def test_attention_keeps_requests_apart(dev):
    """NaN and infinities in one request's keys, values or queries stay in its rows."""
    x = Paged([30, 40, 50, 60], [2, 3, 1, 5], 200, 16, 28, 4, 128, seed=12)
    clean = x.check()
    table = x.s.table.cpu().tolist()
    x.vc[table[1][0], :, 3] = float("inf")
    x.kc[table[2][1], :, 2] = float("nan")
    x.q[9] = float("nan")
    out = x.call()
    ok = [0, 1] + [6, 7, 8, 10]
    assert torch.equal(out[ok], clean[ok])
    for bad in (2, 3, 4, 5, 9):
        assert bool((~torch.isfinite(out[bad])).any())


def test_attention_strides_scale_and_offsets_past_32_bits(dev):
    """q rows inside a wider array, a scale of its own, and pages 2^28 elements apart: 5 GB from the first."""
    x = Paged([50, 100], [30, 1], 64, 32, 28, 4, 128, seed=13)
    wide = torch.zeros(31, 40 * 128, device="cuda", dtype=torch.bfloat16)
    wide[:, 256:256 + 28 * 128] = x.q.view(31, -1)
    dense = x.check(scale=0.03)
    x.q = wide[:, 256:256 + 28 * 128].view(31, 28, 128)
    assert torch.equal(x.call(scale=0.03), dense)
    far = Paged([50, 100], [30, 1], 64, 32, 28, 4, 128, seed=13, stride=1 << 28)
    far.check()


def test_attention_repeats_its_bits_and_runs_in_a_graph_on_another_stream(dev):
    x = Paged([500, 0, 77], [1, 64, 32], 3000, 64, 32, 32, 128, seed=14)
    first = x.call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(first)
    L, Q = _i32([500, 0, 77]), _i32([1, 64, 32])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            x.s.dllm_serve_plan(L, Q, 97, prefix_len=3000)
            x.call(out=out)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
    x.s.dllm_serve_check()


def test_attention_reads_pages_outside_the_pool_as_zeros(dev):
    """Page numbers outside the pool, in a request's row or the prefix: zeros for keys and values, and a report."""
    from paper_2606_13740_gb300 import DllmError
    for page in (16, 64):
        x = Paged([20, 90], [2, 3], 70, page, 4, 2, 64, seed=16)
        clean = x.check()
        x.s.table[1, 0] = 1 << 30
        x.s.dllm_serve_plan(_i32([20, 90]), _i32([2, 3]), 5, prefix_len=70)
        out = x.call()
        with pytest.raises(DllmError, match="status bits 64"):
            x.s.dllm_serve_check()
        n = min(page, 93)
        x.k[2][:n] = 0
        x.v[2][:n] = 0
        want, size, _ = x.want()
        assert torch.equal(out[:2], clean[:2])
        assert bool(((out.double() - want).abs() <= U["bf16"] * want.abs() + (U["bf16"] + 2e-5) * size).all())
        bad = x.prefix.clone()
        bad[0] = -7
        x.s.dllm_serve_attention(x.q, x.kc, x.vc, bad)
        with pytest.raises(DllmError, match="status bits 16"):
            x.s.dllm_serve_check()


def test_attention_random_batches(dev):
    """Ragged batches at random: requests without rows, of one token and of many, causal or not, tiles that several
    requests share, pages of every size."""
    r = random.Random(17)
    for k in range(24):
        H, Hkv, hd = r.choice(SHAPES)
        B = r.choice([1, 2, 5, 23])
        top = r.choice([1, 9, 140])
        Q = [r.choice([0, 1, r.randint(1, top)]) for _ in range(B)]
        Q[r.randrange(B)] = top
        L = [r.choice([0, r.randint(0, 300)]) for _ in range(B)]
        Paged(L, Q, r.choice([0, 1, 63, 64, 500]), r.choice([16, 32, 64, 128, 256]), H, Hkv, hd, causal=r.random() < 0.5,
              dtype=r.choice(["bf16", "f16"]), seed=100 + k, pad=r.choice([0, 0, 4])).check()


def test_attention_without_a_plan_writes_zeros(dev):
    s = _serve(max_batch=2, max_rows=8, page=16, n_pages=4, max_pages=2, n_heads=4, n_kv_heads=2, head_dim=64)
    q = torch.ones(8, 4, 64, device="cuda", dtype=torch.bfloat16)
    kc = torch.ones(4, 2, 16, 64, device="cuda", dtype=torch.bfloat16)
    s.rows = 8
    out = s.dllm_serve_attention(q, kc, kc)
    s.dllm_serve_check()
    assert bool((out == 0).all())


def test_binding_refuses_what_does_not_fit(dev):
    x = Paged([10], [4], 40, 16, 4, 2, 64, seed=15)
    with pytest.raises(ValueError, match="rows"):
        x.s.dllm_serve_attention(x.q[:3], x.kc, x.vc, x.prefix)
    with pytest.raises(ValueError, match="prefix"):
        x.s.dllm_serve_attention(x.q, x.kc, x.vc, x.prefix[:2])
    with pytest.raises(ValueError, match="strides"):
        x.s.dllm_serve_attention(x.q.transpose(0, 1).contiguous().transpose(0, 1), x.kc, x.vc, x.prefix)
    with pytest.raises(ValueError):
        x.s.dllm_serve_attention(x.q.half(), x.kc, x.vc, x.prefix)
    with pytest.raises(ValueError):
        x.s.dllm_serve_attention(x.q, x.kc[:, :, :8], x.vc, x.prefix)
    with pytest.raises(ValueError):
        x.s.dllm_serve_plan(torch.zeros(1, device="cuda"), _i32([1]), 1)


# ------------------------------------------------------------------ logits
def _logits_case(N, V, R, dtype, seed, hist=300, nb=20):
    g = np.random.default_rng(seed)
    z = torch.from_numpy((g.standard_normal((N, V)) * 3).astype(np.float32)).to(DT[dtype])
    req = np.sort(g.integers(0, R, N)).astype(np.int32)
    h = g.integers(0, max(2, V // 3), (R, hist)).astype(np.int32)
    h[:, ::17] = V + 5  # no ids: skipped
    h[:, 5::29] = -1
    hl = g.integers(0, hist + 1, R).astype(np.int32)
    ids = g.integers(0, V, (R, nb)).astype(np.int32)
    if nb > 3:
        ids[:, 3] = ids[:, 1]  # the later one counts
    words = (V + 31) // 32
    return dict(z=z, req=req, hist=h, hist_len=hl, rep=(1 + 0.5 * g.random(R)).astype(np.float32),
                freq=(0.3 * g.random(R)).astype(np.float32), pres=(0.3 * g.random(R)).astype(np.float32), bias_ids=ids,
                bias=(2 * g.standard_normal((R, nb))).astype(np.float32), bias_len=g.integers(0, nb + 1, R).astype(np.int32),
                grammar=g.integers(0, 2 ** 32, (3, words), dtype=np.uint64).astype(np.uint32),
                grammar_row=g.integers(-1, 3, N).astype(np.int32), cur=g.integers(0, V, N).astype(np.int32))


def _logits_want(c, mask_id):
    """z in fp32, operation by operation; the decision in 64 bits from it."""
    z = c["z"].float().numpy().copy()
    N, V = z.shape
    f = np.float32
    for n in range(N):
        r = c["req"][n]
        if 0 <= r < len(c["hist_len"]):
            h = c["hist"][r, :c["hist_len"][r]]
            ids, cnt = np.unique(h[(h >= 0) & (h < V)], return_counts=True)
            w = z[n, ids]
            with np.errstate(all="ignore"):
                w = np.where(w > 0, w / c["rep"][r], w * c["rep"][r]).astype(f)
                z[n, ids] = w - (c["freq"][r] * cnt.astype(f) + c["pres"][r])
            last = {int(i): c["bias"][r, k] for k, i in enumerate(c["bias_ids"][r, :c["bias_len"][r]])}
            for i, v in last.items():
                if 0 <= i < V:
                    z[n, i] = z[n, i] + v
        g = c["grammar_row"][n]
        if g >= 0:
            ok = np.unpackbits(c["grammar"][g].view(np.uint8), bitorder="little")[:V].astype(bool)
            z[n, ~ok] = -np.inf
    d = z.astype(np.float64)
    if mask_id >= 0:
        d[:, mask_id] = -np.inf
    x0 = np.full(N, -1)
    conf, tok = np.zeros(N), np.zeros(N)
    for n in range(N):
        m = np.nanmax(d[n]) if not np.isnan(d[n]).all() else -np.inf
        if m > -np.inf:
            x0[n] = int(np.argmax(np.where(np.isnan(d[n]), -np.inf, d[n]) == m))
        with np.errstate(all="ignore"):
            e = np.exp(d[n] - (m if m > -np.inf else 0.0))
        if e.sum() != 0:
            conf[n] = 1 / e.sum()
            cur = c["cur"][n]
            tok[n] = e[cur] / e.sum() if 0 <= cur < V and cur != mask_id else 0.0
    return z, x0, conf, tok


def _logits_run(c, mask_id, out=True, inplace=False, ld=0, **drop):
    from paper_2606_13740_gb300 import serve
    N, V = c["z"].shape
    z = c["z"].cuda()
    if ld:  # rows farther apart, from an odd place on
        wide = torch.zeros(N, ld, dtype=z.dtype, device="cuda")
        wide[:, 1:V + 1] = z
        z = wide[:, 1:V + 1]
    t = {k: torch.from_numpy(v.view(np.int32) if v.dtype == np.uint32 else v).cuda() for k, v in c.items() if k != "z"}
    t.update(drop)
    o = z if inplace else (torch.empty_like(c["z"], device="cuda") if out else None)
    x0, conf, tok = serve.dllm_serve_logits(z, mask_id, out=o, **t)
    return None if o is None else o.float().cpu().numpy(), x0.cpu().numpy(), conf.cpu().numpy(), tok.cpu().numpy()


def _logits_check(c, mask_id, **kw):
    z, x0, conf, tok = _logits_want(c, mask_id)
    gz, gx0, gconf, gtok = _logits_run(c, mask_id, **kw)
    if gz is not None:
        assert np.array_equal(gz, torch.from_numpy(z).to(c["z"].dtype).float().numpy(), equal_nan=True)
    assert np.array_equal(gx0, x0)
    # an exponential's argument is rounded (|z - max| < 64 in log2 units: 2^-18), and fp32 sums
    for got, want in ((gconf, conf), (gtok, tok)):
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.all(np.abs(got - want)[~np.isnan(want)] <= 1e-5 * want[~np.isnan(want)] + 1e-30)


@pytest.mark.parametrize("N,V,R,dtype", [
    (1, 1, 1, "f32"), (1, 2, 1, "f32"), (3, 33, 2, "bf16"), (1, 126464, 1, "f32"), (5, 8192, 5, "f16"), (7, 8193, 3, "f32"),
    (64, 1024, 2, "f32"), (33, 20001, 4, "bf16"), (100, 5000, 100, "f32"), (9, 152064, 2, "bf16"),
])
def test_logits_match_definition(dev, N, V, R, dtype):
    c = _logits_case(N, V, R, dtype, N + V)
    _logits_check(c, V - 1)
    _logits_check(c, -1, out=False)
    _logits_check(c, 0, inplace=True)
    _logits_check(c, V // 2, ld=V + 3)


def test_logits_ties_masks_and_infinities(dev):
    V = 9000
    c = _logits_case(8, V, 8, "f32", 3)
    c["req"] = np.array([0, 1, 2, -1, 99, 5, 6, 7], np.int32)  # rows without a request among them
    c["z"][0] = 1.5                      # all alike but for penalties
    c["z"][1, 100] = float("nan")        # hidden by the grammar below
    c["z"][2, 7] = float("nan")          # not hidden
    c["z"][3] = torch.finfo(torch.float32).min
    c["z"][5, 3:] = float("-inf")
    c["z"][6, 8500] = float("inf")
    c["grammar_row"][:] = [-1, 0, -1, -1, 1, -1, 2, -1]
    c["grammar"][0, 100 // 32] &= ~np.uint32(1 << (100 % 32))
    c["grammar"][1] = 0                  # nothing allowed
    c["grammar"][2] = 0xffffffff
    c["hist_len"][5] = c["bias_len"][5] = c["hist_len"][6] = c["bias_len"][6] = 0
    c["hist"][7], c["hist_len"][7] = 77, c["hist"].shape[1]  # one id, three hundred times
    c["cur"][:] = [V - 1, 5, 7, 8, 9, 4, 8500, 77]
    _logits_check(c, V - 1)
    assert _logits_run(c, V - 1)[1][4] == -1


def test_logits_without_lists(dev):
    """Only what is given applies; without req there is a list for each row."""
    from paper_2606_13740_gb300 import serve
    c = _logits_case(6, 3001, 6, "f32", 4)
    c["req"] = np.arange(6, dtype=np.int32)
    z = c["z"].cuda()
    out = torch.empty_like(z)
    x0, conf, tok = serve.dllm_serve_logits(z, out=out)
    assert torch.equal(out, z) and tok is None and torch.equal(x0.long(), z.argmax(1))
    assert torch.allclose(conf, torch.softmax(z, 1).amax(1), rtol=1e-5, atol=0)
    plain = dict(c, bias_len=np.zeros(6, np.int32), grammar_row=np.full(6, -1, np.int32))
    _logits_check(plain, -1, req=None, bias_ids=None, bias=None, bias_len=None, grammar=None, grammar_row=None)
    with pytest.raises(ValueError):
        serve.dllm_serve_logits(z, rep=torch.ones(6, device="cuda"))
    with pytest.raises(ValueError):
        serve.dllm_serve_logits(z, hist=torch.zeros(5, 3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        serve.dllm_serve_logits(z.T)
    assert serve.dllm_serve_logits(z[:0])[0].numel() == 0


def test_logits_more_rows_than_a_grid_dimension(dev):
    from paper_2606_13740_gb300 import serve
    z = torch.randn(70000, 40, device="cuda")
    x0, conf, _ = serve.dllm_serve_logits(z)
    assert torch.equal(x0.long(), z.argmax(1)) and torch.allclose(conf, torch.softmax(z, 1).amax(1), rtol=1e-5, atol=0)
