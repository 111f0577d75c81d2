"""Trees, attention by bits, accepted paths, compaction, forks and log probabilities on the GPU, against plain
implementations: whole numbers and moved values in plain Python, the others in 64 bits."""
import math
import random

import pytest

torch = pytest.importorskip("torch")
from test_gpu_serve import DT, SHAPES, U, Paged, _i32, _serve, dev  # noqa: E402,F401

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def _tree_of(r, q, back=8, roots=0.0):
    return [-1 if i == 0 or r.random() < roots else r.randint(max(0, i - back), i - 1) for i in range(q)]


def _seen(tree):
    out = []
    for i, p in enumerate(tree):
        out.append((out[p] if p >= 0 else 0) | 1 << i)
    return out


def _signed(words):
    return [w - (1 << 32) if w >= 1 << 31 else w for w in words]


def _words(bits, words):
    return _signed([bits >> 32 * k & 0xffffffff for k in range(words)])


# ------------------------------------------------------------------ tree
@pytest.mark.parametrize("q,words,extra", [
    ([1], 1, 0), ([0, 1, 0, 31, 32, 33, 64, 65, 0], 3, 4), ([500, 3], 16, 0), ([2100, 5], 66, 1), ([1] * 700, 1, 5),
    ([5, 9] * 1200, 2, 0),
])
def test_tree_bits_and_positions(dev, q, words, extra):
    r = random.Random(sum(q))
    B, N, P = len(q), sum(q) + extra, 11
    L = [r.randint(0, 40) for _ in q]
    page = 16
    need = [-(-(a + b) // page) for a, b in zip(L, q)]
    s = _serve(max_batch=B + 2, max_rows=N + 3, page=page, n_pages=sum(need) + 1, max_pages=max(need), n_heads=2, n_kv_heads=2, head_dim=64)
    trees = [_tree_of(r, n, r.choice([1, 3, 50]), 0.1) for n in q]
    parent = _i32([p for t in trees for p in t] + [7] * extra)
    s.dllm_serve_plan(_i32(L), _i32(q), N, prefix_len=P)
    plain = s.pos.cpu().tolist()
    for _ in range(2):  # (positions are made from the plan's first one, which stays)
        mask = s.dllm_serve_tree(parent, 32 * words)
        bits = [b for t in trees for b in _seen(t)]
        assert mask.cpu().tolist() == [_words(b, words) for b in bits] + [[0] * words] * extra
        want = [P + l + bin(b).count("1") - 1 for l, t in zip(L, trees) for b in _seen(t)]
        assert s.pos.cpu().tolist() == want + plain[sum(q):]
    s.dllm_serve_check()


def test_tree_refuses_what_is_no_tree(dev):
    """Parents that are not earlier tokens, trees of more tokens than bits: that request gets no bits and keeps its
    positions, the others are as ever; refused requests keep position 0."""
    from paper_2606_13740_gb300 import DllmError
    q = [3, 40, 4, 2, 5]
    s = _serve(max_batch=5, max_rows=60, page=16, n_pages=8, max_pages=3, n_heads=2, n_kv_heads=2, head_dim=64)
    s.dllm_serve_plan(_i32([0, 1, 0, -4, 6]), _i32(q), 54)
    with pytest.raises(DllmError, match="status bits 2"):
        s.dllm_serve_check()
    plain = s.pos.cpu().tolist()
    for wrong in (2, 3, -2, 1 << 30, -(1 << 31)):
        trees = [[-1, 0, 0], [-1] + list(range(39)), [-1, 0, wrong, 0], [-1, 0], [-1, 0, 0, 2, 2]]
        mask = s.dllm_serve_tree(_i32([p for t in trees for p in t]), 32).cpu().tolist()
        assert mask[:3] == [[1], [3], [5]] and mask[3:47] == [[0]] * 44 and mask[47:] == [[1], [3], [1], [3], [5], [13], [21]]
        got = s.pos.cpu().tolist()
        assert got[:3] == [0, 1, 1] and got[3:49] == plain[3:49] and got[47:49] == [0, 0] and got[49:54] == [6, 7, 7, 8, 8]
        with pytest.raises(DllmError, match="status bits 128"):
            s.dllm_serve_check()


def test_tree_and_accept_without_a_plan(dev):
    s = _serve(max_batch=2, max_rows=8, page=16, n_pages=4, max_pages=2, n_heads=4, n_kv_heads=2, head_dim=64)
    s.rows = 8
    parent = _i32([-1] * 8)
    assert not bool(s.dllm_serve_tree(parent, 40).any())
    keep, n, nxt = s.dllm_serve_accept(parent, parent, parent, 2, 3)
    s.dllm_serve_check()
    assert bool((keep == -1).all()) and n.cpu().tolist() == [0, 0] and nxt.cpu().tolist() == [-1, -1]


# ------------------------------------------------------------------ attention by bits
class Tree(Paged):
    """Paged with bits for the new tokens: those of trees, or any."""

    def __init__(self, L, Q, P, page, H, Hkv, hd, form="tree", words=None, **kw):
        super().__init__(L, Q, P, page, H, Hkv, hd, **kw)
        r = random.Random(kw.get("seed", 0))
        self.words = words or max(1, -(-max(Q + [1]) // 32))
        self.bits = []
        for q in Q:
            if form == "tree":
                self.bits += _seen(_tree_of(r, q, roots=0.1))
            else:
                self.bits += [0 if r.random() < 0.1 else r.getrandbits(32 * self.words) for _ in range(q)]
        if form == "all":
            self.bits = [(1 << 32 * self.words) - 1] * sum(Q)
        rows = [_words(b, self.words) for b in self.bits]
        self.mask = _i32(rows + [[-1] * self.words] * (self.q.shape[0] - len(rows)))

    def call(self, **kw):
        return self.s.dllm_serve_tree_attention(self.q, self.kc, self.vc, self.mask, self.prefix, **kw)

    def check(self, **kw):
        if self.P + sum(self.L) == 0 and len(self.bits) == 1 and not self.bits[0] & 1:
            # nothing to see at all: no mean error to speak of (0 / 0), but zeros
            out, lse = self.call(lse=True, **kw)
            self.s.dllm_serve_check()
            assert bool((out == 0).all()) and bool((lse == -INF).all())
            return out
        return super().check(**kw)

    def want(self, scale=None):
        G, hd = self.H // self.Hkv, self.hd
        scale = hd ** -0.5 if scale is None else scale
        N = self.q.shape[0]
        out = torch.zeros(N, self.H, hd, dtype=torch.float64, device="cuda")
        size, lse = torch.zeros_like(out), torch.full((N, self.H), -math.inf, dtype=torch.float64, device="cuda")
        at = 0
        for b, (l, q) in enumerate(zip(self.L, self.Q)):
            k, v = (torch.cat([x[0], x[b + 1]]).double() for x in (self.k, self.v))
            for t in range(q if len(k) else 0):
                sees = torch.ones(len(k), dtype=torch.bool)
                for j in range(min(q, len(k) - self.P - l)):
                    sees[self.P + l + j] = bool(self.bits[at + t] >> j & 1) and (j <= t or not self.causal)
                sees = sees.cuda()
                if bool(sees.any()):
                    ks, vs = (x[sees].repeat_interleave(G, 1) for x in (k, v))
                    z = torch.einsum("hd,khd->hk", self.q[at + t].double(), ks) * scale
                    p = torch.softmax(z, -1)
                    out[at + t], size[at + t] = torch.einsum("hk,khd->hd", p, vs), torch.einsum("hk,khd->hd", p, vs.abs())
                    lse[at + t] = torch.logsumexp(z, -1)
            at += q
        return out.reshape(N, -1), size.reshape(N, -1), lse


@pytest.mark.parametrize("H,Hkv,hd", SHAPES)
@pytest.mark.parametrize("L,Q,P,page,form", [
    ([0], [1], 0, 16, "tree"),
    ([0], [1], 0, 16, "any"),
    ([5], [26], 300, 64, "tree"),
    ([63, 64, 65, 0, 1], [1, 3, 70, 0, 130], 0, 16, "any"),
    ([130, 0, 2], [1, 200, 65], 64, 128, "tree"),
    ([0] * 40, [2] * 40, 130, 16, "tree"),
])
def test_tree_attention_matches_64_bits(dev, H, Hkv, hd, L, Q, P, page, form):
    Tree(L, Q, P, page, H, Hkv, hd, form=form, seed=P + hd).check()


def test_tree_attention_of_rows_that_see_nothing(dev):
    """No prefix, nothing cached and no bits: zeros and -inf, padding rows too; with a causal plan bits past the row
    itself say nothing."""
    x = Tree([0, 3, 0], [70, 5, 2], 0, 16, 16, 4, 64, form="any", seed=3, pad=4)
    x.bits[0] = x.bits[69] = 0
    x.bits[75], x.bits[76] = 4, 1 << 63 | 2  # of two tokens: none of them, the second
    x.mask[0] = x.mask[69] = 0
    x.mask[75:77] = _i32([_words(x.bits[75], 3), _words(x.bits[76], 3)])
    out = x.check(out=torch.full((81, 1024), 9.0, device="cuda", dtype=torch.bfloat16))
    assert all(bool((out[n] == 0).all()) for n in (0, 69, 75, 77, 80)) and bool((out[70] != 0).any())
    for seed in (4, 5):
        Tree([0, 30, 100], [90, 5, 130], 20, 32, 28, 4, 128, form="any", seed=seed, causal=True).check()


def test_tree_attention_with_every_bit_is_attention(dev):
    """The same bits of output, causal or not; words of fewer tokens than there are leave the others out."""
    for causal in (False, True):
        x = Tree([40, 0, 500], [33, 100, 7], 200, 32, 28, 4, 128, form="all", seed=6, causal=causal)
        assert torch.equal(x.check(), Paged.call(x))
    x = Tree([40, 0], [33, 100], 0, 32, 4, 2, 64, form="any", words=1, seed=7)
    x.check()


def test_tree_attention_of_a_long_chain_is_causal_attention(dev):
    """A chain of 2100 tokens: by the bits alone, and after a causal plan bit for bit what the plan alone gives."""
    def chain(x):
        at, rows = 0, []
        for q in x.Q:
            rows += [_words((2 << t) - 1, x.words) for t in range(q)]
        x.mask = _i32(rows)
        return x

    a = chain(Tree([100, 7], [2100, 65], 70, 64, 8, 2, 128, form="all", seed=21, causal=True))
    b = chain(Tree([100, 7], [2100, 65], 70, 64, 8, 2, 128, form="all", seed=21))
    want = Paged.call(a)
    assert torch.equal(a.call(), want)
    # the same sums in blocks cut otherwise: a rounding of P and one of the output each, of values of size 1 or so
    assert float((b.call().double() - want.double()).norm() / want.double().norm()) <= 2 * 1.2 * U["bf16"]


@pytest.mark.parametrize("dtype,spread", [("f16", 1.0), ("bf16", 12.0), ("f16", 12.0), ("bf16", 0.0)])
def test_tree_attention_types_and_spreads(dev, dtype, spread):
    Tree([900, 31, 0, 2000], [1, 32, 100, 7], 1500, 32, 28, 4, 128, dtype=dtype, seed=5, spread=spread).check()
    Tree([900, 31, 0], [1, 32, 100], 500, 16, 16, 4, 64, dtype=dtype, form="any", seed=6, spread=spread).check()


def test_tree_attention_keeps_what_a_row_does_not_see_from_it(dev):
    """Infinities and NaN in keys and values of a token: they reach the rows that see it, and no others."""
    for hd, page in ((64, 16), (128, 64)):
        x = Tree([70, 10], [150, 20], 100, page, 8, 2, hd, form="any", seed=8)
        clean = x.check()
        table = x.s.table.cpu().tolist()
        for j, what in ((3, NAN), (77, INF), (149, NAN)):
            at = 70 + j
            x.vc[table[0][at // page], :, at % page, 5] = what
            out = x.call()
            sees = torch.tensor([b >> j & 1 for b in x.bits[:150]], dtype=torch.bool, device="cuda")
            assert torch.equal(out[:150][~sees], clean[:150][~sees]) and torch.equal(out[150:], clean[150:])
            hit = out[:150].view(150, 8, hd)[sees]
            assert bool((~torch.isfinite(hit[..., 5])).all()) and bool(torch.isfinite(hit[..., 6]).all())
            x.vc[table[0][at // page], :, at % page, 5] = 0.5
            x.kc[table[0][at // page], :, at % page] = what
            out = x.call()
            assert torch.equal(out[150:], clean[150:]) and bool(torch.isfinite(out[:150][~sees]).all())
            x.kc[table[0][at // page], :, at % page] = 0.5
            clean = x.call()
        x.s.dllm_serve_check()


def test_tree_attention_random_batches(dev):
    r = random.Random(18)
    for k in range(24):
        H, Hkv, hd = r.choice(SHAPES)
        B, top = r.choice([1, 2, 5, 23]), r.choice([1, 9, 140])
        Q = [r.choice([0, 1, r.randint(1, top)]) for _ in range(B)]
        Q[r.randrange(B)] = top
        L = [r.choice([0, r.randint(0, 300)]) for _ in range(B)]
        Tree(L, Q, r.choice([0, 1, 63, 64, 500]), r.choice([16, 32, 64, 128, 256]), H, Hkv, hd, causal=r.random() < 0.3,
             form=r.choice(["tree", "any"]), dtype=r.choice(["bf16", "f16"]), seed=200 + k, pad=r.choice([0, 0, 4]),
             words=r.choice([None, -(-top // 32) + 2])).check()


# ------------------------------------------------------------------ accept
def _path(tree, ids, x0, most):
    path, nxt = ([0] if tree else []), -1
    while path:
        nxt = x0[path[-1]]
        step = [c for c in range(path[-1] + 1, len(tree)) if tree[c] == path[-1] and ids[c] == nxt]
        if len(path) == most or not step:
            break
        path.append(step[0])
    return path, nxt


@pytest.mark.parametrize("q,most,back", [([26], 16, 8), ([0, 1, 5, 100, 0, 33, 64, 2], 6, 8), ([700], 800, 1), ([9] * 300, 1, 3)])
def test_accept_follows_the_decisions(dev, q, most, back):
    r = random.Random(len(q) * 7 + most)
    s = _serve(max_batch=len(q) + 3, max_rows=sum(q) + 9, page=64, n_pages=len(q) + 50, max_pages=20, n_heads=2, n_kv_heads=2, head_dim=64)
    for ids_of in (3, 40):
        trees = [_tree_of(r, n, back) for n in q]
        ids = [[r.randrange(ids_of) for _ in t] for t in trees]
        x0 = []
        for t, d in zip(trees, ids):
            kids = [[c for c in range(len(t)) if t[c] == i] for i in range(len(t))]
            x0.append([d[r.choice(k)] if k and r.random() < 0.97 else r.randrange(ids_of) for k in kids])
        s.dllm_serve_plan(_i32([3] * len(q)), _i32(q), sum(q) + 2)
        flat = [_i32([x for t in v for x in t] + [0, 0]) for v in (trees, ids, x0)]
        keep, n, nxt = s.dllm_serve_accept(*flat, len(q) + 1, most)  # (a request past the plan's batch: nothing)
        want = [_path(t, i, x, most) for t, i, x in zip(trees, ids, x0)] + [([], -1)]
        assert n.cpu().tolist() == [len(p) for p, _ in want] and nxt.cpu().tolist() == [x for _, x in want]
        assert keep.cpu().tolist() == [p + [-1] * (most - len(p)) for p, _ in want]
        s.dllm_serve_check()


# ------------------------------------------------------------------ pages
class Caches:
    """Requests whose own positions lie in pages of a small pool, in some layers."""

    def __init__(self, L, page, layers=2, Hkv=3, hd=64, dtype="bf16", seed=0, spare=2, stride=0, batch=None):
        self.L, self.page = L, page
        need = [-(-n // page) for n in L]
        n_pages = sum(need) + spare
        self.s = _serve(max_batch=batch or len(L), max_rows=max(1, sum(L)), page=page, n_pages=n_pages, max_pages=max(need + [1]) + 1,
                        n_heads=Hkv, n_kv_heads=Hkv, head_dim=hd, dtype=dtype, page_stride=stride)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.s.ring.copy_(torch.randperm(n_pages, device="cuda", generator=g, dtype=torch.int32))
        self.s.dllm_serve_plan(_i32(L), _i32([0] * len(L)), 0)

        def cache():
            if not stride:
                return torch.randn(n_pages, Hkv, page, hd, device="cuda", generator=g).to(DT[dtype])
            c = torch.zeros(n_pages * stride, device="cuda", dtype=DT[dtype])
            c = c.as_strided((n_pages, Hkv, page, hd), (stride, page * hd, hd, 1))
            return c.copy_(torch.randn(n_pages, Hkv, page, hd, device="cuda", generator=g))

        self.k, self.v = [cache() for _ in range(layers)], [cache() for _ in range(layers)]
        self.layers = self.s.layers(self.k, self.v)

    def copy(self):
        return [c.clone() for c in self.k + self.v]

    def same(self, want):
        assert all(torch.equal(a, b) for a, b in zip(self.k + self.v, want))


def _compacted(x, caches, table, first, keep):
    for c in caches:
        new = c.clone()
        for b, (f, ks) in enumerate(zip(first, keep)):
            for i, k in enumerate(ks):
                src, dst = f + k, f + i
                new[table[b][dst // x.page], :, dst % x.page] = c[table[b][src // x.page], :, src % x.page]
        c.copy_(new)
    return caches


@pytest.mark.parametrize("hd,dtype,stride", [(64, "bf16", 0), (128, "f16", 0), (128, "bf16", 3 * 64 * 128 + 8)])
@pytest.mark.parametrize("page", [16, 64])
def test_compact_moves_what_is_kept(dev, hd, dtype, stride, page):
    r = random.Random(page + hd)
    L = [0, 1, 5, 16, 17, 300, 129, 64]
    x = Caches(L, page, hd=hd, dtype=dtype, stride=stride, seed=1)
    table = x.s.table.cpu().tolist()
    for _ in range(4):
        first = [r.choice([0, r.randint(0, n)]) for n in L]
        keep = [sorted(r.sample(range(n - f), r.choice([0, n - f, r.randint(0, n - f)]))) for n, f in zip(L, first)]
        most = max(map(len, keep)) + 1
        want = _compacted(x, x.copy(), table, first, keep)
        x.s.dllm_serve_compact(x.layers, _i32(first), _i32([k + [9] * (most - len(k)) for k in keep]), _i32([len(k) for k in keep]))
        x.s.dllm_serve_check()
        x.same(want)
    assert x.s.table.cpu().tolist() == table


@pytest.mark.parametrize("hd", [64, 128])
def test_compact_of_short_lists(dev, hd):
    """Lists of up to 64 places, in steps of one warp; more requests than are asked for; no requests that move."""
    r = random.Random(hd)
    L = [r.randint(0, 90) for _ in range(37)]
    x = Caches(L, 16, hd=hd, layers=3, Hkv=1, seed=3)
    table = x.s.table.cpu().tolist()
    for most in (1, 16, 17, 64):
        keep = [sorted(r.sample(range(n), min(n, r.choice([0, 1, most, r.randint(0, most)])))) for n in L[:30]]
        want = _compacted(x, x.copy(), table, [0] * 30, keep)
        x.s.dllm_serve_compact(x.layers, _i32([0] * 30), _i32([k + [-1] * (most - len(k)) for k in keep]), _i32([len(k) for k in keep]))
        x.s.dllm_serve_check()
        x.same(want)
    x.s.dllm_serve_compact(x.layers, _i32([0] * 30), torch.zeros(30, 0, device="cuda", dtype=torch.int32), _i32([0] * 30))
    x.s.dllm_serve_check()
    x.same(want)


def test_compact_leaves_out_what_makes_no_sense(dev):
    """Lists that do not ascend, places past the request's, a wrong count: that request stays, the others are done."""
    from paper_2606_13740_gb300 import DllmError
    x = Caches([40, 40, 0], 16, seed=2)
    table = x.s.table.cpu().tolist()
    good = list(range(0, 40, 2))
    for first, keep, n in ((0, [3, 2, 5], 3), (0, [3, 3, 5], 3), (0, [-1, 2, 3], 3), (9, [1, 2, 39], 3), (0, [1, 2, 48], 3),
                           (-1, [1, 2, 3], 3), (0, [1, 2, 3], 21), (0, [1, 2, 3], -1), (2 ** 31 - 1, [1, 2, 3], 3),
                           (0, [1, 2, 2 ** 31 - 1], 3), (0, list(range(1, 19)) + [18, 20], 20)):
        want = _compacted(x, x.copy(), table, [0, 0], [[], good])
        x.s.dllm_serve_compact(x.layers, _i32([first, 0, 0]), _i32([keep + [0] * (20 - len(keep)), good, good]), _i32([n, 20, 0]))
        with pytest.raises(DllmError, match="status bits 128"):
            x.s.dllm_serve_check()
        x.same(want)
    want = x.copy()
    x.s.dllm_serve_compact(x.layers, _i32([0, 0, 0]), _i32([good] * 3), _i32([0, 0, 1]))  # a place that it does not hold
    with pytest.raises(DllmError, match="status bits 128"):
        x.s.dllm_serve_check()
    x.s.table[0, 1] = 1 << 20  # a page that is not of the pool
    x.s.dllm_serve_compact(x.layers, _i32([0, 0, 0]), _i32([good] * 3), _i32([20, 0, 0]))
    with pytest.raises(DllmError, match="status bits 64"):
        x.s.dllm_serve_check()
    x.same(want)


class Forks:
    """The fork's definition in plain Python, on a pool's state."""

    def __init__(self, s, page):
        self.page, self.n = page, s.cfg.n_pages
        held, table = s.held.cpu().tolist(), s.table.cpu().tolist()
        self.rows = [t[:h] for t, h in zip(table, held)]
        head, count = s.ring_pos.cpu().tolist()
        ring = s.ring.cpu().tolist()
        self.free = [ring[(head + i) % self.n] for i in range(count)]

    def fork(self, src, length):
        """Copies (page, its copy, places), or None: refused."""
        B, page = len(src), self.page
        if any(not 0 <= s < len(self.rows) or n < 0 or -(-n // page) > len(self.rows[s]) for s, n in zip(src, length)):
            return None
        new = [list(self.rows[s][:-(-n // page)]) for s, n in zip(src, length)]
        whole = set(p for r in self.rows[B:] for p in r)
        whole |= set(p for r, n in zip(new, length) for p in r[:n // page])
        writer, copies = {}, []
        for b, n in enumerate(length):
            if n % page:
                writer.setdefault(new[b][-1], b)
        for b, n in enumerate(length):
            if n % page and (new[b][-1] in whole or writer[new[b][-1]] != b):
                if len(copies) == len(self.free):
                    return None
                copies.append((new[b][-1], self.free[len(copies)], n % page))
                new[b][-1] = copies[-1][1]
        before = set(p for r in self.rows for p in r)
        self.rows[:B] = new
        self.free = self.free[len(copies):] + sorted(before - set(p for r in self.rows for p in r))
        return copies

    def same(self, s):
        table, held = s.table.cpu().tolist(), s.held.cpu().tolist()
        for b, row in enumerate(self.rows):
            assert held[b] == len(row) and table[b] == row + [-1] * (len(table[b]) - len(row)), b
        head, count = s.ring_pos.cpu().tolist()
        ring = s.ring.cpu().tolist()
        assert [ring[(head + i) % self.n] for i in range(count)] == self.free


@pytest.mark.parametrize("B,batch,page,hd,most,spare,steps", [
    (1, 1, 16, 64, 40, 3, 6), (4, 4, 16, 64, 70, 20, 12), (6, 9, 32, 128, 100, 12, 10), (40, 40, 16, 64, 200, 90, 6),
    (300, 310, 16, 64, 33, 500, 4), (1500, 1500, 16, 64, 20, 1000, 3),
])
def test_fork_matches_its_definition(dev, B, batch, page, hd, most, spare, steps):
    """Beams over some steps: shared, copied and given back, plans in between, requests past the batch, and forks that
    cannot be carried out."""
    from paper_2606_13740_gb300 import DllmError
    r = random.Random(B)
    x = Caches([r.randint(0, most) for _ in range(batch)], page, layers=2 if B < 50 else 1, Hkv=2 if B < 50 else 1, hd=hd,
               spare=spare, seed=B)
    ref = Forks(x.s, page)
    for step in range(steps):
        have = [len(row) * page for row in ref.rows]
        src = [r.choice([b, r.randrange(batch), 0]) for b in range(B)]
        length = [r.choice([have[c], r.randint(0, have[c]), have[c] // page * page, 0]) for c in src]
        if step % 4 == 3:
            src[r.randrange(B)], wrong = r.choice([-1, batch, 1 << 31 - 1, 0]), r.randrange(B)
            length[wrong] = r.choice([-1, (1 << 31) - 1, length[wrong] + 10 ** 6])
        want = x.copy()
        copies = ref.fork(src, length)
        x.s.dllm_serve_fork(x.layers, _i32(src), _i32(length))
        status = x.s.status.cpu().tolist()
        if copies is None:
            with pytest.raises(DllmError):
                x.s.dllm_serve_check()
            assert status[1:] == [B, 0, 0]
        else:
            x.s.dllm_serve_check()
            assert status[1] == 0 and status[2] == len(copies) and x.s.n_keys.cpu().tolist()[:B] == length
            for a, b, n in copies:
                for c in want:
                    c[b, :, :n] = c[a, :, :n]
        x.same(want)
        ref.same(x.s)


def test_pages_past_32_bits(dev):
    """Pages 2^28 elements apart, 3 GB from the first: compaction and fork."""
    x = Caches([70, 33], 16, layers=1, Hkv=1, hd=128, stride=1 << 28, seed=9, spare=3)
    table = x.s.table.cpu().tolist()

    def dense():
        return [c[:].clone(memory_format=torch.contiguous_format) for c in x.k + x.v]

    want = _compacted(x, dense(), table, [0, 1], [list(range(1, 70, 3)), [4, 8]])
    x.s.dllm_serve_compact(x.layers, _i32([0, 1]), _i32([list(range(1, 70, 3)), [4, 8] + [0] * 21]), _i32([23, 2]))
    x.s.dllm_serve_check()
    x.same(want)
    ref = Forks(x.s, 16)
    copies = ref.fork([0, 0], [70, 69])
    for a, b, n in copies:
        for c in want:
            c[b, :, :n] = c[a, :, :n]
    x.s.dllm_serve_fork(x.layers, _i32([0, 0]), _i32([70, 69]))
    x.s.dllm_serve_check()
    x.same(want)
    ref.same(x.s)


@pytest.mark.parametrize("B,most,spare", [(4096, 20, 3000), (5, 50000, 4000)])
def test_fork_of_the_largest(dev, B, most, spare):
    """As many requests as there may be; rows of thousands of pages in a large pool."""
    r = random.Random(B)
    x = Caches([r.randint(0, most) for _ in range(B)], 16, layers=1, Hkv=1, spare=spare, seed=B)
    ref = Forks(x.s, 16)
    for step in range(3):
        have = [len(row) * 16 for row in ref.rows]
        src = [r.choice([b, r.randrange(B)]) for b in range(B)]
        length = [r.choice([have[c], r.randint(have[c] // 2, have[c])]) for c in src]
        want = x.copy()
        copies = ref.fork(src, length)
        assert copies is not None
        for a, b, n in copies:
            for c in want:
                c[b, :, :n] = c[a, :, :n]
        x.s.dllm_serve_fork(x.layers, _i32(src), _i32(length))
        x.s.dllm_serve_check()
        x.same(want)
        ref.same(x.s)


def test_plan_keeps_shared_pages(dev):
    """After a fork: a plan that would write to a shared page, or give it back, is refused and reported, others are not;
    the last pages are written to; a fork that ends the others frees the pages for plans again."""
    from paper_2606_13740_gb300 import DllmError
    x = Caches([40, 0, 0, 20], 16, spare=12, seed=3)
    s = x.s
    s.dllm_serve_fork(x.layers, _i32([0, 0, 0]), _i32([40, 40, 33]))  # 2 pages of three, each its own last
    s.dllm_serve_check()
    rows = s.table.cpu().tolist()
    assert rows[0][:2] == rows[1][:2] == rows[2][:2] and len({r[2] for r in rows[:3]}) == 3
    s.dllm_serve_plan(_i32([40, 32, 33, 20]), _i32([3, 5, 30, 1]), 39)
    s.dllm_serve_check()
    assert s.held.cpu().tolist() == [3, 3, 4, 2]
    for length, q in ((31, 2), (16, 0), (0, 0), (5, 40)):
        s.dllm_serve_plan(_i32([43, length, 63, 21]), _i32([1, q, 1, 1]), 3 + q)
        with pytest.raises(DllmError, match="status bits 256"):
            s.dllm_serve_check()
        assert s.n_keys.cpu().tolist() == [44, 0, 64, 22] and s.held.cpu().tolist() == [3, 3, 4, 2]
        assert s.table.cpu().tolist()[1][:2] == rows[0][:2] and s.slot[1:1 + q].cpu().tolist() == [-1] * q
    s.dllm_serve_plan(_i32([44, 32, 64, 22]), _i32([0] * 4), 0)  # the last page of its own goes back
    s.dllm_serve_check()
    want = x.copy()
    for first in (0, 17, 31):  # nor does a compaction write to one
        s.dllm_serve_compact(x.layers, _i32([first]), _i32([[1, 5]]), _i32([2]))
        with pytest.raises(DllmError, match="status bits 256"):
            s.dllm_serve_check()
    x.same(want)
    s.dllm_serve_compact(x.layers, _i32([30]), _i32([[0, 1, 3, 4]]), _i32([4]))
    s.dllm_serve_check()
    free = s.ring_pos.cpu().tolist()[1]
    s.dllm_serve_fork(x.layers, _i32([0, 1, 2]), _i32([0, 32, 0]))
    assert s.ring_pos.cpu().tolist()[1] == free + 1 + 2  # (the last pages of the first and the third; two stay with the second)
    s.dllm_serve_plan(_i32([0, 0, 0, 22]), _i32([0, 0, 0, 0]), 0)
    s.dllm_serve_check()
    assert s.held.cpu().tolist() == [0, 0, 0, 2] and s.ring_pos.cpu().tolist()[1] == s.cfg.n_pages - 2
    s.dllm_serve_fork(x.layers, _i32([3, 3]), _i32([20, 20]))
    s.dllm_serve_reset()  # forgets what is shared
    s.dllm_serve_plan(_i32([3, 3, 0, 0]), _i32([4, 4, 1, 1]), 10)
    s.dllm_serve_check()


def test_fork_reports_broken_tables(dev):
    """Held counts, pages and ring places that no plan leaves: nothing is changed."""
    from paper_2606_13740_gb300 import DllmError
    for breaks in (lambda s: s.held[1].fill_(99), lambda s: s.held[2].fill_(-1), lambda s: s.table[0, 0].fill_(-5),
                   lambda s: s.table[1, 1].fill_(1 << 28), lambda s: s.ring_pos[0].fill_(-1), lambda s: s.ring_pos[1].fill_(1 << 20),
                   lambda s: s.ring[s.ring_pos[0].item()].fill_(77)):
        x = Caches([40, 20, 5], 16, seed=4)
        breaks(x.s)
        want, table, held = x.copy(), x.s.table.clone(), x.s.held.clone()
        x.s.dllm_serve_fork(x.layers, _i32([0, 0]), _i32([40, 39]))
        with pytest.raises(DllmError, match="status bits 64"):
            x.s.dllm_serve_check()
        x.same(want)
        assert torch.equal(x.s.table, table) and torch.equal(x.s.held, held)


# ------------------------------------------------------------------ log probabilities
def _logprobs(z, tokens, mask, top):
    from paper_2606_13740_gb300 import serve
    return serve.dllm_serve_logprobs(z, tokens, mask, top)


def _check_logprobs(z, tokens, mask, top):
    """Against 64 bits.  A lane adds at most `chain` terms one after another, each of an exponential a few roundings
    wide (of 8 + |z - m| at most against its reference): a sum is off by (chain + 64) half steps of 2^-24 of the sum of its terms' sizes."""
    N, V = z.shape
    lp, entropy, top_ids, top_lp, lse = _logprobs(z, tokens, mask, top)
    x = z.double().clone()
    if mask >= 0:
        x[:, mask] = -INF
    m, at = x.max(1)
    d = x - m[:, None]
    e = torch.exp(d)
    rest = e.scatter(1, at[:, None], 0.0)
    O = rest.sum(1)
    off = (V / 256 + 64) * 2.0 ** -24
    log_rest = torch.log1p(O)
    moment = torch.where(rest > 0, rest * d, 0.0).sum(1)
    tol_rest = off * torch.minimum(O, torch.ones_like(O)) + 2.0 ** -22 * log_rest
    assert bool(((lse.double() - (m + log_rest)).abs() <= tol_rest + 2.0 ** -23 * (m.abs() + log_rest)).all())
    want = log_rest - moment / (1 + O)
    size = (rest * 8).sum(1) + moment.abs()
    assert bool(((entropy.double() - want).abs() <= tol_rest + (off * size) / (1 + O) + 2.0 ** -22 * want.abs()).all())

    def close(got, ids):
        v = torch.gather(d, 1, ids)
        w = v - log_rest[:, None]
        dead = w == -INF
        assert bool((got[dead] == -INF).all())
        return bool(((got.double() - w)[~dead].abs() <= (tol_rest[:, None] + 2.0 ** -22 * (v.abs() + log_rest[:, None]))[~dead]).all())

    if tokens is not None and tokens.numel():
        assert close(lp, tokens.long())
    if top:
        order = torch.sort(x, dim=1, descending=True, stable=True)
        n = min(top, V)
        want = torch.where(order.values[:, :n] > -INF, order.indices[:, :n], -1)
        assert torch.equal(top_ids[:, :n].long(), want) and bool((top_ids[:, n:] == -1).all())
        assert bool((top_lp[top_ids < 0] == -INF).all()) and close(top_lp[:, :n], order.indices[:, :n])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,V,top,tokens,mask", [
    (1, 1, 1, 1, -1), (3, 2, 5, 2, 1), (2, 31, 32, 3, 30), (5, 511, 7, 1, -1), (4, 512, 0, 0, 0), (3, 513, 32, 9, 512),
    (1, 126464, 5, 1, 126463), (33, 5000, 20, 2, 4999), (700, 1024, 32, 1, 1023), (2, 152064, 32, 300, 152063),
    (2, 600001, 32, 1, 17), (1, 2300000, 20, 2, -1),  # groups of several steps
])
def test_logprobs_match_64_bits(dev, dtype, N, V, top, tokens, mask):
    g = torch.Generator(device="cuda").manual_seed(N + V)
    for spread in (0.0, 1.0, 5.0):
        z = (torch.randn(N, V, device="cuda", generator=g) * spread).to(DT[dtype])
        if spread == 5.0 and V > 8:
            z[torch.rand(N, V, device="cuda", generator=g) < 0.9] = -INF
            z[:, 3] = 1.0
        _check_logprobs(z, torch.randint(0, V, (N, tokens), device="cuda", generator=g, dtype=torch.int32), mask, top)


def test_logprobs_of_peaked_rows_keep_their_digits(dev):
    """One id far above the others: its log probability and the entropy are small, and right relative to themselves."""
    V = 20000
    g = torch.Generator(device="cuda").manual_seed(1)
    for where in (0, 700, V - 1):
        for height in (12.0, 25.0, 60.0, 85.0):
            z = torch.randn(2, V, device="cuda", generator=g)
            z[:, where] = height
            lp, entropy, _, _, _ = _logprobs(z, _i32([[where], [where]]), -1, 0)
            d = z.double() - height
            rest = torch.exp(d).scatter(1, _i32([[where]] * 2).long(), 0.0)
            O = rest.sum(1)
            want = torch.log1p(O) - (rest * d).sum(1) / (1 + O)
            # (V / 256 + 64) 2^-24, an argument of up to 90 rounded twice, and flushed terms below 2^-126
            tol = (V / 256 + 64 + 2 * 90) * 2.0 ** -24
            assert bool(((lp[:, 0].double() + torch.log1p(O)).abs() <= tol * O + V * 2.0 ** -126).all())
            assert bool(((entropy.double() - want).abs() <= tol * want + 90 * V * 2.0 ** -126).all())


def test_logprobs_of_extremes(dev):
    """Rows of nothing but -inf, the type's lowest value, +inf, NaN (under the mask too), ids that are none."""
    V = 3000
    z = torch.randn(9, V, device="cuda")
    z[0] = -INF
    z[1] = torch.finfo(torch.float32).min
    z[2, 5] = INF
    z[3, 5] = z[3, 9] = INF
    z[4, 7] = NAN
    z[5, V - 1] = NAN
    z[6] = -INF
    z[6, 2000] = -3.0
    z[7] = torch.finfo(torch.float32).max
    z[8, :] = NAN
    tokens = _i32([[5, 7, -1, V, V - 1, 2000]] * 9)
    lp, entropy, ids, top_lp, lse = (x.cpu().double() for x in _logprobs(z, tokens, V - 1, 3))
    assert lse[0] == -INF and entropy[0] == 0 and bool((lp[0] == -INF).all()) and ids[0].tolist() == [-1] * 3
    n = V - 1
    assert abs(entropy[1] - math.log(n)) < 1e-4 and bool(((lp[1, [0, 1, 5]] + math.log(n)).abs() < 1e-4).all())
    assert ids[1].tolist() == [0, 1, 2] and ids[7].tolist() == [0, 1, 2] and abs(entropy[7] - math.log(n)) < 1e-4
    for r in (2, 3):
        assert lse[r] == INF and math.isnan(entropy[r]) and math.isnan(lp[r, 0]) and lp[r, 1] == lp[r, 5] == -INF
    assert ids[2, 0] == 5 and ids[3, :2].tolist() == [5, 9]
    for r in (4, 8):
        assert math.isnan(lse[r]) and math.isnan(entropy[r]) and bool(lp[r, [0, 1, 5]].isnan().all())
    assert bool((ids[4] != 7).all()) and bool((ids[4] >= 0).all()) and ids[8].tolist() == [-1] * 3
    assert bool(torch.isfinite(lse[5])) and bool(torch.isfinite(entropy[5])) and lp[5, 4] == -INF
    assert bool((lp[[0, 1, 2, 3, 5, 6, 7]][:, [2, 3, 4]] == -INF).all())
    assert lse[6] == -3 and entropy[6] == 0 and lp[6, 5] == 0 and ids[6].tolist() == [2000, -1, -1] and top_lp[6, 0] == 0


def test_logprobs_of_masks_of_the_lowest_value(dev):
    """Ids that a program has set to the type's lowest value, in runs and alone, and values past 10^37."""
    g = torch.Generator(device="cuda").manual_seed(6)
    V = 20000
    for dtype in ("f32", "bf16", "f16"):
        z = torch.randn(8, V, device="cuda", generator=g).to(DT[dtype])
        low = torch.finfo(DT[dtype]).min
        z[0, :V // 2] = low
        z[1, V // 3:] = low
        z[2, torch.rand(V, device="cuda", generator=g) < 0.9] = low
        z[3] = low
        z[3, 17] = low / 2
        z[4, ::512] = -INF
        z[4, 600:7000] = -INF
        if dtype != "f16":
            z[5] = (torch.randn(V, device="cuda", generator=g) * 3e37).to(DT[dtype])
            z[6, 5000:] = -2e38
            z[6, 9000] = 3e37
            z[7] = -1e37 - 1e36 * torch.rand(V, device="cuda", generator=g).to(DT[dtype]).abs()
        best = z[:, :V - 1].argmax(1, keepdim=True).to(torch.int32)
        _check_logprobs(z, best, V - 1, 1)
        _check_logprobs(z[:3], best[:3], V - 1, 32)


def test_logprobs_ties_go_to_the_lowest_id(dev):
    """Few values over many ids, more equal ones than are ranked side by side among them."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for kinds, V in ((2, 40000), (3, 5000), (1, 9000), (300, 152064)):
        z = torch.randint(0, kinds, (7, V), device="cuda", generator=g).float()
        z[3, V // 2] = 1e4
        for dtype in ("f32", "bf16"):
            _check_logprobs(z.to(DT[dtype]), None, V // 3, 32)


def test_logprobs_strides_and_offsets(dev):
    """Rows in a wider array, at odd places, past 2^32 bytes; the buffers around the results stay."""
    wide = torch.randn(6, 5003, device="cuda")
    for a, b in ((0, 5000), (1, 4097), (3, 5003)):
        _check_logprobs(wide[:, a:b], _i32([[0, 5]] * 6), -1, 4)
    half = wide.to(torch.bfloat16)
    _check_logprobs(half[:, 1:], _i32([[0, 5]] * 6), -1, 4)
    far = torch.empty(2, 1 << 30, device="cuda")[:, :1000]
    far.copy_(torch.randn(2, 1000, device="cuda"))
    _check_logprobs(far, _i32([[0], [5]]), -1, 4)
    many = torch.randn(66000, 40, device="cuda")
    _check_logprobs(many, torch.full((66000, 1), 7, device="cuda", dtype=torch.int32), 3, 2)


# ------------------------------------------------------------------ together
def test_a_step_in_a_graph_on_another_stream(dev):
    """Plan, tree, attention, log probabilities, accept, compact and fork, captured and replayed: what they give eagerly."""
    from paper_2606_13740_gb300 import serve
    L, Q, page = [40, 7, 0, 90], [26, 1, 9, 33], 16

    def setup():
        r = random.Random(5)
        s = _serve(max_batch=4, max_rows=80, page=page, n_pages=60, max_pages=12, n_heads=4, n_kv_heads=2, head_dim=64)
        g = torch.Generator(device="cuda").manual_seed(7)
        trees = [_tree_of(r, n) for n in Q]
        N = sum(Q)
        k, v = (torch.randn(2, 60, 2, page, 64, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
        d = dict(s=s, parent=_i32([p for t in trees for p in t]), q=torch.randn(N, 4, 64, device="cuda", generator=g).to(torch.bfloat16),
                 k=k, v=v, layers=s.layers(k, v), z=torch.randn(N, 900, device="cuda", generator=g), L=_i32(L), Q=_i32(Q), src=_i32([0, 0, 3, 3]))
        d["ids"] = torch.randint(0, 3, (N,), device="cuda", generator=g, dtype=torch.int32)
        d["x0"] = torch.randint(0, 3, (N,), device="cuda", generator=g, dtype=torch.int32)
        return d

    def step(d):
        s = d["s"]
        s.dllm_serve_plan(d["L"], d["Q"], sum(Q))
        mask = s.dllm_serve_tree(d["parent"], 64)
        out, lse = s.dllm_serve_tree_attention(d["q"], d["k"][0], d["v"][0], mask, lse=True)
        lp = serve.dllm_serve_logprobs(d["z"], d["ids"][:, None], 899, top=5)
        keep, n, nxt = s.dllm_serve_accept(d["parent"], d["ids"], d["x0"], 4, 10)
        s.dllm_serve_compact(d["layers"], d["L"], keep, n)
        s.dllm_serve_fork(d["layers"], d["src"], (d["L"] + n)[d["src"].long()])
        return [mask, out, lse, *lp, keep, n, nxt, s.pos, s.table, s.held, s.ring_pos, s.n_keys, d["k"], d["v"]]

    a, b = setup(), setup()
    want = [x.clone() for x in step(a)]
    a["s"].dllm_serve_check()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        k0, v0 = b["k"].clone(), b["v"].clone()
        with torch.cuda.graph(graph, stream=side):
            b["s"].dllm_serve_reset()
            got = step(b)
        for _ in range(3):
            b["k"].copy_(k0), b["v"].copy_(v0)
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    with torch.cuda.stream(side):
        b["s"].dllm_serve_check()


def test_host_threads_on_streams_of_their_own(dev):
    """Four threads, each with a handle, caches and logits of its own on a stream of its own: what one alone gives."""
    import threading

    def work(seed, out):
        r = random.Random(seed)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            x = Caches([r.randint(20, 200) for _ in range(6)], 16, hd=128 if seed % 2 else 64, spare=40, seed=seed)
            z = torch.randn(30 + 400 * (seed % 2), 9000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
            for step in range(15):
                keep = [sorted(r.sample(range(n), n * 2 // 3)) for n in x.L]
                most = max(map(len, keep))
                x.s.dllm_serve_compact(x.layers, _i32([0] * 6), _i32([k + [0] * (most - len(k)) for k in keep]), _i32([len(k) for k in keep]))
                have = [n // 2 + 1 for n in x.L]
                x.s.dllm_serve_fork(x.layers, _i32([b // 2 for b in range(6)]), _i32([have[b // 2] for b in range(6)]))
                x.L = [have[b // 2] for b in range(6)]
                lp = _logprobs(z, None, step, 1 + step)
            out.append([c.cpu() for c in x.k + x.v] + [x.s.table.cpu(), x.s.ring_pos.cpu()] + [v.cpu() for v in lp if v is not None])

    alone, together = [[] for _ in range(4)], [[] for _ in range(4)]
    for seed in range(4):
        work(seed, alone[seed])
    threads = [threading.Thread(target=work, args=(seed, together[seed])) for seed in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for a, b in zip(alone, together):
        assert len(a) == len(b) == 1 and all(torch.equal(p, q) for p, q in zip(a[0], b[0]))


def test_results_repeat(dev):
    x = Tree([500, 0, 77], [1, 64, 32], 3000 + 8, 64, 32, 32, 128, seed=14)
    first = x.call()
    assert all(torch.equal(first, x.call()) for _ in range(3))
    z = torch.randn(37, 126464, device="cuda")
    a = _logprobs(z, _i32([[5]] * 37), -1, 32)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(a, _logprobs(z, _i32([[5]] * 37), -1, 32)))
