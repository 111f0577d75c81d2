"""Requests that share pages after a fork, on the GPU: plans and attention over keys that are more, all requests together,
than the pool has places."""
import random

import pytest

torch = pytest.importorskip("torch")
from test_gpu_serve import DT, Paged, _i32, _serve, dev  # noqa: E402,F401
from test_gpu_serve_drafts import Caches, Forks, Tree, _compacted, _path, _seen, _tree_of, _words  # noqa: E402
from test_gpu_serve_drafts_example import _alone, ex  # noqa: E402,F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ plans after a fork
class Forked(Tree):
    """Requests that continue the first one's own positions, each up to a place of its own, with new tokens behind."""

    def __init__(self, base, cuts, Q, P, page, H, Hkv, hd, causal=False, dtype="bf16", seed=0):
        self.L, self.Q, self.P, self.page, self.H, self.Hkv, self.hd, self.causal = cuts, Q, P, page, H, Hkv, hd, causal
        self.dtype = DT[dtype]
        B, N, r = len(cuts), sum(Q), random.Random(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        held, npre = -(-base // page), -(-P // page)
        n_pages = npre + held + sum(1 + -(-q // page) for q in Q)
        self.s = s = _serve(max_batch=B, max_rows=N, page=page, n_pages=n_pages, max_pages=held + 1 + -(-max(Q) // page), n_heads=H,
                            n_kv_heads=Hkv, head_dim=hd, dtype=dtype)
        order = torch.randperm(n_pages, device="cuda", generator=g, dtype=torch.int32)
        s.ring.copy_(order)
        self.prefix = order[:npre].clone()
        s.ring_pos.copy_(_i32([npre, n_pages - npre]))
        self.kc, self.vc = (torch.full((n_pages, Hkv, page, hd), float("nan"), device="cuda", dtype=self.dtype) for _ in range(2))

        def fresh(n):
            return [torch.randn(n, Hkv, hd, device="cuda", generator=g).to(self.dtype) for _ in range(2)]

        def put(pages, first, kv):
            at = torch.arange(first, first + len(kv[0]), device="cuda")
            for c, x in zip((self.kc, self.vc), kv):
                c[pages[at // page].long(), :, at % page] = x

        shared, prefix = fresh(base), fresh(P)
        s.dllm_serve_plan(_i32([base] + [0] * (B - 1)), _i32([0] * B), 0)
        put(s.table[0], 0, shared), put(self.prefix, 0, prefix)
        s.dllm_serve_fork(s.layers([self.kc], [self.vc]), _i32([0] * B), _i32(cuts))
        s.dllm_serve_check()
        s.dllm_serve_plan(_i32(cuts), _i32(Q), N, prefix_len=P, causal=causal)
        self.k, self.v = [prefix[0]], [prefix[1]]
        for b, (cut, q) in enumerate(zip(cuts, Q)):
            new = fresh(q)
            put(s.table[b], cut, new)
            self.k.append(torch.cat([shared[0][:cut], new[0]])), self.v.append(torch.cat([shared[1][:cut], new[1]]))
        self.q = torch.randn(N, H, hd, device="cuda", generator=g).to(self.dtype)
        self.words = -(-max(Q) // 32)
        self.bits = [b for q in Q for b in _seen(_tree_of(r, q))]
        self.mask = _i32([_words(b, self.words) for b in self.bits])

    def check_plain(self):
        """dllm_serve_attention, whose rows see all new tokens (causal: those up to themselves)."""
        out, lse = self.s.dllm_serve_attention(self.q, self.kc, self.vc, self.prefix, lse=True)
        self.s.dllm_serve_check()
        want, size, wlse = Paged.want(self)
        u = 2.0 ** -8 if self.dtype == torch.bfloat16 else 2.0 ** -11
        # a rounding of the output, one of each probability (which in f16 lose what is below 2^-25 too), fp32 sums
        tol = u * want.abs() + (u + 2e-5) * size + ((self.P + max(map(len, self.k))) * 2.0 ** -25 if u < 2.0 ** -10 else 0.0)
        assert bool(((out.double() - want).abs() <= tol).all())
        assert bool(((lse.double() - wlse).abs() <= 1e-5 * (1 + wlse.abs())).all())


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("base,n,q,P,page,H,Hkv,hd,dtype", [
    (1900, 12, 1, 0, 64, 8, 8, 64, "bf16"), (1920, 8, 5, 100, 64, 28, 4, 128, "f16"), (500, 40, 3, 0, 16, 16, 4, 64, "bf16"),
    (3000, 9, 70, 300, 256, 4, 2, 128, "bf16"),
])
def test_requests_that_share_more_keys_than_the_pool_has_places(dev, base, n, q, P, page, H, Hkv, hd, dtype, causal):
    """Beams of a long prompt: by bits and without, against 64 bits; nothing is refused or reported."""
    r = random.Random(base)
    cuts = [base - r.choice([0, 0, r.randint(0, 40)]) for _ in range(n)]
    x = Forked(base, cuts, [q] * n, P, page, H, Hkv, hd, causal=causal, dtype=dtype, seed=n)
    assert x.s.status.cpu().tolist()[:2] == [0, 0]
    assert sum(-(-(c + q) // 64) for c in cuts) > x.s.cfg.n_pages * page // 64 + n
    x.check()
    x.check_plain()


def test_as_many_shared_keys_as_a_plan_takes(dev):
    """4000 requests that share 65600 keys are attended to; with 4090 of them there are more than 2^22 blocks of 64 keys:
    the plan refuses all, takes no page, and a plan of fewer goes on."""
    from paper_2606_13740_gb300 import DllmError
    base, most, hd = 65600, 4090, 64
    held = base // 16
    s = _serve(max_batch=most, max_rows=most, page=16, n_pages=held + most, max_pages=held + 1, n_heads=1, n_kv_heads=1, head_dim=hd)
    kc, vc = (torch.randn(held + most, 1, 16, hd, device="cuda").to(torch.bfloat16) for _ in range(2))
    s.dllm_serve_plan(_i32([base]), _i32([0]), 0)
    s.dllm_serve_fork(s.layers([kc], [vc]), _i32([0] * most), _i32([base] * most))
    s.dllm_serve_check()
    table, ring = s.table.clone(), s.ring_pos.clone()
    q = torch.randn(most, 1, hd, device="cuda").to(torch.bfloat16)
    s.dllm_serve_plan(_i32([base] * most), _i32([1] * most), most)
    out = s.dllm_serve_attention(q, kc, vc)
    assert s.status.cpu().tolist()[1:] == [most, 0, 0]
    with pytest.raises(DllmError, match="status bits 64"):
        s.dllm_serve_check()
    assert bool((out == 0).all()) and bool((s.slot == -1).all()) and bool((s.n_keys == 0).all())
    assert torch.equal(s.table, table) and torch.equal(s.ring_pos, ring) and bool((s.held == held).all())
    n = 4000
    s.dllm_serve_plan(_i32([base] * n), _i32([1] * n), n)
    out = s.dllm_serve_attention(q[:n], kc, vc)
    s.dllm_serve_check()
    assert s.status.cpu().tolist()[1:] == [0, n, 0]
    k, v = (c[table[0, :held].long()].reshape(base, hd).double() for c in (kc, vc))
    last = s.table[:n, held].long()
    for i in range(0, n, 500):
        z = torch.cat([q[i:i + 500, 0].double() @ k.T, (q[i:i + 500, 0].double() * kc[last[i:i + 500], 0, 0].double()).sum(1, True)], 1)
        p = torch.softmax(z * hd ** -0.5, 1)
        own = vc[last[i:i + 500], 0, 0].double()
        want, size = p[:, :-1] @ v + p[:, -1:] * own, p[:, :-1] @ v.abs() + p[:, -1:] * own.abs()
        # as of the attention elsewhere: the output's rounding, the probabilities', and sums of 65601 terms in 32 bits
        assert bool(((out[i:i + 500].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2e-5) * size).all())


# ------------------------------------------------------------------ paths of requests that were left out
def test_accept_gives_no_path_to_requests_that_are_left_out(dev):
    """Refused by the plan (pages, lengths), or with a wrong tree: no path, no next token, nothing moved; the others as
    without them.  A right tree after a wrong one, and the next plan, are judged for themselves."""
    from paper_2606_13740_gb300 import DllmError
    q = [5, 40, 6, 3, 4]
    s = _serve(max_batch=5, max_rows=60, page=16, n_pages=5, max_pages=4, n_heads=2, n_kv_heads=2, head_dim=64)
    kc, vc = (torch.randn(5, 2, 16, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    layers, x0 = s.layers([kc], [vc]), _i32([1] * 58)

    def flat(trees):
        return _i32([p for t in trees for p in t])

    def chain(n):
        return list(range(-1, n - 1))

    def paths(trees):
        keep, n, nxt = s.dllm_serve_accept(flat(trees), x0, x0, 5, 8)
        at = [c.clone() for c in (kc, vc)]
        s.dllm_serve_compact(layers, _i32(first), keep, n)
        assert torch.equal(at[0], kc) and torch.equal(at[1], vc)  # (paths from token 0 on stay where they are)
        for row, k in zip(keep.cpu().tolist(), n.cpu().tolist()):
            assert row == list(range(k)) + [-1] * (8 - k)
        return n.cpu().tolist(), nxt.cpu().tolist()

    right = [chain(n) for n in q]
    first = [0, 0, 4, 0, 3]
    s.dllm_serve_plan(_i32(first), _i32([0] * 5), 0)
    s.dllm_serve_plan(_i32([0, 0, 4, -1, 3]), _i32(q), 58)  # three pages for the second when two are left; a length of -1
    with pytest.raises(DllmError, match="status bits 6"):
        s.dllm_serve_check()
    refused = [i for i, b in enumerate((0, 5, 45, 51, 54)) if int(s.slot[b]) < 0]
    assert refused == [1, 3]
    want = [0 if b in refused else min(n, 8) for b, n in enumerate(q)]
    assert paths(right) == (want, [1 if n else -1 for n in want])
    for wrong in (0, 5, -2, 1 << 30):  # of the first request, whose tree is otherwise a chain
        trees = [[-1, 0, 1, wrong if wrong else 3, 3]] + right[1:]
        s.dllm_serve_tree(flat(trees), 64)
        with pytest.raises(DllmError, match="status bits 128"):
            s.dllm_serve_check()
        less = [0] + want[1:]
        assert paths(trees) == (less, [1 if n else -1 for n in less])
    s.dllm_serve_tree(flat(right), 64)
    assert paths(right) == (want, [1 if n else -1 for n in want])
    s.dllm_serve_tree(flat(right), 32)  # the second has more tokens than bits (it is refused all the same)
    with pytest.raises(DllmError, match="status bits 128"):
        s.dllm_serve_check()
    assert paths(right)[0] == want

    s.dllm_serve_reset()
    first = [0] * 5
    q = [33, 2, 1, 1, 1]
    right = [chain(n) for n in q]
    for wide, n in ((32, [0, 2, 1, 0, 0]), (64, [8, 2, 1, 0, 0])):
        s.dllm_serve_plan(_i32([0] * 5), _i32(q), 38)
        x0 = _i32([1] * 38)
        if wide == 32:  # without a tree, a path is judged by the plan alone
            assert paths(right)[0] == [8, 2, 1, 0, 0]
        with pytest.raises(DllmError, match="status bits 4"):
            s.dllm_serve_check()
        s.dllm_serve_tree(flat(right), wide)
        if wide == 32:
            with pytest.raises(DllmError, match="status bits 128"):
                s.dllm_serve_check()
        assert paths(right)[0] == n
    s.dllm_serve_check()
    s.dllm_serve_tree(flat(right), 32)
    s.dllm_serve_plan(_i32([0] * 5), _i32(q), 38)
    assert paths(right)[0] == [8, 2, 1, 0, 0]


# ------------------------------------------------------------------ the pool's state, written by the program
STATE = ("table", "held", "ring", "ring_pos", "shared")


def _beams(**kw):
    """Three requests that continue the first one's 40 positions, in pages of 16, and a fourth of 20."""
    x = Caches([40, 0, 0, 20], 16, spare=12, **kw)
    before = {n: getattr(x.s, n).clone() for n in STATE}
    x.s.dllm_serve_fork(x.layers, _i32([0, 0, 0]), _i32([40, 40, 33]))
    x.s.dllm_serve_check()
    assert x.s.shared.cpu().tolist() == [2, 2, 2, 0] and not bool(before["shared"].any())
    return x, before


def test_a_state_from_before_a_fork_is_written_back(dev):
    """Nothing is shared then: plans give pages back and write to them, and compactions move."""
    x, before = _beams(seed=3)
    s = x.s
    for n, v in before.items():
        getattr(s, n).copy_(v)
    want = _compacted(x, x.copy(), s.table.cpu().tolist(), [1], [[2, 30]])
    s.dllm_serve_compact(x.layers, _i32([1]), _i32([[2, 30]]), _i32([2]))
    x.same(want)
    s.dllm_serve_plan(_i32([3, 0, 0, 0]), _i32([2, 1, 0, 0]), 3)
    s.dllm_serve_check()
    assert s.status.cpu().tolist()[1:] == [0, 1, 4] and s.held.cpu().tolist() == [1, 1, 0, 0]


def test_a_forked_state_moves_to_a_larger_handle(dev):
    """With what is shared: a plan there that would give back or write to a shared page is refused, others are not, and a
    fork there ends the sharing.  A fork of requests onto themselves finds it where a program does not know it."""
    from paper_2606_13740_gb300 import DllmError
    x, _ = _beams(seed=5)
    a, n = x.s, x.s.cfg.n_pages
    b = _serve(max_batch=9, max_rows=50, page=16, n_pages=n + 7, max_pages=20, n_heads=3, n_kv_heads=3, head_dim=64)
    kc, vc = ([torch.cat([c, torch.zeros_like(c[:7])]) for c in cs] for cs in (x.k, x.v))
    layers = b.layers(kc, vc)
    wide = a.cfg.max_pages
    b.table[:4, :wide].copy_(a.table), b.held[:4].copy_(a.held), b.shared[:4].copy_(a.shared)
    head, free = a.ring_pos.cpu().tolist()
    ring = a.ring.cpu().tolist()
    left = [ring[(head + i) % n] for i in range(free)] + list(range(n, n + 7))
    b.ring[:len(left)].copy_(_i32(left)), b.ring_pos.copy_(_i32([0, len(left)]))

    def refused():
        for length, q in ((0, 0), (16, 0), (31, 2)):
            b.dllm_serve_plan(_i32([40, length, 33, 20]), _i32([1, q, 1, 1]), 3 + q)
            with pytest.raises(DllmError, match="status bits 256"):
                b.dllm_serve_check()
            assert b.n_keys.cpu().tolist()[:4] == [41, 0, 34, 21] and b.held.cpu().tolist()[:4] == [3, 3, 3, 2]

    refused()
    b.shared.zero_()  # as by a program that does not know
    for src in ([0, 1, 2, 3], [0, 1]):  # (all of them, or some: the rows of the others count too)
        b.dllm_serve_fork(layers, _i32(src), _i32([40, 40, 33, 20][:len(src)]))
        b.dllm_serve_check()
        assert b.shared.cpu().tolist() == [2, 2, 2] + [0] * 6 and b.status.cpu().tolist()[1:] == [0, 0, 0]
        refused()
        b.shared.zero_()
    b.dllm_serve_fork(layers, _i32([0, 1, 2]), _i32([40, 0, 0]))
    b.dllm_serve_plan(_i32([5, 0, 0, 20]), _i32([1, 0, 0, 1]), 2)
    b.dllm_serve_check()
    assert b.shared.cpu().tolist() == [0] * 9 and b.held.cpu().tolist() == [1, 0, 0, 2] + [0] * 5
    assert b.ring_pos.cpu().tolist()[1] == n + 7 - 3


def test_reset_forgets_what_is_shared(dev):
    x, _ = _beams(seed=6)
    x.s.dllm_serve_reset()
    assert not bool(x.s.shared.any())
    x.s.dllm_serve_plan(_i32([3, 3, 0, 0]), _i32([4, 4, 1, 1]), 10)
    x.s.dllm_serve_check()


# ------------------------------------------------------------------ plans and forks in turn
class Pages(Forks):
    """Forks with the plan's definition beside the fork's."""

    def __init__(self, s, page):
        super().__init__(s, page)
        self.most, self.shared = s.cfg.max_pages, [0] * len(self.rows)

    def fork(self, src, length):
        copies = super().fork(src, length)
        if copies is not None:
            count = {}
            for p in (p for row in self.rows for p in row):
                count[p] = count.get(p, 0) + 1
            self.shared = [max([i + 1 for i, p in enumerate(row) if count[p] > 1] + [0]) for row in self.rows]
        return copies

    def plan(self, L, Q):
        """(n_keys, bits, pages taken, pages given back)."""
        budget, asked, bits, taken, back, keys = len(self.free), 0, 0, 0, [], []
        for b, (l, q) in enumerate(zip(L, Q)):
            row, need = self.rows[b], -(-(l + q) // self.page)
            others = need < self.shared[b] or (q > 0 and l // self.page < self.shared[b])
            bad = l < 0 or q < 0 or need > self.most
            grow = 0 if bad or others else max(0, need - len(row))
            asked += grow
            no = 2 if bad else 256 if others else 4 if grow and asked > budget else 0
            bits |= no
            keys.append(0 if no else l + q)
            if no:
                continue
            for _ in range(grow):
                row.append(self.free.pop(0))
            taken += grow
            back += row[need:]
            del row[need:]
        self.free += back
        return keys, bits, taken, len(back)


@pytest.mark.parametrize("B,page,base,spare,steps", [(2, 16, 50, 6, 25), (7, 64, 300, 14, 25), (40, 16, 90, 100, 12),
                                                      (1100, 16, 40, 3000, 6)])
def test_plans_and_forks_in_turn(dev, B, page, base, spare, steps):
    """Requests grow by plans, shrink, end, and continue one another by forks, step after step; some plans and forks cannot be
    carried out.  Tables, ring, key counts, what is shared, and the caches."""
    r = random.Random(B)
    x = Caches([r.randint(0, base) for _ in range(B)], page, layers=1, Hkv=1, spare=spare, seed=B)
    s, ref = x.s, Pages(x.s, page)
    own = list(x.L)
    seen = 0
    for step in range(steps):
        L, Q = [], []
        for b in range(B):
            low = ref.shared[b] * page
            kind = r.random()
            L.append(own[b] if kind < 0.7 else r.randint(min(low, own[b]), own[b]) if kind < 0.9 else r.randint(0, own[b]))
            Q.append(0 if r.random() < 0.2 else r.randint(1, 20))
        rows = min(sum(Q), s.cfg.max_rows)
        keys, bits, taken, given = ref.plan(L, Q)
        s.dllm_serve_plan(_i32(L), _i32(Q), rows)
        assert s.status.cpu().tolist() == [bits | (8 if sum(Q) > rows else 0), keys.count(0) - sum(l + q == 0 for l, q in zip(L, Q)),
                                           taken, given]
        s.status.zero_()
        seen |= bits
        assert s.n_keys.cpu().tolist() == keys
        ref.same(s)
        own = [k or min(o, len(row) * page) for k, o, row in zip(keys, own, ref.rows)]
        own = [0 if l + q == 0 else o for l, q, o in zip(L, Q, own)]
        src = [r.choice([b, b, r.randrange(B)]) for b in range(B)]
        length = [r.choice([own[c], own[c], r.randint(0, own[c]), 0]) for c in src]
        if step % 5 == 4:
            length[r.randrange(B)] = -1
        want, copies = x.copy(), ref.fork(src, length)
        s.dllm_serve_fork(x.layers, _i32(src), _i32(length))
        status = s.status.cpu().tolist()
        s.status.zero_()
        if copies is None:
            assert status[0] in (2, 4) and status[1:] == [B, 0, 0]
        else:
            assert status[:3] == [0, 0, len(copies)]
            own = length
            for a, b, n in copies:
                for c in want:
                    c[b, :, :n] = c[a, :, :n]
        x.same(want)
        ref.same(s)
        assert s.shared.cpu().tolist() == ref.shared
    assert B == 2 or seen & 256  # (two requests happen not to run into it)


def test_forks_of_many_requests_that_cannot_be_carried_out(dev):
    """Past the one-CTA form: a wrong request, a broken row or place of the ring, wherever it lies, or too few pages: all CTAs
    leave everything as it was, and the next fork goes on."""
    B = 1500
    r = random.Random(8)
    x = Caches([r.randint(17, 60) for _ in range(B)], 16, layers=1, Hkv=1, spare=900, seed=8)
    s, names = x.s, STATE + ("n_keys",)
    want, state = x.copy(), {n: getattr(x.s, n).clone() for n in names}
    same, half = list(range(B)), [n // 2 for n in x.L]

    def fork(src, length, bits):
        s.dllm_serve_fork(x.layers, _i32(src), _i32(length))
        assert s.status.cpu().tolist() == [bits, B, 0, 0]
        s.status.zero_()
        x.same(want)

    for b in (0, 255, 256, 511, 700, 1023, 1024, B - 1):
        for src, n in ((-1, 5), (B, 5), (1 << 30, 0), (b, -1), (b, len(x.L) * 16), (b, (1 << 31) - 1), (b, -(1 << 31))):
            fork(same[:b] + [src] + same[b + 1:], half[:b] + [n] + half[b + 1:], 2)
        for break_it in (lambda: s.held[b].fill_(99), lambda: s.held[b].fill_(-1), lambda: s.table[b, 0].fill_(-5),
                         lambda: s.table[b, 1].fill_(1 << 28)):
            break_it()
            now = {n: getattr(s, n).clone() for n in names}
            s.dllm_serve_fork(x.layers, _i32(same), _i32(half))
            assert s.status.cpu().tolist()[0] & 64 and s.status.cpu().tolist()[1:] == [B, 0, 0]
            s.status.zero_()
            x.same(want)
            assert all(torch.equal(getattr(s, n), v) for n, v in now.items())
            for n, v in state.items():
                getattr(s, n).copy_(v)
    head = s.ring_pos.cpu().tolist()[0]
    for k in (0, 5, 899):
        kept = s.ring[(head + k) % s.cfg.n_pages].clone()
        s.ring[(head + k) % s.cfg.n_pages] = -3
        fork(same, half, 64)
        s.ring[(head + k) % s.cfg.n_pages] = kept
    few = [n - n % 16 + 1 if n % 16 != 1 else n - 1 for n in x.L]
    fork([0] * B, [min(few[0], 17)] * B, 4)  # 1499 copies, 900 pages
    assert all(torch.equal(getattr(s, n), v) for n, v in state.items())
    ref = Pages(s, 16)
    assert ref.fork(same, half) == []
    s.dllm_serve_fork(x.layers, _i32(same), _i32(half))
    s.dllm_serve_check()
    x.same(want)
    ref.same(s)


# ------------------------------------------------------------------ together
def test_tree_attention_of_pages_far_apart(dev):
    """Pages farther apart than dense, and 2^28 elements apart: 5 GB from the first."""
    for hd, stride in ((64, 2 * 32 * 64 * 4), (128, 4 * 32 * 128 + 8), (128, 1 << 28)):
        for form in ("tree", "any"):
            Tree([50, 100], [30, 65], 64, 32, 28, 4, hd, form=form, seed=13, stride=stride).check()


def test_beams_of_a_long_prompt(ex):
    """Beams whose prompt is longer, all beams together, than the pool: scores are those of their sequences."""
    rng = random.Random(6)
    prompt = [rng.randrange(ex.VOCAB) for _ in range(700)]
    b = ex.Beams(prompt, 4, 8, seed=5)
    assert 4 * 700 > b.serve.cfg.n_pages * 16
    for _ in range(7):
        b.step()
    for score, t in zip(b.score.tolist(), b.tokens.tolist()):
        z = torch.log_softmax(_alone(ex, prompt + t, seed=5).double(), 1)
        want = sum(float(z[699 + i, v]) for i, v in enumerate(t))
        # logits 1e-2 off relative to their size (about 1.5 rms): 0.015 a log probability, rms, 8 of them
        assert abs(score - want) <= 8 * 0.03


@pytest.mark.parametrize("hd", [64, 128])
def test_compact_where_one_form_gives_way_to_the_other(dev, hd):
    """Rows of 127 to 130 places, full, short and in between."""
    r = random.Random(hd)
    L = [r.randint(100, 300) for _ in range(9)] + [130, 128]
    x = Caches(L, 16, hd=hd, layers=2, Hkv=2, seed=4)
    table = x.s.table.cpu().tolist()
    for most in (65, 127, 128, 129, 130):
        keep = [sorted(r.sample(range(n), min(n, r.choice([most, most, 3, r.randint(0, most)])))) for n in L]
        want = _compacted(x, x.copy(), table, [0] * 11, keep)
        x.s.dllm_serve_compact(x.layers, _i32([0] * 11), _i32([k + [-1] * (most - len(k)) for k in keep]), _i32([len(k) for k in keep]))
        x.s.dllm_serve_check()
        x.same(want)


def test_a_wrong_tree_after_a_right_one_has_the_plan_s_positions(dev):
    from paper_2606_13740_gb300 import DllmError
    q = [4, 300, 3]
    s = _serve(max_batch=3, max_rows=310, page=16, n_pages=24, max_pages=20, n_heads=2, n_kv_heads=2, head_dim=64)
    s.dllm_serve_plan(_i32([7, 2, -1]), _i32(q), 307, prefix_len=5)
    plain = s.pos.cpu().tolist()
    assert plain[:6] == [12, 13, 14, 15, 7, 8] and plain[304:307] == [0, 0, 0]
    with pytest.raises(DllmError, match="status bits 2"):
        s.dllm_serve_check()
    right = [-1, 0, 0, 0] + [-1] + [0] * 299 + [-1, 0, 0]
    s.dllm_serve_tree(_i32(right), 320)
    assert s.pos.cpu().tolist()[:304] == [12] + [13] * 3 + [7] + [8] * 299
    s.dllm_serve_check()
    for wrong in ([-1, 0, 2, 0] + [-1] + [0] * 298 + [300] + [-1, 0, 3], right):
        s.dllm_serve_tree(_i32(wrong), 320 if wrong is not right else 32)
        with pytest.raises(DllmError, match="status bits 128"):
            s.dllm_serve_check()
        want = plain if wrong is not right else [12, 13, 13, 13] + plain[4:]
        assert s.pos.cpu().tolist() == want


@pytest.mark.parametrize("B,page,H,Hkv,hd,most,spare,steps,cuts", [
    (3, 16, 4, 2, 64, 6, 4, 12, 4), (7, 32, 28, 4, 128, 40, 9, 8, 4), (12, 64, 4, 4, 64, 9, 14, 10, 4), (5, 16, 4, 2, 64, 12, 6, 40, 60),
    (9, 16, 28, 4, 128, 20, 1, 30, 80),
])
def test_drafting_beams_step_after_step(dev, B, page, H, Hkv, hd, most, spare, steps, cuts):
    """Plan, keys stored at their slots, tree, attention, accepted path, compaction and fork, over and over, some requests refused
    for lack of pages: the attention of every row against 64 bits, and every key and value that a request holds, where it should be."""
    r = random.Random(B * hd)
    g = torch.Generator(device="cuda").manual_seed(B)
    n_pages = B * 2 + spare
    s = _serve(max_batch=B, max_rows=B * most, page=page, n_pages=n_pages, max_pages=n_pages, n_heads=H, n_kv_heads=Hkv, head_dim=hd)
    cache = torch.full((2, n_pages, Hkv, page, hd), float("nan"), device="cuda", dtype=torch.bfloat16)
    layers = s.layers([cache[0]], [cache[1]])
    own = [torch.zeros(2, 0, Hkv, hd, device="cuda", dtype=torch.bfloat16) for _ in range(B)]
    refusals = shared = 0
    for step in range(steps):
        L, Q = [x.shape[1] for x in own], [r.choice([0, 1, r.randint(1, most), most]) for _ in range(B)]
        N = max(1, sum(Q))
        s.dllm_serve_plan(_i32(L), _i32(Q), N)
        status = s.status.cpu().tolist()[0]
        s.status.zero_()
        assert status in (0, 4)
        refused = [L[b] + Q[b] > 0 and k == 0 for b, k in enumerate(s.n_keys.cpu().tolist())]
        refusals += sum(refused)
        trees = [_tree_of(r, n) for n in Q]
        parent = _i32(([p for t in trees for p in t] + [-1])[:N])
        mask = s.dllm_serve_tree(parent, max(Q + [1]))
        new = torch.randn(2, N, Hkv, hd, device="cuda", generator=g).to(torch.bfloat16)
        slot = s.slot[:N].long()
        there = (slot >= 0).nonzero()[:, 0]
        cache[:, slot[there] // page, :, slot[there] % page] = new[:, there].transpose(0, 1)
        q = torch.randn(N, H, hd, device="cuda", generator=g).to(torch.bfloat16)
        out = s.dllm_serve_tree_attention(q, cache[0], cache[1], mask).view(N, H, hd)
        ids = [[r.randrange(3) for _ in t] for t in trees]
        x0 = [[r.randrange(3) for _ in t] for t in trees]
        flat = [_i32(([x for t in v for x in t] + [0])[:N]) for v in (ids, x0)]
        keep, n, nxt = s.dllm_serve_accept(parent, *flat, B, most)
        s.dllm_serve_compact(layers, _i32(L), keep, n)
        s.dllm_serve_check()
        at = 0
        for b in range(B):
            bits = _seen(trees[b])
            for t in range(Q[b]):
                if refused[b]:
                    assert bool((out[at + t] == 0).all())
                    continue
                sees = [j for j in range(Q[b]) if bits[t] >> j & 1]
                k, v = (torch.cat([own[b][c], new[c, [at + j for j in sees]]]).double().repeat_interleave(H // Hkv, 1) for c in (0, 1))
                p = torch.softmax(torch.einsum("hd,khd->hk", q[at + t].double(), k) * hd ** -0.5, 1)
                want, size = torch.einsum("hk,khd->hd", p, v), torch.einsum("hk,khd->hd", p, v.abs())
                # as of the attention elsewhere: the output's rounding and the probabilities'
                assert bool(((out[at + t].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2e-5) * size).all())
            path, last = _path(trees[b], ids[b], x0[b], most) if Q[b] and not refused[b] else ([], -1)
            assert keep[b].cpu().tolist() == path + [-1] * (most - len(path)) and int(n[b]) == len(path) and int(nxt[b]) == last
            own[b] = torch.cat([own[b], new[:, [at + j for j in path]]], 1)
            at += Q[b]

        def same():
            table = s.table.cpu().tolist()
            for b, x in enumerate(own):
                if x.shape[1]:
                    i = torch.arange(x.shape[1], device="cuda")
                    pages = torch.tensor(table[b], device="cuda")[i // page]
                    assert bool((pages >= 0).all()) and torch.equal(cache[:, pages, :, i % page].transpose(0, 1), x), (step, b)

        same()
        src = [r.choice([b, b, r.randrange(B)]) for b in range(B)]
        length = [r.choice([own[c].shape[1]] * (cuts - 1) + [r.randint(0, own[c].shape[1])]) for c in src]
        s.dllm_serve_fork(layers, _i32(src), _i32(length))
        status = s.status.cpu().tolist()
        s.status.zero_()
        assert status[0] in (0, 4) and status[1] == (B if status[0] else 0)
        if status[0] == 0:
            own = [own[c][:, :m] for c, m in zip(src, length)]
        same()
        shared += int((s.shared > 0).sum())
    assert cuts == 4 or shared > 0  # (where a request is cut at every fourth fork, hardly one fills a page)
    assert cuts < 80 or refusals > 0
