"""Edges of the serving operators: sizes, lengths, page numbers and values at the ends of what the calls take, beside
the ordinary ones of test_gpu_serve.py."""
import os
import subprocess
import sys
import threading

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_serve import U, Paged, Pool, _i32, _logits_case, _logits_run, _same_plan, _serve, dev  # noqa: E402,F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H,Hkv,hd", [(28, 4, 128), (4, 4, 64)])
def test_attention_first_blocks_far_from_zero(dev, H, Hkv, hd, dtype):
    """The first block of a run's every unit makes its probabilities twice, with no reference and with the block's
    maximum: with scores beyond 100 the first ones are infinities and zeros, and must not be what is used."""
    x = Paged([900, 3, 0, 64, 130] * 4, [1, 32, 100, 7, 2] * 4, 700, 32, H, Hkv, hd, dtype=dtype, seed=21, spread=30.0)
    first = x.check()
    for _ in range(20):
        assert torch.equal(x.call(), first)


# ------------------------------------------------------------------ shared memory that has to be asked for
def _fresh(code):
    """In a process of its own, whose kernels have no larger limit from an earlier call."""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]


def test_plan_batches_around_the_limit_of_shared_memory(dev):
    """In ascending order, so that no larger batch has raised the limit before."""
    _fresh("""
import torch
from paper_2606_13740_gb300 import serve
for B in (1274, 1275, 1400, 1477, 1478, 4096):
    s = serve.Serve(serve.ServeConfig(max_batch=B, max_rows=B, page=16, n_pages=B + 1, max_pages=2, n_heads=4, n_kv_heads=2,
                                      head_dim=64))
    L = torch.zeros(B, dtype=torch.int32, device="cuda")
    s.dllm_serve_plan(L, L + 1, B)
    s.dllm_serve_check()
    assert torch.equal(s.slot.long(), torch.arange(B, device="cuda") * 16), B
""")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_lists_around_the_limit_of_shared_memory(dev, dtype):
    """Histories (and biases) in ascending order, at a size that is cut into the longest stretches (64 x 11 of 8192)."""
    _fresh(f"""
import torch
from paper_2606_13740_gb300 import serve
N, V = 64, 90000
z = torch.randn(N, V, device="cuda").to({'torch.float32' if dtype == 'f32' else 'torch.bfloat16'})
for n, nb in ((7664, 0), (7665, 0), (7632, 48), (7680, 0), (7681, 0), (8192, 0), (20000, 0)):
    ids = torch.randperm(V, device="cuda")[:n].to(torch.int32)
    more = {{}} if not nb else dict(bias_ids=torch.full((N, nb), -1, dtype=torch.int32, device="cuda"),
                                  bias=torch.zeros(N, nb, device="cuda"))
    out = torch.empty_like(z)
    x0, _, _ = serve.dllm_serve_logits(z, hist=ids.repeat(N, 1), rep=torch.full((N,), 2.0, device="cuda"), out=out, **more)
    want = z.clone()
    w = z[:, ids.long()]
    want[:, ids.long()] = torch.where(w > 0, w / 2, w * 2)
    assert torch.equal(out, want), (n, nb)
    top = want.float().amax(1, keepdim=True)
    first = torch.where(want.float() == top, torch.arange(V, device="cuda"), V).amin(1)
    assert torch.equal(x0.long(), first), (n, nb)
""")


def test_logits_of_two_host_threads(dev):
    """Calls whose lists need shared memory of different sizes, on streams and workspaces of their own."""
    from paper_2606_13740_gb300 import serve
    import ctypes as C
    L = serve.serve_lib()
    N, V, wrong, keep = 64, 90000, [], []

    def job(n_hist):
        t = dict(z=torch.randn(N, V, device="cuda"), hist=torch.arange(n_hist, dtype=torch.int32, device="cuda").repeat(N, 1),
                 x0=torch.empty(N, dtype=torch.int32, device="cuda"),
                 ws=torch.empty(serve._logits_bytes(N, V), dtype=torch.uint8, device="cuda"), stream=torch.cuda.Stream())
        a = serve.dllm_serve_logits_args()
        a.logits, a.ld, a.dtype, a.rows, a.vocab, a.mask_id, a.n_req = t["z"].data_ptr(), V, 2, N, V, -1, N
        a.hist, a.hist_ld, a.x0 = t["hist"].data_ptr(), n_hist, t["x0"].data_ptr()
        a.ws, a.ws_bytes = t["ws"].data_ptr(), t["ws"].numel()
        keep.append((t, a))

        def loop():
            for _ in range(20000):
                rc = L.dllm_serve_logits(C.byref(a), t["stream"].cuda_stream)
                if rc:
                    wrong.append((n_hist, rc, L.dllm_last_error(None)))
                    return
        return loop

    threads = [threading.Thread(target=job(n)) for n in (7700, 8192)]
    torch.cuda.synchronize()
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong, wrong
    for t, _ in keep:
        assert torch.equal(t["x0"].long(), t["z"].argmax(1))


@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_attention_reports_each_prefix_page_outside_the_pool(dev, page):
    """Any page of the prefix, not the first of a block of 64 keys alone: reported, and read as zeros."""
    from paper_2606_13740_gb300 import DllmError
    x = Paged([20, 90], [2, 3], 300, page, 4, 2, 64, seed=22)
    x.check()
    k0, v0 = x.k[0].clone(), x.v[0].clone()
    n_pages = x.kc.shape[0]
    for i in range(x.prefix.numel()):
        bad = x.prefix.clone()
        bad[i] = (-1, n_pages, 1 << 30, -2 ** 31)[i % 4]
        out = x.s.dllm_serve_attention(x.q, x.kc, x.vc, bad)
        with pytest.raises(DllmError, match="status bits 16"):
            x.s.dllm_serve_check()
        x.k[0][i * page:(i + 1) * page] = 0
        x.v[0][i * page:(i + 1) * page] = 0
        want, size, _ = x.want()
        assert bool(((out.double() - want).abs() <= U["bf16"] * want.abs() + (U["bf16"] + 2e-5) * size).all())
        x.k[0].copy_(k0), x.v[0].copy_(v0)
    x.check()


# ------------------------------------------------------------------ logits
@pytest.mark.parametrize("N,V,R,dtype", [(6, 20001, 6, "f32"), (64, 1024, 2, "bf16"), (6, 3000, 2, "f16")])
def test_logits_of_a_grammar_that_there_is_not(dev, N, V, R, dtype):
    """A row that names a grammar past the last one is allowed nothing; the others are as they were."""
    c = _logits_case(N, V, R, dtype, 23)
    c["grammar_row"][1::3] = 0
    c["cur"][:] = c["cur"] % (V - 1)
    good = {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in c.items()}
    rows = np.arange(0, N, 3)
    c["grammar_row"][rows] = np.array([3, 1 << 30, 4] * N, np.int32)[:len(rows)]
    for kw in (dict(), dict(inplace=True), dict(ld=V + 3)):
        z, x0, conf, tok = _logits_run(c, V - 1, **kw)
        want = _logits_run(good, V - 1, **kw)
        assert np.all(z[rows] == -np.inf) and np.all(x0[rows] == -1) and np.all(conf[rows] == 0) and np.all(tok[rows] == 0)
        rest = np.setdiff1d(np.arange(N), rows)
        for got, w in zip((z, x0, conf, tok), want):
            assert np.array_equal(got[rest], w[rest])
    _, x0, conf, _ = _logits_run(c, V - 1, out=False)
    assert np.all(x0[rows] == -1) and np.all(conf[rows] == 0)


# ------------------------------------------------------------------ plan
def test_plan_lengths_at_the_end_of_32_bits(dev):
    """A refused request of 2^31 - 1 new tokens: its rows are those that are left, the requests before it and their
    attention are as without it."""
    from paper_2606_13740_gb300 import DllmError
    x = Paged([10, 70], [5, 3], 40, 16, 28, 4, 128, seed=24, pad=150)
    x.check()
    for causal in (False, True):
        s = _serve(max_batch=5, max_rows=158, page=16, n_pages=x.kc.shape[0], max_pages=8, n_heads=28, n_kv_heads=4, head_dim=128)
        s.table[:2, :6].copy_(x.s.table[:2]), s.held[:2].copy_(x.s.held[:2]), s.ring_pos.zero_()
        most = 2 ** 31 - 1
        s.dllm_serve_plan(_i32([10, 70, 0, 4, most]), _i32([5, 3, most, most, most]), 158, prefix_len=40, causal=causal)
        assert s.row_start.cpu().tolist() == [0, 5, 8, most, most, most]
        assert s.n_keys.cpu().tolist() == [15, 73, 0, 0, 0] and s.req.cpu().tolist() == [0] * 5 + [1] * 3 + [2] * 150
        assert s.slot[8:].cpu().tolist() == [-1] * 150 and s.pos[8:].cpu().tolist() == [0] * 150
        assert torch.equal(s.slot[:8], x.s.slot[:8]) and torch.equal(s.pos[:8], x.s.pos[:8])
        out = s.dllm_serve_attention(x.q, x.kc, x.vc, x.prefix)
        with pytest.raises(DllmError, match="status bits 10"):  # lengths, rows
            s.dllm_serve_check()
        # the refused rows see the prefix alone
        x.causal = causal
        want, size, _ = x.want()
        k, v = (y[0].double().repeat_interleave(7, 1) for y in (x.k, x.v))
        z = torch.einsum("thd,khd->htk", x.q[8:].double(), k) * 128 ** -0.5
        p = torch.softmax(z, -1)
        want[8:] = torch.einsum("htk,khd->thd", p, v).reshape(150, -1)
        size[8:] = torch.einsum("htk,khd->thd", p, v.abs()).reshape(150, -1)
        assert bool(((out.double() - want).abs() <= U["bf16"] * want.abs() + (U["bf16"] + 2e-5) * size).all())


def test_plan_positions_stay_within_32_bits(dev):
    """Prefix and own positions together fit 32 bits, or the request is refused (half a gigabyte of lists)."""
    from paper_2606_13740_gb300 import DllmError
    n = (1 << 22) + 2
    s = _serve(max_batch=2, max_rows=8, page=256, n_pages=n, max_pages=n, n_heads=4, n_kv_heads=2, head_dim=64)
    P = (1 << 30) - 1
    s.dllm_serve_plan(_i32([(1 << 30) - 2, 3]), _i32([2, 2]), 4, prefix_len=P)
    s.dllm_serve_check()
    assert s.pos[:4].cpu().tolist() == [2 ** 31 - 3, 2 ** 31 - 2, P + 3, P + 4] and s.n_keys.cpu().tolist() == [1 << 30, 5]
    s.dllm_serve_plan(_i32([(1 << 30) - 1, 5]), _i32([2, 1]), 3, prefix_len=P)
    assert s.pos[:3].cpu().tolist() == [0, 0, P + 5] and s.slot[:2].cpu().tolist() == [-1, -1]
    assert s.n_keys.cpu().tolist() == [0, 6] and s.held.cpu().tolist() == [1 << 22, 1]
    with pytest.raises(DllmError, match="status bits 2"):
        s.dllm_serve_check()


@pytest.mark.parametrize("B", [1, 7, 300, 4096])
def test_plan_takes_its_own_key_counts_as_lengths(dev, B):
    """The step after: length is the plan's own n_keys, which it replaces."""
    r = np.random.default_rng(B)
    s = _serve(max_batch=B, max_rows=B * 20, page=16, n_pages=B * 8 + 8, max_pages=9, n_heads=4, n_kv_heads=2, head_dim=64)
    pool, have = Pool(B, 16, B * 8 + 8, 9), [0] * B
    for step in range(6):
        Q = r.integers(0, 20, B).tolist()
        rows = sum(Q)
        want = pool.plan(have, Q, rows, 3)
        s.dllm_serve_plan(s.n_keys[:B], _i32(Q), rows, prefix_len=3)
        _same_plan(s, pool, want, B, rows)
        s.dllm_serve_check()
        have = want["n_keys"]


# ------------------------------------------------------------------ more of the attention
def test_attention_refuses_the_plan_of_another_head_dim(dev):
    """Buffers laid out and planned for heads of 64 are too small for the parts of heads of 128: zeros, and a report."""
    import ctypes as C
    from paper_2606_13740_gb300 import DllmError, serve
    kw = dict(max_batch=2, max_rows=8, page=16, n_pages=8, max_pages=4, n_heads=4, n_kv_heads=2)
    s = _serve(head_dim=64, **kw)
    s.dllm_serve_plan(_i32([0, 20]), _i32([4, 4]), 8)
    c = serve.ServeConfig(head_dim=128, **kw).c()
    q = torch.ones(8, 4, 128, device="cuda", dtype=torch.bfloat16)
    kc = torch.ones(8, 2, 16, 128, device="cuda", dtype=torch.bfloat16)
    out = torch.full((8, 512), 9.0, device="cuda", dtype=torch.bfloat16)
    assert s._L.dllm_serve_attention(C.byref(c), s._tp, q.data_ptr(), 512, kc.data_ptr(), kc.data_ptr(), None, 0, 0.1,
                                     out.data_ptr(), None, 8, s._stream()) == 0
    with pytest.raises(DllmError, match="status bits 64"):
        s.dllm_serve_check()
    assert bool((out == 0).all())


@pytest.mark.parametrize("H,Hkv,hd,dtype", [(28, 4, 128, "bf16"), (4, 4, 64, "f16"), (32, 32, 128, "f16"), (3, 1, 128, "bf16")])
@pytest.mark.parametrize("L,Q,P,page", [([0, 100], [300, 70], 200, 16), ([5], [200], 0, 64), ([0, 0, 60], [1, 64, 9], 64, 128)])
def test_causal_rows_do_not_see_later_values(dev, H, Hkv, hd, dtype, L, Q, P, page):
    """Infinities and NaN among the values (and keys) of later tokens leave the rows before them as they are; the rows
    that see them get what the softmax makes of them."""
    x = Paged(L, Q, P, page, H, Hkv, hd, dtype=dtype, causal=True, seed=25)
    clean = x.check()
    table = x.s.table.cpu().tolist()
    start = np.cumsum([0] + Q)
    G = H // Hkv
    ok = torch.ones(sum(Q), H, hd, dtype=torch.bool, device="cuda")
    sums = torch.zeros(sum(Q), H, hd, device="cuda")
    r, placed = np.random.default_rng(26), set()
    for b in range(len(L)):
        for _ in range(4):
            t = int(r.integers(0, Q[b]))  # a new token's value
            at, h, f = L[b] + t, int(r.integers(0, Hkv)), int(r.integers(0, hd))
            v = float(r.choice([np.inf, -np.inf, np.nan]))
            if (b, t, h, f) in placed:
                continue
            placed.add((b, t, h, f))
            x.vc[table[b][at // page], h, at % page, f] = v
            rows = slice(int(start[b]) + t, int(start[b + 1]))
            ok[rows, h * G:(h + 1) * G, f] = False
            sums[rows, h * G:(h + 1) * G, f] += v
    out, lse = x.call(lse=True)
    x.s.dllm_serve_check()
    out = out.view(sum(Q), H, hd)
    assert torch.equal(out[ok], clean.view(sum(Q), H, hd)[ok])
    assert torch.equal(out[~ok].float().nan_to_num(7.0, 8.0, 9.0), sums[~ok].nan_to_num(7.0, 8.0, 9.0))
    assert bool(torch.isfinite(lse).all())
    # a key that is not a number: the rows from it on, all features
    b = int(np.argmax(Q))
    t = Q[b] // 2
    at = L[b] + t
    x.kc[table[b][at // page], 0, at % page, 0] = float("nan")
    out = x.call().view(sum(Q), H, hd)
    gone = torch.zeros_like(ok)
    gone[int(start[b]) + t:int(start[b + 1]), :G] = True
    assert bool(out[gone].isnan().all()) and torch.equal(out[ok & ~gone], clean.view(sum(Q), H, hd)[ok & ~gone])


def test_norm_refuses_rows_past_the_plan(dev):
    """Slots past a plan's rows are an earlier plan's."""
    s = _serve(max_batch=2, max_rows=8, page=16, n_pages=8, max_pages=4, n_heads=4, n_kv_heads=2, head_dim=64)
    s.dllm_serve_plan(_i32([0, 0]), _i32([4, 4]), 8)
    s.dllm_serve_plan(_i32([4, 4]), _i32([1, 1]), 2)
    x = torch.randn(8, 8 * 64, device="cuda").to(torch.bfloat16)
    kc = torch.zeros(8, 2, 16, 64, device="cuda", dtype=torch.bfloat16)
    vc, theta = torch.zeros_like(kc), torch.ones(32, device="cuda")
    with pytest.raises(ValueError, match="rows"):
        s.dllm_serve_qk_norm_rope(x[:, :256], x[:, 256:384], x[:, 384:], theta, kc, vc)
    s.dllm_serve_qk_norm_rope(x[:2, :256], x[:2, 256:384], x[:2, 384:], theta, kc, vc)
    assert int((kc != 0).any(-1).any(1).sum()) == 2
