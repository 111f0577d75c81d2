"""The serving header and its binding: every entry point exported and typed, structures of the sizes the
library reads, and the refusals that need no GPU."""
import ctypes as C
import os
import re

import pytest

pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    from paper_2606_13740_gb300 import serve
    return serve.serve_lib()


def _header():
    src = open(os.path.join(ROOT, "include", "dllm_serve.h")).read()
    return re.sub(r"/\*.*?\*/", "", src, flags=re.S)


def test_binding_covers_the_header(L):
    from paper_2606_13740_gb300 import serve
    names = set(re.findall(r"\bint (dllm_serve_\w+)\s*\(", _header()))
    assert names == set(serve.SIGNATURES) and len(names) == 8
    assert all(hasattr(L, n) for n in names)


@pytest.mark.parametrize("name", ["dllm_serve_config", "dllm_serve_tables", "dllm_serve_logits_args"])
def test_structures_match_the_header(name):
    from paper_2606_13740_gb300 import serve
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, _header()).group(1)
    fields = []
    for line in body.split(";"):
        line = line.strip()
        if line:
            line = re.sub(r"^(const )?\w+", "", line)
            fields += [f.strip(" *\n") for f in line.split(",")]
    assert fields == [n for n, _ in getattr(serve, name)._fields_]


@pytest.mark.parametrize("bad", [
    dict(max_batch=0), dict(max_batch=4097), dict(max_rows=0), dict(max_rows=(1 << 22) + 1), dict(page=8), dict(page=48),
    dict(page=512), dict(n_pages=0), dict(n_pages=1 << 26, page=64), dict(max_pages=0), dict(max_pages=1 << 26, page=64),
    dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=30, n_kv_heads=4), dict(n_heads=256, n_kv_heads=1),
    dict(head_dim=96), dict(page_stride=64), dict(page_stride=32 * 64 * 128 + 4)])
def test_bad_configs_are_refused(bad):
    from paper_2606_13740_gb300 import DllmError, serve
    with pytest.raises(DllmError) as e:
        serve.dllm_serve_bytes(serve.ServeConfig(**bad))
    assert e.value.code == -1 and "serve config" in str(e.value)
    with pytest.raises(ValueError):
        serve.dllm_serve_bytes(serve.ServeConfig(dtype="f32"))


def test_layout_is_dense_and_aligned(L):
    from paper_2606_13740_gb300 import serve
    cfg = serve.ServeConfig(max_batch=3, max_rows=77, n_pages=5, max_pages=9)
    c, t, n = cfg.c(), serve.dllm_serve_tables(), C.c_size_t()
    assert L.dllm_serve_layout(C.byref(c), 4096, C.byref(t), C.byref(n)) == 0
    at = [getattr(t, f) for f, _ in t._fields_]
    assert at == sorted(at) and at[0] == 4096 and all(p % 256 == 0 for p in at) and at[-1] <= 4096 + n.value
    assert t.held - t.table >= 3 * 9 * 4 and t.pos - t.slot >= 77 * 4 and t.n_keys - t.row_start >= 4 * 4
    assert n.value == serve.dllm_serve_bytes(cfg)
    assert L.dllm_serve_layout(C.byref(c), 4097, C.byref(t), None) == -1


def _tables(L, c):
    from paper_2606_13740_gb300 import serve
    t = serve.dllm_serve_tables()
    assert L.dllm_serve_layout(C.byref(c), 4096, C.byref(t), None) == 0  # (never followed: the calls are refused)
    return t


P = 1 << 20  # an aligned address that no refused call follows


def test_calls_refuse_bad_arguments(L):
    from paper_2606_13740_gb300 import serve
    c = serve.ServeConfig(max_batch=4, max_rows=64, n_heads=4, n_kv_heads=2, head_dim=64).c()
    t = _tables(L, c)
    cp, tp, empty = C.byref(c), C.byref(t), serve.dllm_serve_tables()

    def plan(length=P, q_len=P, batch=2, rows=8, prefix=0, tables=tp):
        return L.dllm_serve_plan(cp, tables, length, q_len, batch, rows, prefix, 0, None)

    for bad in (dict(length=None), dict(q_len=None), dict(batch=0), dict(batch=5), dict(rows=-1), dict(rows=65),
                dict(prefix=-1), dict(prefix=1 << 30), dict(tables=C.byref(empty)), dict(tables=None)):
        assert plan(**bad) == -1, bad

    def norm(q=P, k=P, v=P, kind=0, ldq=256, ldk=128, ldv=128, eps=1e-5, theta=P, out=P, ldo=256, kc=P, vc=P, rows=4):
        return L.dllm_serve_qk_norm_rope(cp, tp, q, k, v, kind, ldq, ldk, ldv, None, None, eps, theta, out, ldo, kc, vc,
                                         rows, None)

    for bad in (dict(q=None), dict(k=None), dict(v=P + 8), dict(kind=1), dict(kind=3), dict(ldq=248), dict(ldk=120),
                dict(ldv=132), dict(ldo=200), dict(eps=-1.0), dict(eps=float("nan")), dict(theta=None), dict(out=None),
                dict(kc=None), dict(vc=P + 2), dict(rows=-1), dict(rows=65), dict(kind=2, out=P, q=P), dict(ldo=264)):
        assert norm(**bad) == -1, bad

    def attn(q=P, ldq=256, kc=P, vc=P, pages=P, n=1, scale=0.1, out=P, rows=4):
        return L.dllm_serve_attention(cp, tp, q, ldq, kc, vc, pages, n, scale, out, None, rows, None)

    for bad in (dict(q=None), dict(ldq=248), dict(ldq=260), dict(kc=None), dict(vc=P + 2), dict(pages=None), dict(n=-1),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(out=None), dict(out=P + 16),
                dict(rows=65), dict(rows=-1)):
        assert attn(**bad) == -1, bad
    # no rows: nothing to do, and no GPU needed for it
    assert norm(rows=0, q=None, k=None, v=None, out=None) == 0 and attn(rows=0, q=None, out=None) == 0
    assert L.dllm_serve_check(None, None, None) == -1


def test_logits_refuse_bad_arguments(L):
    from paper_2606_13740_gb300 import serve
    n = C.c_size_t()
    assert L.dllm_serve_logits_bytes(4, 1000, C.byref(n)) == 0 and n.value > 0
    assert L.dllm_serve_logits_bytes(-1, 1000, C.byref(n)) == -1 and L.dllm_serve_logits_bytes(1, 0, C.byref(n)) == -1
    assert L.dllm_serve_logits_bytes(1, 1000, None) == -1

    def call(**over):
        a = serve.dllm_serve_logits_args()
        good = dict(logits=P, ld=1000, dtype=0 + 2, rows=4, vocab=1000, mask_id=999, x0=P, ws=P, ws_bytes=n.value)
        for k, v in {**good, **over}.items():
            setattr(a, k, v)
        return L.dllm_serve_logits(C.byref(a), None)

    for bad in (dict(logits=None), dict(rows=-1), dict(vocab=0), dict(ld=999), dict(dtype=3), dict(mask_id=1000),
                dict(mask_id=-2), dict(logits=P + 2), dict(out=P + 1, ld_out=1000), dict(out=P, ld_out=999),
                dict(out=P, ld_out=1004), dict(hist=P, hist_ld=4), dict(hist=P, n_req=1, hist_ld=1 << 20),
                dict(bias_ids=P, n_req=1, bias_ld=4), dict(bias_ids=P, bias=P, n_req=1, bias_ld=4096),
                dict(grammar=P, n_grammar=1), dict(tokconf=P), dict(x0=None), dict(ws=None), dict(ws=P + 8),
                dict(ws_bytes=n.value - 1)):
        assert call(**bad) == -1, bad
    assert L.dllm_serve_logits(None, None) == -1
    assert call(rows=0, logits=None, ws=None) == 0
