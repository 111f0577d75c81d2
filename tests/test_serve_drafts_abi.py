"""The drafts' header and its binding: every entry point exported and typed, the structure of the size the library
reads, and the refusals that need no GPU."""
import ctypes as C
import os
import re
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")
from test_serve_refusals import P, _bf16, _f32, _handle, _i32, _on  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    from paper_2606_13740_gb300 import serve
    return serve.serve_lib()


def _header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "dllm_serve_drafts.h")).read(), flags=re.S)


def test_binding_covers_the_header(L):
    from paper_2606_13740_gb300 import serve
    names = set(re.findall(r"\bint (dllm_serve_\w+)\s*\(", _header()))
    assert names == set(serve.DRAFT_SIGNATURES) and all(hasattr(L, n) for n in names)
    body = re.search(r"typedef struct \{([^}]*)\} dllm_serve_logprobs_args;", _header()).group(1)
    fields = [f.strip(" *\n") for line in body.split(";") if line.strip()
              for f in re.sub(r"^(const )?\w+", "", line.strip()).split(",")]
    assert fields == [n for n, _ in serve.dllm_serve_logprobs_args._fields_]
    bits = dict(re.findall(r"DLLM_(SERVE_\w+) = (\d+)", _header()))
    assert bits == {"SERVE_TREE": str(serve.SERVE_TREE), "SERVE_SHARED": str(serve.SERVE_SHARED)}


def _setup(L):
    from paper_2606_13740_gb300 import serve
    c = serve.ServeConfig(max_batch=4, max_rows=64, n_heads=4, n_kv_heads=2, head_dim=64).c()
    t = serve.dllm_serve_tables()
    assert L.dllm_serve_layout(C.byref(c), 4096, C.byref(t), None) == 0  # (never followed: the calls are refused)
    return C.byref(c), c, C.byref(t), t


def test_calls_refuse_bad_arguments(L):
    from paper_2606_13740_gb300 import serve
    cp, c, tp, t = _setup(L)
    empty = C.byref(serve.dllm_serve_tables())

    def tree(parent=P, mask=P, words=1, rows=4, tables=tp):
        return L.dllm_serve_tree(cp, tables, parent, mask, words, rows, None)

    for bad in (dict(parent=None), dict(mask=None), dict(parent=P + 2), dict(mask=P + 1), dict(words=0), dict(words=1025),
                dict(rows=-1), dict(rows=65), dict(tables=empty), dict(tables=None)):
        assert tree(**bad) == -1, bad
    assert tree(rows=0, parent=None, mask=None) == 0

    def attn(q=P, ldq=256, kc=P, vc=P, pages=P, n=1, scale=0.1, out=P, lse=None, mask=P, words=1, rows=4, tables=tp):
        return L.dllm_serve_tree_attention(cp, tables, q, ldq, kc, vc, pages, n, scale, mask, words, out, lse, rows, None)

    for bad in (dict(q=None), dict(q=P + 8), dict(ldq=248), dict(ldq=260), dict(kc=None), dict(vc=P + 2), dict(pages=None),
                dict(pages=P + 2), dict(n=-1), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(out=None),
                dict(out=P + 16), dict(lse=P + 2), dict(mask=None), dict(mask=P + 2), dict(words=0), dict(words=(1 << 16) + 1),
                dict(rows=65), dict(rows=-1), dict(tables=empty)):
        assert attn(**bad) == -1, bad
    assert attn(rows=0, q=None, out=None, mask=None) == 0

    def accept(parent=P, ids=P, x0=P, batch=2, rows=4, most=3, keep=P, n=P, nxt=P, tables=tp):
        return L.dllm_serve_accept(cp, tables, parent, ids, x0, batch, rows, most, keep, n, nxt, None)

    for bad in (dict(parent=None), dict(ids=None), dict(x0=None), dict(keep=None), dict(n=None), dict(nxt=None), dict(ids=P + 2),
                dict(keep=P + 1), dict(nxt=P + 2), dict(batch=0), dict(batch=5), dict(rows=-1), dict(rows=65), dict(most=0),
                dict(most=(1 << 22) + 1), dict(tables=None)):
        assert accept(**bad) == -1, bad

    def pointers(*p):
        return (C.c_void_p * len(p))(*p)

    def caches(call):
        good = dict(kc=pointers(P, P + 4096), vc=pointers(2 * P, 2 * P + 4096), layers=2)
        for bad in (dict(kc=None), dict(vc=None), dict(layers=0), dict(layers=129), dict(kc=pointers(P, None)),
                    dict(vc=pointers(2 * P, 2 * P + 8)), dict(kc=pointers(P, P)), dict(vc=pointers(2 * P, P))):
            assert call(**{**good, **bad}) == -1, bad
        return good

    def compact(kc, vc, layers, first=P, keep=P, ld=3, n=P, batch=2, tables=tp):
        return L.dllm_serve_compact(cp, tables, kc, vc, layers, first, keep, ld, n, batch, None)

    good = caches(compact)
    for bad in (dict(first=None), dict(keep=None), dict(n=None), dict(first=P + 2), dict(keep=P + 2), dict(n=P + 1), dict(ld=-1),
                dict(batch=0), dict(batch=5), dict(tables=empty)):
        assert compact(**good, **bad) == -1, bad

    def fork(kc, vc, layers, src=P, length=P, batch=2, tables=tp):
        return L.dllm_serve_fork(cp, tables, kc, vc, layers, src, length, batch, None)

    good = caches(fork)
    for bad in (dict(src=None), dict(length=None), dict(src=P + 2), dict(length=P + 3), dict(batch=0), dict(batch=5),
                dict(tables=empty)):
        assert fork(**good, **bad) == -1, bad

    # tables that are misaligned, a bad config
    for name, _ in serve.dllm_serve_tables._fields_:
        t2 = serve.dllm_serve_tables()
        assert L.dllm_serve_layout(cp, 4096, C.byref(t2), None) == 0
        setattr(t2, name, getattr(t2, name) + (8 if name in ("work", "partials") else 2))
        off = dict(tables=C.byref(t2))
        assert {tree(**off), attn(**off), accept(**off), compact(**good, **off), fork(**good, **off)} == {-1}, name
    c.page = 17
    assert {tree(), attn(), accept(), compact(**good), fork(**good)} == {-1}


def test_logprobs_refuse_bad_arguments(L):
    from paper_2606_13740_gb300 import serve
    def call(**over):
        a = serve.dllm_serve_logprobs_args()
        good = dict(logits=P, ld=1000, dtype=2, rows=4, vocab=1000, mask_id=999, tokens=P, n_tokens=1, n_top=3, lp=P, entropy=P, lse=P,
                    top_ids=P, top_lp=P)
        for k, v in {**good, **over}.items():
            setattr(a, k, v)
        return L.dllm_serve_logprobs(C.byref(a), None)

    for bad in (dict(logits=None), dict(rows=-1), dict(vocab=0), dict(ld=999), dict(dtype=3), dict(mask_id=1000), dict(mask_id=-2),
                dict(logits=P + 2), dict(logits=P + 1, dtype=0), dict(tokens=None), dict(lp=None), dict(top_ids=None),
                dict(top_lp=None), dict(n_tokens=-1), dict(n_tokens=(1 << 20) + 1), dict(n_top=-1), dict(n_top=33),
                dict(n_top=0, n_tokens=0, lse=None, entropy=None),
                *(dict([(k, P + 2)]) for k in ("tokens", "lp", "entropy", "lse", "top_ids", "top_lp"))):
        assert call(**bad) == -1, bad
    assert L.dllm_serve_logprobs(None, None) == -1 and call(rows=0, logits=None) == 0


@pytest.fixture
def serve(monkeypatch):
    """The binding, as on a machine whose current device is cuda:0, with a library that launches nothing."""
    from paper_2606_13740_gb300 import serve
    serve.serve_lib()

    def launch(*a):
        raise AssertionError("launched")

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(serve, "_stream_of", lambda: lambda index: 0)
    monkeypatch.setattr(serve, "_lib", SimpleNamespace(**{n: launch for n in serve.DRAFT_SIGNATURES}))
    return serve


def test_tensors_lie_on_the_current_device(serve, monkeypatch):
    """Each call with one tensor on cuda:1 or in host memory, of another type or another shape: refused; else it gets
    through; and none on another device than the current one."""
    real = torch.empty

    def calls(index, **at):
        s = _handle(serve, index)

        def i32(name, *shape):
            how = at.get(name)
            if how == "type":
                return _on(index, torch.zeros(shape, dtype=torch.int64))
            if how == "shape":
                return _on(index, torch.zeros(tuple(n + 1 for n in shape), dtype=torch.int32))
            return _i32(index if how is None else how, *shape)

        cache = [_bf16(at.get("cache", index), 4, 2, 16, 64) for _ in range(4)]
        q = _bf16(at.get("q", index), 4, 128)
        return {
            "parent mask": lambda: s.dllm_serve_tree(i32("parent", 4), 40, i32("mask", 4, 2)),
            "bits q cache": lambda: s.dllm_serve_tree_attention(q, cache[0], cache[1], i32("bits", 4, 2), out=_bf16(index, 4, 128)),
            "parent ids x0": lambda: s.dllm_serve_accept(i32("parent", 4), i32("ids", 4), i32("x0", 4), 2, 3),
            "first keep n cache": lambda: s.dllm_serve_compact(s.layers(cache[:2], cache[2:]), i32("first", 2),
                                                               _i32(index, 2, 3) if at.get("keep") in ("shape",) else i32("keep", 2, 3),
                                                               i32("n", 2)),
            "src length cache": lambda: s.dllm_serve_fork(s.layers(cache[:2], cache[2:]), i32("src", 2), i32("length", 2)),
        }

    for call in calls(0).values():
        with pytest.raises(AssertionError, match="launched"):
            call()
    for call in calls(1).values():
        with pytest.raises(ValueError, match="current"):
            call()
    for names in calls(0):
        for name in names.split():
            for how in (1, -1) + (() if name in ("q", "cache", "keep") else ("type", "shape")):
                with pytest.raises(ValueError):
                    calls(0, **{name: how})[names]()
    s = _handle(serve, 0)
    with pytest.raises(ValueError, match="caches"):
        s.layers([_bf16(0, 4, 2, 16, 64)], [])
    with pytest.raises(ValueError, match="words"):
        s.dllm_serve_tree_attention(_bf16(0, 4, 128), None, None, _i32(0, 4))

    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: SimpleNamespace(
        data_ptr=lambda: P, numel=lambda: P, element_size=lambda: 1, unbind=lambda d: (_f32(0, 4), _f32(0, 4))))

    def logprobs(z=0, tokens=0, top=2, shape=(4, 2)):
        serve.dllm_serve_logprobs(_f32(z, 4, 100), _i32(tokens, *shape), 99, top)

    with pytest.raises(AssertionError, match="launched"):
        logprobs()
    for bad in (dict(z=1), dict(z=-1), dict(tokens=1), dict(tokens=-1), dict(top=33), dict(top=-1), dict(shape=(3, 2)),
                dict(shape=(4,))):
        with pytest.raises(ValueError):
            logprobs(**bad)
    monkeypatch.setattr(torch, "empty", real)
