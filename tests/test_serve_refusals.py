"""Refusals of the serving calls that need no GPU: devices that are not the current one, tensors that lie elsewhere,
pointers of 32-bit values that are not aligned."""
import ctypes as C
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def serve(monkeypatch):
    """The binding, as on a machine whose current device is cuda:0, with a library that launches nothing."""
    from paper_2606_13740_gb300 import serve
    serve.serve_lib()

    def launch(*a):
        raise AssertionError("launched")

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(serve, "_stream_of", lambda: lambda index: 0)
    monkeypatch.setattr(serve, "_lib", SimpleNamespace(**{n: launch for n in serve.SIGNATURES}))
    monkeypatch.setattr(serve, "_logits_bytes", lambda rows, vocab: 16)
    return serve


def _handle(serve, index):
    """A Serve of device `index` (2 heads of 64, pages of 16), without its buffers."""
    s = serve.Serve.__new__(serve.Serve)
    s.cfg = serve.ServeConfig(max_batch=2, max_rows=8, page=16, n_pages=4, max_pages=2, n_heads=2, n_kv_heads=2, head_dim=64)
    s._L, s._cp, s._tp, s._index, s.device = serve._lib, None, None, index, torch.device("cuda", index)
    s._dt, s._i32, s._f32, s._kinds = torch.bfloat16, torch.int32, torch.float32, serve._names()
    s._H, s._Hkv, s._hd, s._scale, s.rows, s.prefix_len = 2, 2, 64, 0.125, 4, 0
    s._cache_shape, s._cache_strides = (4, 2, 16, 64), (2048, 1024, 64, 1)
    s._empty = lambda shape, dtype, device: _on(index, torch.empty(shape, dtype=dtype))
    return s


def _on(index, x):
    """x as if it lay on device `index` (-1: in host memory)."""
    return SimpleNamespace(dtype=x.dtype, shape=x.shape, is_cuda=index >= 0, stride=x.stride, numel=x.numel,
                           device=torch.device("cuda", index) if index >= 0 else torch.device("cpu"),
                           is_contiguous=x.is_contiguous, get_device=lambda: index, data_ptr=lambda: 1 << 20,
                           element_size=x.element_size)


def _i32(index, *shape):
    return _on(index, torch.zeros(shape, dtype=torch.int32))


def _bf16(index, *shape):
    return _on(index, torch.zeros(shape, dtype=torch.bfloat16))


def _f32(index, *shape):
    return _on(index, torch.zeros(shape))


def test_a_handle_is_of_the_current_device(serve, monkeypatch):
    monkeypatch.setattr(serve, "dllm_serve_bytes", lambda cfg: 1 << 12)
    for device in ("cuda:1", torch.device("cuda", 3), "cpu"):
        with pytest.raises(ValueError, match="device"):
            serve.Serve(serve.ServeConfig(), device=device)


def test_calls_on_another_device_than_the_current_one(serve):
    """Each call with everything on cuda:1, cuda:0 being current: refused before it reaches the library."""
    s = _handle(serve, 1)
    q, cache = _bf16(1, 4, 128), _bf16(1, 4, 2, 16, 64)
    for call in (lambda: s.dllm_serve_reset(), lambda: s.dllm_serve_plan(_i32(1, 2), _i32(1, 2), 4),
                 lambda: s.dllm_serve_qk_norm_rope(q, q, q, _f32(1, 32), cache, cache, out=q),
                 lambda: s.dllm_serve_attention(q, cache, cache, out=q), lambda: s.dllm_serve_check(),
                 lambda: serve.dllm_serve_logits(_f32(1, 4, 100))):
        with pytest.raises(ValueError, match="current"):
            call()


def test_tensors_of_another_device_than_the_handle(serve):
    """One tensor of each call on cuda:1 or in host memory: refused; with all on cuda:0 it gets through."""
    s = _handle(serve, 0)

    def plan(length=0, q_len=0):
        s.dllm_serve_plan(_i32(length, 2), _i32(q_len, 2), 4)

    def norm(q=0, k=0, v=0, theta=0, kc=0, vc=0, gain=0, out=0):
        s.dllm_serve_qk_norm_rope(_bf16(q, 4, 128), _bf16(k, 4, 128), _bf16(v, 4, 128), _f32(theta, 32),
                                  _bf16(kc, 4, 2, 16, 64), _bf16(vc, 4, 2, 16, 64), q_gain=_f32(gain, 64), out=_bf16(out, 4, 128))

    def attention(q=0, kc=0, vc=0, pages=0, out=0):
        s.dllm_serve_attention(_bf16(q, 4, 128), _bf16(kc, 4, 2, 16, 64), _bf16(vc, 4, 2, 16, 64), _i32(pages, 1),
                               out=_bf16(out, 4, 128))

    for call, names in ((plan, "length q_len"), (norm, "q k v theta kc vc gain out"), (attention, "q kc vc pages out")):
        with pytest.raises(AssertionError, match="launched"):
            call()
        for name in names.split():
            for index in (1, -1):
                with pytest.raises(ValueError):
                    call(**{name: index})


def test_logits_take_tensors_of_one_device(serve, monkeypatch):
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: SimpleNamespace(
        data_ptr=lambda: 1 << 20, numel=lambda: 1 << 20, element_size=lambda: 1, unbind=lambda d: (_f32(0, 4), _f32(0, 4))))

    def call(**at):
        d = {k: at.get(k, 0) for k in ("req", "hist", "hist_len", "rep", "bias_ids", "bias", "grammar", "row", "cur", "out", "ws")}
        serve.dllm_serve_logits(
            _f32(0, 4, 100), req=_i32(d["req"], 4), hist=_i32(d["hist"], 2, 7), hist_len=_i32(d["hist_len"], 2),
            rep=_f32(d["rep"], 2), bias_ids=_i32(d["bias_ids"], 2, 3), bias=_f32(d["bias"], 2, 3),
            grammar=_i32(d["grammar"], 1, 4), grammar_row=_i32(d["row"], 4), cur=_i32(d["cur"], 4),
            out=_f32(d["out"], 4, 100), ws=_on(d["ws"], torch.zeros(64, dtype=torch.uint8)))

    with pytest.raises(AssertionError, match="launched"):
        call()
    for name in ("req", "hist", "hist_len", "rep", "bias_ids", "bias", "grammar", "row", "cur", "out", "ws"):
        for index in (1, -1):
            with pytest.raises(ValueError):
                call(**{name: index})


P = 1 << 20  # an aligned address that no refused call follows


def test_misaligned_words_are_refused():
    """Lengths, pages, lists and results two bytes off, and tables: a kernel would fault on them."""
    from paper_2606_13740_gb300 import serve
    L = serve.serve_lib()
    c = serve.ServeConfig(max_batch=4, max_rows=64, n_heads=4, n_kv_heads=2, head_dim=64).c()
    cp = C.byref(c)

    def tables(**off):
        t = serve.dllm_serve_tables()
        assert L.dllm_serve_layout(cp, 4096, C.byref(t), None) == 0
        for k, v in off.items():
            setattr(t, k, getattr(t, k) + v)
        return C.byref(t)

    def plan(length=P, q_len=P, t=None):
        return L.dllm_serve_plan(cp, t or tables(), length, q_len, 2, 8, 0, 0, None)

    def attention(pages=P, lse=P, t=None):
        return L.dllm_serve_attention(cp, t or tables(), P, 256, P, P, pages, 1, 0.1, P, lse, 4, None)

    def norm(t):
        return L.dllm_serve_qk_norm_rope(cp, t, P, P, P, 0, 256, 128, 128, None, None, 1e-5, P, P, 256, P, P, 4, None)

    assert plan(length=P + 2) == -1 and plan(q_len=P + 1) == -1
    assert attention(pages=P + 2) == -1 and attention(lse=P + 2) == -1
    for name, _ in serve.dllm_serve_tables._fields_:
        off = 8 if name in ("work", "partials") else 2
        for call in (plan, attention):
            assert call(t=tables(**{name: off})) == -1, name
        assert norm(tables(**{name: off})) == -1 and L.dllm_serve_reset(cp, tables(**{name: off}), None) == -1, name

    n = C.c_size_t()
    assert L.dllm_serve_logits_bytes(4, 1000, C.byref(n)) == 0
    words = ("req hist hist_len rep freq pres bias_ids bias bias_len grammar grammar_row cur x0 conf tokconf").split()
    for name in words:
        a = serve.dllm_serve_logits_args(ld=1000, dtype=2, rows=4, vocab=1000, mask_id=-1, n_req=4, hist_ld=8, bias_ld=8,
                                         n_grammar=1, ws_bytes=n.value, logits=P, ws=P, **{w: P for w in words})
        setattr(a, name, P + 2)
        assert L.dllm_serve_logits(C.byref(a), None) == -1, name
