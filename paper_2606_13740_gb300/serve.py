"""Python binding of ``include/dllm_serve.h``: the operators that serve a batch of unequal requests over a
paged K/V cache, under a prefix that all of them share.

Argument marshalling only.  Calls run on torch's current stream and do not wait; what a kernel found wrong
(lengths, a pool that ran out) is raised by ``Serve.dllm_serve_check``.  The library launches on the current
device: buffers and tensors of another one are refused.
"""
from __future__ import annotations

import ctypes as C
import functools
from dataclasses import dataclass

from .dllm import _check, lib

SERVE_TIMEOUT, SERVE_LENGTHS, SERVE_PAGES, SERVE_ROWS, SERVE_PREFIX, SERVE_SLOT, SERVE_STATE = 1, 2, 4, 8, 16, 32, 64
DTYPES = {"bf16": 0, "f16": 1, "f32": 2}

_P, _I, _F, _I64, _SZ = C.c_void_p, C.c_int, C.c_float, C.c_int64, C.c_size_t


class dllm_serve_config(C.Structure):
    _fields_ = [("max_batch", _I), ("max_rows", _I), ("page", _I), ("n_pages", _I), ("max_pages", _I), ("n_heads", _I),
                ("n_kv_heads", _I), ("head_dim", _I), ("dtype", _I), ("page_stride", _I64)]


class dllm_serve_tables(C.Structure):
    _fields_ = [(n, _P) for n in ("table", "held", "ring", "ring_pos", "row_start", "n_keys", "slot", "pos", "req",
                                  "status", "work", "partials")]


class dllm_serve_logits_args(C.Structure):
    _fields_ = [("logits", _P), ("out", _P), ("ld", _I64), ("ld_out", _I64), ("dtype", _I), ("rows", _I), ("vocab", _I),
                ("mask_id", _I), ("n_req", _I), ("req", _P), ("hist", _P), ("hist_len", _P), ("hist_ld", _I), ("rep", _P),
                ("freq", _P), ("pres", _P), ("bias_ids", _P), ("bias", _P), ("bias_len", _P), ("bias_ld", _I),
                ("grammar", _P), ("grammar_row", _P), ("n_grammar", _I), ("cur", _P), ("x0", _P), ("conf", _P),
                ("tokconf", _P), ("ws", _P), ("ws_bytes", _SZ)]


# name -> (restype, argtypes); every entry point of include/dllm_serve.h
SIGNATURES = {
    "dllm_serve_layout": (_I, [_P, _P, _P, _P]),
    "dllm_serve_reset": (_I, [_P, _P, _P]),
    "dllm_serve_plan": (_I, [_P, _P, _P, _P, _I, _I, _I, _I, _P]),
    "dllm_serve_qk_norm_rope": (_I, [_P, _P, _P, _P, _P, _I, _I64, _I64, _I64, _P, _P, _F, _P, _P, _I64, _P, _P, _I, _P]),
    "dllm_serve_attention": (_I, [_P, _P, _P, _I64, _P, _P, _P, _I, _F, _P, _P, _I, _P]),
    "dllm_serve_check": (_I, [_P, _P, _P]),
    "dllm_serve_logits_bytes": (_I, [_I, _I, _P]),
    "dllm_serve_logits": (_I, [_P, _P]),
}

_lib = None


def serve_lib():
    """The library with this header's entry points typed."""
    global _lib
    if _lib is None:
        L = lib()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


@dataclass
class ServeConfig:
    max_batch: int = 16
    max_rows: int = 512
    page: int = 64
    n_pages: int = 1024
    max_pages: int = 128
    n_heads: int = 32
    n_kv_heads: int = 32
    head_dim: int = 128
    dtype: str = "bf16"
    page_stride: int = 0

    def c(self):
        if self.dtype not in ("bf16", "f16"):
            raise ValueError(f"dtype must be 'bf16' or 'f16', not {self.dtype!r}")
        return dllm_serve_config(self.max_batch, self.max_rows, self.page, self.n_pages, self.max_pages, self.n_heads,
                                 self.n_kv_heads, self.head_dim, DTYPES[self.dtype], self.page_stride)


def dllm_serve_bytes(cfg: ServeConfig) -> int:
    n = _SZ()
    c = cfg.c()
    _check(serve_lib().dllm_serve_layout(C.byref(c), None, None, C.byref(n)))
    return n.value


@functools.cache
def _names():
    import torch

    return {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


@functools.cache
def _stream_of():
    """index of a device -> handle of torch's current stream there."""
    import torch

    return torch._C._cuda_getCurrentRawStream


def _stream_on(index):
    """Handle of torch's current stream on device `index`, which has to be the current device."""
    import torch

    now = torch.cuda.current_device()
    if now != index:
        raise ValueError(f"cuda:{index} is not the current device, cuda:{now} is")
    return _stream_of()(index)


@functools.cache
def _logits_bytes(rows, vocab):
    n = _SZ()
    _check(serve_lib().dllm_serve_logits_bytes(rows, vocab, C.byref(n)))
    return n.value


class Serve:
    """The buffers of one serving batch (a torch tensor), and the calls on them with the ABI's names.  The
    attributes table, held, ring, ring_pos, row_start, n_keys, slot, pos, req and status are int32 views of
    them.  One stream at a time."""

    def __init__(self, cfg: ServeConfig, device=None):
        import torch

        self.cfg = cfg
        self._c = cfg.c()
        self._cp = C.byref(self._c)
        self._L = L = serve_lib()
        n = dllm_serve_bytes(cfg)
        device = torch.device(device or "cuda")
        if device.type != "cuda":
            raise ValueError(f"device must be a CUDA device, not {device}")
        if device.index is not None:
            _stream_on(device.index)
        self.buffer = torch.empty(n, dtype=torch.uint8, device=device)
        self.device, self._index = self.buffer.device, self.buffer.device.index
        self._t = dllm_serve_tables()
        self._tp = C.byref(self._t)
        self._dt = {"bf16": torch.bfloat16, "f16": torch.float16}[cfg.dtype]
        self._i32, self._f32, self._empty, self._kinds = torch.int32, torch.float32, torch.empty, _names()
        self._H, self._Hkv, self._hd, self._scale = cfg.n_heads, cfg.n_kv_heads, cfg.head_dim, cfg.head_dim ** -0.5
        self._cache_shape = (cfg.n_pages, cfg.n_kv_heads, cfg.page, cfg.head_dim)
        row = cfg.page * cfg.head_dim
        self._cache_strides = (cfg.page_stride or cfg.n_kv_heads * row, row, cfg.head_dim, 1)
        _check(L.dllm_serve_layout(self._cp, self.buffer.data_ptr(), self._tp, None))
        base = self.buffer.data_ptr()

        def view(name, *shape):
            at = (getattr(self._t, name) - base) // 4
            count = 1
            for d in shape:
                count *= d
            return self.buffer.view(torch.int32)[at:at + count].view(*shape)

        self.table = view("table", cfg.max_batch, cfg.max_pages)
        self.held, self.n_keys = view("held", cfg.max_batch), view("n_keys", cfg.max_batch)
        self.ring, self.ring_pos = view("ring", cfg.n_pages), view("ring_pos", 2)
        self.row_start, self.status = view("row_start", cfg.max_batch + 1), view("status", 4)
        self.slot, self.pos, self.req = (view(n, cfg.max_rows) for n in ("slot", "pos", "req"))
        self.rows = self.prefix_len = 0
        self.dllm_serve_reset()

    def _stream(self):
        return _stream_on(self._index)

    def dllm_serve_reset(self):
        """Nothing held, every page free."""
        _check(self._L.dllm_serve_reset(self._cp, self._tp, self._stream()))
        self.rows = self.prefix_len = 0

    def dllm_serve_plan(self, length, q_len, rows, prefix_len=0, causal=False):
        """length, q_len: int32 CUDA tensors [batch], own positions cached and new tokens; rows: rows of the step's
        packed arrays (at least the sum of q_len, else the last are left out)."""
        i32, index = self._i32, self._index
        if (length.dtype != i32 or q_len.dtype != i32 or length.shape != q_len.shape or length.get_device() != index
                or q_len.get_device() != index or not length.is_contiguous() or not q_len.is_contiguous()):
            raise ValueError(f"length and q_len must be contiguous int32 tensors of one shape on cuda:{index}")
        rc = self._L.dllm_serve_plan(self._cp, self._tp, length.data_ptr(), q_len.data_ptr(), length.numel(), rows,
                                     prefix_len, causal, self._stream())
        if rc:
            _check(rc)
        self.rows, self.prefix_len = rows, prefix_len

    def _row_stride(self, name, x, heads, dtype):
        """Elements from row to row of x: [rows][heads * head_dim] or [rows][heads][head_dim], rows dense."""
        st, shape, hd = x.stride(), x.shape, self._hd
        if x.dtype == dtype and x.get_device() == self._index:
            n = heads * hd
            if (len(shape) == 2 and shape[1] == n and st[1] == 1) or (
                    len(shape) == 3 and shape[1] == heads and shape[2] == hd and st[2] == 1 and (st[1] == hd or heads == 1)):
                return st[0] if shape[0] > 1 or st[0] >= n else n
        raise ValueError(f"{name} must be [rows][{heads * hd}] or [rows][{heads}][{hd}] of {dtype} with dense rows on "
                         f"cuda:{self._index}, not {x.dtype} {tuple(shape)} of strides {st} on {x.device}")

    def _cache(self, name, x):
        if x.dtype != self._dt or x.get_device() != self._index or x.shape != self._cache_shape or (
                x.stride() != self._cache_strides and not (x.shape[0] == 1 and x.stride()[1:] == self._cache_strides[1:])):
            raise ValueError(f"{name} must be {self._cache_shape} of {self._dt}, strides {self._cache_strides}, on "
                             f"cuda:{self._index}, not {tuple(x.shape)} of {x.dtype}, strides {x.stride()}, on {x.device}")
        return x.data_ptr()

    def _vector(self, name, x, n):
        if x is None:
            return None
        if x.dtype != self._f32 or x.shape != (n,) or x.get_device() != self._index or not x.is_contiguous():
            raise ValueError(f"{name} must be {n} contiguous fp32 values on cuda:{self._index}")
        return x.data_ptr()

    def dllm_serve_qk_norm_rope(self, q, k, v, theta, kc, vc, q_gain=None, k_gain=None, eps=1e-5, out=None):
        """q [rows][n_heads * head_dim], k, v [rows][n_kv_heads * head_dim] (views of one projection's output, of
        the config's dtype or fp32) -> q normalised and rotated [rows][n_heads][head_dim]; k and v go to their slots."""
        rows, dtype, H, Hkv = q.shape[0], q.dtype, self._H, self._Hkv
        ldq, ldk, ldv = (self._row_stride("q", q, H, dtype), self._row_stride("k", k, Hkv, dtype),
                         self._row_stride("v", v, Hkv, dtype))
        if k.shape[0] != rows or v.shape[0] != rows:
            raise ValueError("q, k and v must have the same rows")
        if 0 < self.rows < rows:
            raise ValueError(f"q has {rows} rows, the plan {self.rows}: slots past them are an earlier plan's")
        if out is None:
            out, ld_out = self._empty((rows, H, self._hd), dtype=self._dt, device=self.device), H * self._hd
        else:
            ld_out = self._row_stride("out", out, H, self._dt)
            if out.shape[0] != rows:
                raise ValueError("out must have q's rows")
        rc = self._L.dllm_serve_qk_norm_rope(
            self._cp, self._tp, q.data_ptr(), k.data_ptr(), v.data_ptr(), self._kinds.get(dtype, -1), ldq, ldk, ldv,
            self._vector("q_gain", q_gain, self._hd), self._vector("k_gain", k_gain, self._hd), eps,
            self._vector("theta", theta, self._hd // 2), out.data_ptr(), ld_out, self._cache("kc", kc),
            self._cache("vc", vc), rows, self._stream())
        if rc:
            _check(rc)
        return out

    def dllm_serve_attention(self, q, kc, vc, prefix_pages=None, scale=None, lse=False, out=None):
        """q [rows][n_heads][head_dim] of the plan's rows -> [rows][n_heads * head_dim] (with lse: and the
        logarithms of the softmax sums, fp32 [rows][n_heads])."""
        rows, n_prefix, pages = q.shape[0], 0, None
        ldq = self._row_stride("q", q, self._H, self._dt)
        if rows != self.rows:
            raise ValueError(f"q has {rows} rows, the plan {self.rows}")
        if prefix_pages is not None:
            if (prefix_pages.dtype != self._i32 or prefix_pages.get_device() != self._index
                    or not prefix_pages.is_contiguous()):
                raise ValueError(f"prefix_pages must be a contiguous int32 tensor on cuda:{self._index}")
            n_prefix, pages = prefix_pages.numel(), prefix_pages.data_ptr()
        if n_prefix * self.cfg.page < self.prefix_len:
            raise ValueError(f"{n_prefix} prefix pages of {self.cfg.page} for a prefix of {self.prefix_len}")
        if out is None:
            out = self._empty((rows, self._H * self._hd), dtype=self._dt, device=self.device)
        elif (out.numel() != rows * self._H * self._hd or not out.is_contiguous() or out.dtype != self._dt
              or out.get_device() != self._index):
            raise ValueError("out must be contiguous, of q's rows, type and device")
        ls = self._empty((rows, self._H), dtype=self._f32, device=self.device) if lse else None
        rc = self._L.dllm_serve_attention(self._cp, self._tp, q.data_ptr(), ldq, self._cache("kc", kc), self._cache("vc", vc),
                                          pages, n_prefix, self._scale if scale is None else scale, out.data_ptr(),
                                          None if ls is None else ls.data_ptr(), rows, self._stream())
        if rc:
            _check(rc)
        return (out, ls) if lse else out

    def dllm_serve_check(self):
        """Waits for the stream; raises DllmError for what the kernels found wrong since the last check."""
        bits = _I()
        _check(self._L.dllm_serve_check(self._tp, C.byref(bits), self._stream()))


def dllm_serve_logits(logits, mask_id=-1, req=None, hist=None, hist_len=None, rep=None, freq=None, pres=None,
                      bias_ids=None, bias=None, bias_len=None, grammar=None, grammar_row=None, cur=None, out=None,
                      ws=None):
    """Penalties, biases and grammar masks on logits [rows][vocab] (fp32, bf16 or f16), and the decision: (x0,
    conf, tokconf), tokconf None without cur.  out: where the processed logits go (logits itself: in place)."""
    import torch

    shape, st = logits.shape, logits.stride()
    if len(shape) != 2 or not logits.is_cuda or (shape[1] > 1 and st[1] != 1):
        raise ValueError("logits must be a CUDA tensor [rows][vocab] with dense rows")
    rows, vocab = shape
    i32, f32, dev, index = torch.int32, torch.float32, logits.device, logits.get_device()
    stream = _stream_on(index)
    n_req = hist.shape[0] if hist is not None else bias_ids.shape[0] if bias_ids is not None else 0

    def at(name, x, dtype, want):
        if x is None:
            return None
        if x.dtype != dtype or x.shape != want or x.get_device() != index or not x.is_contiguous():
            raise ValueError(f"{name} must be a contiguous tensor of {dtype} {tuple(want)} on {dev}, not {x.dtype} "
                             f"{tuple(x.shape)} on {x.device}")
        return x.data_ptr()

    hist_ld = bias_ld = n_grammar = ld_out = 0
    if hist is not None:
        hist_ld = hist.shape[-1]
    elif rep is not None or freq is not None or pres is not None or hist_len is not None:
        raise ValueError("penalties come with hist")
    if bias_ids is not None:
        bias_ld = bias_ids.shape[-1]
        if bias is None:
            raise ValueError("bias_ids come with bias")
    if grammar is not None:
        n_grammar = grammar.shape[0]
    if req is None and n_req and n_req != rows:
        raise ValueError("without req there is a list for each row")
    if out is not None:
        so = out.stride()
        if out.shape != shape or out.dtype != logits.dtype or out.get_device() != index or (vocab > 1 and so[1] != 1):
            raise ValueError("out must be like logits")
        ld_out = so[0] if rows > 1 else max(so[0], vocab)
    if ws is None:
        ws = torch.empty(_logits_bytes(rows, vocab), dtype=torch.uint8, device=dev)
    elif ws.get_device() != index or not ws.is_contiguous():
        raise ValueError(f"ws must be contiguous on {dev}")
    x0 = torch.empty(rows, dtype=i32, device=dev)
    conf, tokconf = torch.empty((2, rows), dtype=f32, device=dev).unbind(0)
    per_row, per_req = (rows,), (n_req,)
    a = dllm_serve_logits_args(
        logits.data_ptr(), None if out is None else out.data_ptr(), st[0] if rows > 1 else max(st[0], vocab), ld_out,
        _names().get(logits.dtype, -1), rows, vocab, mask_id, n_req, at("req", req, i32, per_row),
        at("hist", hist, i32, (n_req, hist_ld)), at("hist_len", hist_len, i32, per_req), hist_ld, at("rep", rep, f32, per_req),
        at("freq", freq, f32, per_req), at("pres", pres, f32, per_req), at("bias_ids", bias_ids, i32, (n_req, bias_ld)),
        at("bias", bias, f32, (n_req, bias_ld)), at("bias_len", bias_len, i32, per_req), bias_ld,
        at("grammar", grammar, i32, (n_grammar, (vocab + 31) // 32)), at("grammar_row", grammar_row, i32, per_row), n_grammar,
        at("cur", cur, i32, per_row), x0.data_ptr(), conf.data_ptr(), None if cur is None else tokconf.data_ptr(),
        ws.data_ptr(), ws.numel() * ws.element_size())
    rc = serve_lib().dllm_serve_logits(C.byref(a), stream)
    if rc:
        _check(rc)
    return x0, conf, None if cur is None else tokconf
