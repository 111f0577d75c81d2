"""Python binding of ``include/dllm_serve.h``: the operators that serve a batch of unequal requests over a
paged K/V cache, under a prefix that all of them share.

Argument marshalling only.  Calls run on torch's current stream and do not wait; what a kernel found wrong
(lengths, a pool that ran out) is raised by ``Serve.dllm_serve_check``.
"""
from __future__ import annotations

import ctypes as C
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


def _names():
    import torch

    return {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


def _stream(device):
    import torch

    return torch.cuda.current_stream(device).cuda_stream


def _need(name, x, dtype, shape=None, cols=None):
    """A CUDA tensor of a type and shape whose rows are dense."""
    if not x.is_cuda or x.dtype != dtype:
        raise ValueError(f"{name} must be a CUDA tensor of {dtype}, not {x.dtype} on {x.device}")
    if shape is not None and tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name} must be {tuple(shape)}, not {tuple(x.shape)}")
    if cols is not None and (x.dim() < 2 or x[0].numel() != cols):
        raise ValueError(f"{name} must have rows of {cols} values, not shape {tuple(x.shape)}")
    return x


def _ptr(x):
    return None if x is None else x.data_ptr()


class Serve:
    """The buffers of one serving batch (a torch tensor), and the calls on them with the ABI's names.  The
    attributes table, held, ring, ring_pos, row_start, n_keys, slot, pos, req and status are int32 views of
    them.  One stream at a time."""

    def __init__(self, cfg: ServeConfig, device=None):
        import torch

        self.cfg = cfg
        self._c = cfg.c()
        self._cp = C.byref(self._c)
        L = serve_lib()
        n = dllm_serve_bytes(cfg)
        self.buffer = torch.empty(n, dtype=torch.uint8, device=device or "cuda")
        self.device = self.buffer.device
        self._t = dllm_serve_tables()
        self._tp = C.byref(self._t)
        self._dt = {"bf16": torch.bfloat16, "f16": torch.float16}[cfg.dtype]
        self._kinds = _names()
        with torch.cuda.device(self.device):
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

    def dllm_serve_reset(self):
        """Nothing held, every page free."""
        _check(serve_lib().dllm_serve_reset(self._cp, self._tp, _stream(self.device)))
        self.rows = self.prefix_len = 0

    def dllm_serve_plan(self, length, q_len, rows, prefix_len=0, causal=False):
        """length, q_len: int32 CUDA tensors [batch], own positions cached and new tokens; rows: rows of the step's
        packed arrays (at least the sum of q_len, else the last are left out)."""
        import torch

        _need("length", length, torch.int32)
        _need("q_len", q_len, torch.int32, length.shape)
        if not (length.is_contiguous() and q_len.is_contiguous()):
            raise ValueError("length and q_len must be contiguous")
        _check(serve_lib().dllm_serve_plan(self._cp, self._tp, length.data_ptr(), q_len.data_ptr(), length.numel(), rows,
                                           prefix_len, causal, _stream(self.device)))
        self.rows, self.prefix_len = rows, prefix_len

    def _rows(self, name, x, heads, dtype=None):
        """x as rows of heads * head_dim values: (pointer, stride of a row)."""
        n = heads * self.cfg.head_dim
        if not x.is_cuda or (dtype is not None and x.dtype != dtype):
            raise ValueError(f"{name} must be a CUDA tensor of {dtype}, not {x.dtype} on {x.device}")
        st = x.stride()
        if x.dim() == 2 and x.shape[1] == n and (st[1] == 1 or n == 1):
            return x.data_ptr(), max(st[0], n) if x.shape[0] < 2 else st[0]
        if x.dim() == 3 and x.shape[1:] == (heads, self.cfg.head_dim) and st[2] == 1 and (
                st[1] == self.cfg.head_dim or heads == 1):
            return x.data_ptr(), max(st[0], n) if x.shape[0] < 2 else st[0]
        raise ValueError(f"{name} must be [rows][{n}] or [rows][{heads}][{self.cfg.head_dim}] with dense rows, "
                         f"not shape {tuple(x.shape)} of strides {st}")

    def _cache(self, name, x):
        c = self.cfg
        _need(name, x, self._dt, (c.n_pages, c.n_kv_heads, c.page, c.head_dim))
        st, dense = x.stride(), c.n_kv_heads * c.page * c.head_dim
        if st[1:] != (c.page * c.head_dim, c.head_dim, 1) or (c.n_pages > 1 and st[0] != (c.page_stride or dense)):
            raise ValueError(f"{name}: strides {st} are not those of the config")
        return x.data_ptr()

    def dllm_serve_qk_norm_rope(self, q, k, v, theta, kc, vc, q_gain=None, k_gain=None, eps=1e-5, out=None):
        """q [rows][n_heads * head_dim], k, v [rows][n_kv_heads * head_dim] (views of one projection's output, of
        the config's dtype or fp32) -> q normalised and rotated [rows][n_heads][head_dim]; k and v go to their slots."""
        import torch

        c = self.cfg
        rows = q.shape[0]
        if k.shape[0] != rows or v.shape[0] != rows or k.dtype != q.dtype or v.dtype != q.dtype:
            raise ValueError("q, k and v must have the same rows and type")
        qp, ldq = self._rows("q", q, c.n_heads)
        kp, ldk = self._rows("k", k, c.n_kv_heads)
        vp, ldv = self._rows("v", v, c.n_kv_heads)
        for name, x, n in (("theta", theta, c.head_dim // 2), ("q_gain", q_gain, c.head_dim), ("k_gain", k_gain, c.head_dim)):
            if x is not None and (x.dtype != torch.float32 or x.shape != (n,) or not x.is_cuda or not x.is_contiguous()):
                raise ValueError(f"{name} must be {n} contiguous fp32 values on the GPU")
        if out is None:
            out = torch.empty((rows, c.n_heads, c.head_dim), dtype=self._dt, device=self.device)
        op, ld_out = self._rows("out", out, c.n_heads, self._dt)
        if out.shape[0] != rows:
            raise ValueError("out must have q's rows")
        _check(serve_lib().dllm_serve_qk_norm_rope(self._cp, self._tp, qp, kp, vp, self._kinds.get(q.dtype, -1), ldq, ldk, ldv,
                                                   _ptr(q_gain), _ptr(k_gain), eps, theta.data_ptr(), op, ld_out,
                                                   self._cache("kc", kc), self._cache("vc", vc), rows,
                                                   _stream(self.device)))
        return out

    def dllm_serve_attention(self, q, kc, vc, prefix_pages=None, scale=None, lse=False, out=None):
        """q [rows][n_heads][head_dim] of the plan's rows -> [rows][n_heads * head_dim] (with lse: and the
        logarithms of the softmax sums, fp32 [rows][n_heads])."""
        import torch

        c = self.cfg
        rows, n_prefix = q.shape[0], 0
        qp, ldq = self._rows("q", q, c.n_heads, self._dt)
        if rows != self.rows:
            raise ValueError(f"q has {rows} rows, the plan {self.rows}")
        if prefix_pages is not None:
            n_prefix = _need("prefix_pages", prefix_pages, torch.int32).numel()
            if not prefix_pages.is_contiguous():
                raise ValueError("prefix_pages must be contiguous")
        if n_prefix * c.page < self.prefix_len:
            raise ValueError(f"{n_prefix} prefix pages of {c.page} for a prefix of {self.prefix_len}")
        if out is None:
            out = torch.empty((rows, c.n_heads * c.head_dim), dtype=self._dt, device=self.device)
        elif out.numel() != rows * c.n_heads * c.head_dim or not out.is_contiguous() or out.dtype != self._dt:
            raise ValueError("out must be contiguous, of q's rows and type")
        ls = torch.empty((rows, c.n_heads), dtype=torch.float32, device=self.device) if lse else None
        _check(serve_lib().dllm_serve_attention(self._cp, self._tp, qp, ldq, self._cache("kc", kc), self._cache("vc", vc),
                                                _ptr(prefix_pages), n_prefix,
                                                c.head_dim ** -0.5 if scale is None else scale, out.data_ptr(), _ptr(ls),
                                                rows, _stream(self.device)))
        return (out, ls) if lse else out

    def dllm_serve_check(self):
        """Waits for the stream; raises DllmError for what the kernels found wrong since the last check."""
        bits = _I()
        _check(serve_lib().dllm_serve_check(self._tp, C.byref(bits), _stream(self.device)))


def dllm_serve_logits(logits, mask_id=-1, req=None, hist=None, hist_len=None, rep=None, freq=None, pres=None,
                      bias_ids=None, bias=None, bias_len=None, grammar=None, grammar_row=None, cur=None, out=None,
                      ws=None):
    """Penalties, biases and grammar masks on logits [rows][vocab] (fp32, bf16 or f16), and the decision: (x0,
    conf, tokconf), tokconf None without cur.  out: where the processed logits go (logits itself: in place)."""
    import torch

    if logits.dim() != 2 or not logits.is_cuda or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be a CUDA tensor [rows][vocab] with dense rows")
    rows, vocab = logits.shape
    dev, kind = logits.device, _names().get(logits.dtype, -1)
    a = dllm_serve_logits_args()
    a.logits, a.ld, a.dtype, a.rows, a.vocab, a.mask_id = (logits.data_ptr(), max(logits.stride(0), vocab) if rows < 2
                                                            else logits.stride(0), kind, rows, vocab, mask_id)
    if out is not None:
        if out.shape != logits.shape or out.dtype != logits.dtype or (vocab > 1 and out.stride(1) != 1):
            raise ValueError("out must be like logits")
        a.out, a.ld_out = out.data_ptr(), max(out.stride(0), vocab) if rows < 2 else out.stride(0)
    i32, f32 = torch.int32, torch.float32
    lists = [x for x in (hist, bias_ids) if x is not None]
    n_req = lists[0].shape[0] if lists else 0
    a.n_req = n_req
    for name, x, dtype, shape in (
            ("req", req, i32, (rows,)), ("hist", hist, i32, None), ("hist_len", hist_len, i32, (n_req,)),
            ("rep", rep, f32, (n_req,)), ("freq", freq, f32, (n_req,)), ("pres", pres, f32, (n_req,)),
            ("bias_ids", bias_ids, i32, None), ("bias", bias, f32, None if bias_ids is None else bias_ids.shape),
            ("bias_len", bias_len, i32, (n_req,)), ("grammar", grammar, i32, None), ("grammar_row", grammar_row, i32, (rows,)),
            ("cur", cur, i32, (rows,))):
        if x is None:
            continue
        if x.dtype != dtype or not x.is_cuda or not x.is_contiguous() or (shape is not None and x.shape != shape):
            raise ValueError(f"{name} must be a contiguous CUDA tensor of {dtype}" + (f" {tuple(shape)}" if shape else ""))
        setattr(a, name, x.data_ptr())
    for name, x in (("hist", hist), ("bias_ids", bias_ids)):
        if x is not None and (x.dim() != 2 or x.shape[0] != n_req):
            raise ValueError(f"{name} must be [requests][length]")
    if req is None and n_req and n_req != rows:
        raise ValueError("without req there is a list for each row")
    if hist is None and (rep is not None or freq is not None or pres is not None or hist_len is not None):
        raise ValueError("penalties come with hist")
    if hist is not None:
        a.hist_ld = hist.shape[1]
    if bias_ids is not None:
        if bias is None:
            raise ValueError("bias_ids come with bias")
        a.bias_ld = bias_ids.shape[1]
    if grammar is not None:
        if grammar.dim() != 2 or grammar.shape[1] != (vocab + 31) // 32:
            raise ValueError(f"grammar must be [masks][{(vocab + 31) // 32}]")
        a.n_grammar = grammar.shape[0]
    x0 = torch.empty(rows, dtype=i32, device=dev)
    conf = torch.empty((2 if cur is not None else 1, rows), dtype=f32, device=dev)
    a.x0, a.conf = x0.data_ptr(), conf.data_ptr()
    if cur is not None:
        a.tokconf = conf.data_ptr() + 4 * rows
    if ws is None:
        n = _SZ()
        _check(serve_lib().dllm_serve_logits_bytes(rows, vocab, C.byref(n)))
        ws = torch.empty(n.value, dtype=torch.uint8, device=dev)
    a.ws, a.ws_bytes = ws.data_ptr(), ws.numel()
    _check(serve_lib().dllm_serve_logits(C.byref(a), _stream(dev)))
    return x0, conf[0], conf[1] if cur is not None else None
