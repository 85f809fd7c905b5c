"""GB300-native SDSAT block decode step: Python binding of libsdsat.

Argument marshalling only: every step of the decode path runs in the CUDA
kernels of libsdsat.so (built in-tree from csrc/ for sm_103a).  PyTorch is
used for device memory and streams.  There is no CPU fallback: if the
library cannot be loaded, importing the binding raises.

    ctx = Context(shape, weights)            # weights: synth-style dict of CUDA bf16 tensors
    kv = ctx.kv(batch, max_len)
    ctx.prefill(kv, seq, prompt_ids)
    ctx.block_forward(kv, tokens, logits, b, q)
    ctx.accept_greedy(kv, logits, tokens, b, q, n_verify, acc, out)
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

from . import build as _build

MAX_Q = 16
MAX_ROWS = 64
MAX_ADAPTIVE = 16
TRACE_WORDS = 8        # words per device trace record

DEV_NAN_LOGITS = 0x1
DEV_TIMEOUT = 0x2
DEV_CAPACITY = 0x4
DEV_TOKEN = 0x8
DEV_POSITION = 0x10
DEV_TREE = 0x20
DEV_PAGE = 0x40

PAGE = 64              # slots of a page of a paged cache
ROPE_SCALING = {None: 0, "linear": 1, "parts": 2}
FP32, BF16 = 0, 1      # element types of the kernels that take more than one


class SdsatError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (what, _lib().sdsat_status_string(status).decode(), status))


class Config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("ffn_dim", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float),
                ("max_position", ctypes.c_int32), ("n_adaptive", ctypes.c_int32),
                ("adaptive_ids", ctypes.c_int32 * MAX_ADAPTIVE)]


class KernelStat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int64), ("total_ms", ctypes.c_double)]


class LayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")]


class RopeConfig(ctypes.Structure):
    _fields_ = [("dims", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("max_position", ctypes.c_int32),
                ("scaling", ctypes.c_int32), ("original", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("theta", ctypes.c_double), ("factor", ctypes.c_double), ("low", ctypes.c_double),
                ("high", ctypes.c_double), ("magnitude", ctypes.c_double)]


class Weights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("final_norm", ctypes.c_void_p), ("lm_head", ctypes.c_void_p),
                ("layers", ctypes.POINTER(LayerWeights))]


_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        if _build.is_stale():
            _build.build_library()
        lib = ctypes.CDLL(_build.LIB)
        P, I, F, U64, I64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_uint64, ctypes.c_int64
        sig = {
            "sdsat_create": [ctypes.POINTER(Config), ctypes.POINTER(Weights), P, ctypes.POINTER(P)],
            "sdsat_set_stream": [P, P],
            "sdsat_kv_create": [P, I, I, ctypes.POINTER(P)],
            "sdsat_kv_info": [P, ctypes.POINTER(P), ctypes.POINTER(P), ctypes.POINTER(P),
                              ctypes.POINTER(I), ctypes.POINTER(I)],
            "sdsat_block_forward": [P, P, P, P, I, I, P],
            "sdsat_kv_write": [P, P, I, I, I, I, P, P],
            "sdsat_kv_read": [P, P, I, I, I, I, P, P],
            "sdsat_accept_greedy": [P, P, P, P, I, I, I, P, P, I],
            "sdsat_accept_nucleus": [P, P, P, P, I, I, I, F, F, U64, I, P, P, I],
            "sdsat_kv_commit": [P, P, P, I],
            "sdsat_kv_lengths": [P, P, P, I],
            "sdsat_kv_emitted": [P, P, P, I, I],
            "sdsat_profile_begin": [P, I],
            "sdsat_trace_begin": [P, I],
            "sdsat_trace_end": [P, P, I, ctypes.POINTER(I)],
            "sdsat_profile_end": [P, ctypes.POINTER(KernelStat), I, ctypes.POINTER(I)],
            "sdsat_build_block": [P, P, I, P, P, P, I, I, I, P],
            "sdsat_block_forward_tree": [P, P, P, P, I, I, P],
            "sdsat_accept_tree": [P, P, P, P, P, I, I, F, F, U64, I, P, P, P, I],
            "sdsat_build_tree_block": [P, P, I, P, I, P, P, I, I, I, I, P],
            "sdsat_build_pipelined_block": [P, P, P, P, P, P, P, I, I, I, P],
            "sdsat_accept_pipelined": [P, P, P, P, P, I, I, F, F, U64, I, P, P, I],
            "sdsat_prefill": [P, P, I, P, I],
            "sdsat_get_error": [P, ctypes.POINTER(ctypes.c_uint32)],
            "sdsat_op_gemm": [P, P, I, I, P, I, P],
            "sdsat_op_attention": [P, P, P, P, P, I, I, I, I, I, P],
            "sdsat_op_exp": [P, P, P, I],
            "sdsat_kv_create_paged": [P, I, I, I, ctypes.POINTER(P)],
            "sdsat_kv_pages": [P, ctypes.POINTER(P), ctypes.POINTER(P), ctypes.POINTER(I), ctypes.POINTER(I)],
            "sdsat_kv_fork": [P, P, P, I],
            "sdsat_kv_free": [P, P, I],
            "sdsat_kv_reserve": [P, P, I, I, I],
            "sdsat_kv_compact": [P, P, P],
            "sdsat_op_prefix_attention": [P, P, I64, P, P, I, P, I, P, P, P, I, I, I, I, I, P, I64, I],
            "sdsat_op_logprobs": [P, P, I64, I, I, I, P, F, I, P, P, P, P, P],
            "sdsat_rope_create": [P, ctypes.POINTER(RopeConfig), ctypes.POINTER(P)],
            "sdsat_op_rotary_append": [P, P, P, I64, P, I64, P, I64, I, I, P, P, I, P, P, P, F, I, I, I, P, I64, P, P, I, P, I, P],
            "sdsat_op_chunk_attention": [P, P, I64, I, P, P, I, P, I, P, P, I, I, I, I, P, I64, I],
            "sdsat_op_adjust_logits": [P, P, I64, I, I, I, I, P, I, P, P, P, P, P, P, P, P, P, I, P, I, P, I64],
            "sdsat_debug_workspace": [P, I, I, P],
            "sdsat_debug_wait_timeout": [P],
            "sdsat_attention_grid": [I, P, I, I, ctypes.POINTER(I), ctypes.POINTER(I)],
        }
        for name, args in sig.items():
            fn = getattr(lib, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        lib.sdsat_destroy.argtypes = [P]
        lib.sdsat_destroy.restype = None
        lib.sdsat_kv_destroy.argtypes = [P]
        lib.sdsat_kv_destroy.restype = None
        lib.sdsat_rope_destroy.argtypes = [P]
        lib.sdsat_rope_destroy.restype = None
        lib.sdsat_kernel_class_name.argtypes = [ctypes.c_int]
        lib.sdsat_kernel_class_name.restype = ctypes.c_char_p
        lib.sdsat_status_string.argtypes = [ctypes.c_int]
        lib.sdsat_status_string.restype = ctypes.c_char_p
        _LIB = lib
    return _LIB


def lib():
    """The loaded libsdsat (raises if it cannot be built or loaded)."""
    return _lib()


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


_kinds = _f32 = _bf16 = _i32 = None   # tensor types, once torch is there (the first call that asks for them)
_calls = None                         # the calls whose arguments are checked and converted in C (csrc/binding.c)


def _rows(t):
    """(address, values from one row to the next, element type, rows, columns) of a CUDA matrix whose rows are
    contiguous."""
    if _kinds is None:
        _tensor_types()
    kind = _kinds.get(t.dtype)
    if kind is None or not t.is_cuda or t.dim() != 2:
        raise ValueError("expected a float32 or bfloat16 CUDA matrix")
    (rows, columns), (ld, step) = t.shape, t.stride()
    if step != 1 and columns > 1:
        raise ValueError("expected contiguous rows")
    return t.data_ptr(), ld if rows > 1 else columns, kind, rows, columns


def _tensor_types():
    global _kinds, _f32, _bf16, _i32
    import torch
    _kinds, _f32, _bf16, _i32 = {torch.float32: FP32, torch.bfloat16: BF16}, torch.float32, torch.bfloat16, torch.int32


def _types():
    """The tensor types, and the calls that are in C (which alone need a compiler and the interpreter's headers)."""
    global _calls
    _tensor_types()
    lib = _lib()
    if _build.native_is_stale():
        _build.build_native()
    from . import _native
    _native.library(*[ctypes.cast(getattr(lib, "sdsat_" + n), ctypes.c_void_p).value
                      for n in ("set_stream", "op_rotary_append", "op_chunk_attention", "op_adjust_logits")])
    _native.types(_f32, _bf16, _i32, _stream)
    _calls = _native


def _array(t, dtype, n: int):
    """The address of a contiguous CUDA tensor of n values or more of a type (None and addresses as they are)."""
    if t is None:
        return None
    try:
        if t.dtype is dtype and t.numel() >= n and t.is_cuda and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        if isinstance(t, int):
            return t
        raise
    raise ValueError("expected %d values of %s in a contiguous CUDA tensor, got %d of %s on %s"
                     % (n, dtype, t.numel(), t.dtype, t.device))


def _check(status: int, what: str):
    if status != 0:
        raise SdsatError(status, what)


def attention_grid(pairs: int, max_clusters, cs_cap: int = 16, num_sms: int = 152):
    """(cluster size, clusters) the attention launches for `pairs` (sequence, head) pairs,
    given max_clusters[c] = the most clusters of c CTAs resident at once (c = 1..16)."""
    arr = (ctypes.c_int32 * 17)(0, *[int(v) for v in list(max_clusters)[1:17]])
    cs, nc = ctypes.c_int(0), ctypes.c_int(0)
    _check(_lib().sdsat_attention_grid(pairs, ctypes.cast(arr, ctypes.c_void_p), cs_cap, num_sms,
                                       ctypes.byref(cs), ctypes.byref(nc)), "sdsat_attention_grid")
    return cs.value, nc.value


_current_stream = None


def _stream():
    """The calling thread's current CUDA stream as an integer.  Every compute call asks for it:
    torch.cuda.current_stream() builds a Stream object (2.8 us on the GB300's host, a third of a
    small call's issue time); the raw query is 0.2 us."""
    global _current_stream
    if _current_stream is None:
        import torch
        torch.cuda.current_stream()   # CUDA is initialised before the raw query
        raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch._C._cuda_getDevice
        _current_stream = (lambda: raw(device())) if raw else (lambda: torch.cuda.current_stream().cuda_stream)
    return _current_stream()


def make_config(shape, max_position: int = 8192, adaptive_ids=None) -> Config:
    c = Config()
    c.n_layers, c.d_model, c.n_heads = shape.n_layers, shape.d_model, shape.n_heads
    c.n_kv_heads, c.head_dim, c.ffn_dim, c.vocab = shape.n_heads, shape.head_dim, shape.ffn_dim, shape.vocab
    c.rms_eps, c.rope_theta, c.max_position = shape.rms_eps, shape.rope_theta, max_position
    ids = list(adaptive_ids) if adaptive_ids is not None else [shape.adaptive_id]
    c.n_adaptive = len(ids)
    for i, a in enumerate(ids):
        c.adaptive_ids[i] = a
    return c


class KV:
    """A library-owned KV cache of `batch` sequences and `max_len` slots."""

    def __init__(self, ctx: "Context", batch: int, max_len: int):
        self.ctx = ctx
        h = ctypes.c_void_p()
        _check(_lib().sdsat_kv_create(ctx.handle, batch, max_len, ctypes.byref(h)), "sdsat_kv_create")
        self.handle = h
        self.batch, self.max_len = batch, max_len

    def info(self):
        k, v, ln = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p()
        b, m = ctypes.c_int(), ctypes.c_int()
        _check(_lib().sdsat_kv_info(self.handle, ctypes.byref(k), ctypes.byref(v), ctypes.byref(ln),
                                    ctypes.byref(b), ctypes.byref(m)), "sdsat_kv_info")
        return k.value, v.value, ln.value, b.value, m.value

    def close(self):
        if getattr(self, "handle", None):
            _lib().sdsat_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _Memory:
    """Device memory of a cache as a CUDA array; the cache lives as long as its views."""

    def __init__(self, owner, address: int, shape, typestr: str):
        self.owner = owner
        self.__cuda_array_interface__ = dict(data=(address, False), shape=tuple(shape), typestr=typestr, version=3)


class PagedKV(KV):
    """A library-owned cache of `n_pages` pages of PAGE slots, which sequences may share.

    Its tensors are the cache's own memory.  Block forwards go by the shared pages that kv_fork, kv_free and kv_reserve
    count: after writing to `table` (and `refs`) call one of them."""

    def __init__(self, ctx: "Context", batch: int, max_len: int, n_pages: int):
        import torch
        self.ctx = ctx
        self.device = torch.device("cuda", torch.cuda.current_device())   # where the library allocates it
        h = ctypes.c_void_p()
        _check(_lib().sdsat_kv_create_paged(ctx.handle, batch, max_len, n_pages, ctypes.byref(h)),
               "sdsat_kv_create_paged")
        self.handle = h
        self.batch, self.max_len, self.n_pages = batch, max_len, n_pages
        self.table_ld = -(-max_len // PAGE)

    def pages(self):
        t, r, n, ld = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_int(), ctypes.c_int()
        _check(_lib().sdsat_kv_pages(self.handle, ctypes.byref(t), ctypes.byref(r), ctypes.byref(n), ctypes.byref(ld)),
               "sdsat_kv_pages")
        return t.value, r.value, n.value, ld.value

    # the cache's own memory as tensors (what it holds is read on the stream of the calls before)
    def _view(self, address, shape, typestr="<i4"):
        import torch
        return torch.as_tensor(_Memory(self, address, shape, typestr), device=self.device)

    @property
    def table(self):
        """int32 [batch][table_ld]: the page of slots PAGE*j .. of each sequence, -1 where it has none."""
        return self._view(self.pages()[0], (self.batch, self.table_ld))

    @property
    def refs(self):
        """int32 [n_pages]: the sequences that hold each page."""
        return self._view(self.pages()[1], (self.n_pages,))

    @property
    def lens(self):
        """int32 [batch]: the committed lengths."""
        return self._view(self.info()[2], (self.batch,))

    def _pool(self, which):
        import torch
        s = self.ctx.shape
        shape = (s.n_layers, self.n_pages, s.n_heads, PAGE, s.head_dim)
        return self._view(self.info()[which], shape, "<i2").view(torch.bfloat16)

    @property
    def k(self):
        """bf16 [n_layers][n_pages][n_heads][PAGE][head_dim]."""
        return self._pool(0)

    @property
    def v(self):
        return self._pool(1)


class Rope:
    """The cosines and sines of a rotation: max_position rows of dims / 2 pairs, fp32."""

    def __init__(self, ctx: "Context", cfg: RopeConfig):
        self.ctx, self.dims, self.max_position = ctx, cfg.dims, cfg.max_position
        h = ctypes.c_void_p()
        _check(_lib().sdsat_rope_create(ctx.handle, ctypes.byref(cfg), ctypes.byref(h)), "sdsat_rope_create")
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            _lib().sdsat_rope_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Context:
    """Borrowed weights + TMA descriptors + workspaces for one model shape."""

    def __init__(self, shape, weights: Optional[dict] = None, max_position: int = 8192, adaptive_ids=None,
                 stream=None):
        import torch
        self.shape = shape
        self.cfg = make_config(shape, max_position, adaptive_ids)
        self._keep = weights
        w = None
        if weights is not None:
            L = shape.n_layers
            self._layers = (LayerWeights * L)()
            for l in range(L):
                for n in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down"):
                    setattr(self._layers[l], n, _ptr(weights["layers"][l][n]))
            w = Weights(_ptr(weights["embed"]), _ptr(weights["final_norm"]), _ptr(weights["lm_head"]),
                        ctypes.cast(self._layers, ctypes.POINTER(LayerWeights)))
            self._w = w
        h = ctypes.c_void_p()
        st = stream if stream is not None else torch.cuda.current_stream().cuda_stream
        _check(_lib().sdsat_create(ctypes.byref(self.cfg), ctypes.byref(w) if w is not None else None, st,
                                   ctypes.byref(h)), "sdsat_create")
        self.handle = h

    def _bind_stream(self):
        _lib().sdsat_set_stream(self.handle, _stream())

    def kv(self, batch: int, max_len: int) -> KV:
        return KV(self, batch, max_len)

    # ---- paged caches: many samples of one prompt ----
    def kv_paged(self, batch: int, max_len: int, n_pages: int) -> PagedKV:
        return PagedKV(self, batch, max_len, n_pages)

    def kv_fork(self, kv: PagedKV, src, b: int = None):
        """Sequence s takes the pages and the length of sequence src[s] (int32 CUDA tensor [b]; -1: none)."""
        self._bind_stream()
        if _kinds is None:
            _tensor_types()
        b = src.numel() if b is None else b
        _check(_lib().sdsat_kv_fork(self.handle, kv.handle, _array(src, _i32, min(b, kv.batch)), b), "sdsat_kv_fork")

    def kv_free(self, kv: PagedKV, seq: int):
        self._bind_stream()
        _check(_lib().sdsat_kv_free(self.handle, kv.handle, seq), "sdsat_kv_free")

    def kv_reserve(self, kv: PagedKV, b: int, n: int, seq: int = 0):
        """Pages of their own for the next n slots of sequences seq .. seq+b-1."""
        self._bind_stream()
        _check(_lib().sdsat_kv_reserve(self.handle, kv.handle, seq, b, n), "sdsat_kv_reserve")

    def kv_compact(self, kv: PagedKV, used=None):
        """Pages in use move to the front of the pool; used: int32 CUDA tensor [1] for their number."""
        self._bind_stream()
        if _kinds is None:
            _tensor_types()
        _check(_lib().sdsat_kv_compact(self.handle, kv.handle, _array(used, _i32, 1)), "sdsat_kv_compact")

    def kv_write(self, kv: KV, layer: int, seq: int, slot0: int, k, v):
        """k, v: bf16 CUDA tensors [n_heads, n, head_dim] written to slots slot0 .. slot0+n-1."""
        self._bind_stream()
        _check(_lib().sdsat_kv_write(self.handle, kv.handle, layer, seq, slot0, k.shape[1], _ptr(k), _ptr(v)),
               "sdsat_kv_write")

    def kv_read(self, kv: KV, layer: int, seq: int, slot0: int, n: int):
        import torch
        self._bind_stream()
        H, hd = self.shape.n_heads, self.shape.head_dim
        k = torch.empty(H, n, hd, dtype=torch.bfloat16, device="cuda")
        v = torch.empty_like(k)
        _check(_lib().sdsat_kv_read(self.handle, kv.handle, layer, seq, slot0, n, _ptr(k), _ptr(v)), "sdsat_kv_read")
        return k, v

    # ---- the block decode step ----
    def block_forward(self, kv: KV, tokens, logits, b: int, q: int, positions=None):
        self._bind_stream()
        _check(_lib().sdsat_block_forward(self.handle, kv.handle, _ptr(tokens), _ptr(positions), b, q,
                                          _ptr(logits)), "sdsat_block_forward")

    def accept_greedy(self, kv: KV, logits, drafts, b: int, q: int, n_verify: int, accepted_len, out_tokens,
                      commit: bool = True):
        self._bind_stream()
        _check(_lib().sdsat_accept_greedy(self.handle, kv.handle, _ptr(logits), _ptr(drafts), b, q, n_verify,
                                          _ptr(accepted_len), _ptr(out_tokens), int(commit)), "sdsat_accept_greedy")

    def accept_nucleus(self, kv: KV, logits, drafts, b: int, q: int, n_verify: int, top_p: float,
                       temperature: float, seed: int, accepted_len, out_tokens, top_k: int = 0,
                       commit: bool = True):
        self._bind_stream()
        _check(_lib().sdsat_accept_nucleus(self.handle, kv.handle, _ptr(logits), _ptr(drafts), b, q, n_verify,
                                           top_p, temperature, seed, top_k, _ptr(accepted_len), _ptr(out_tokens),
                                           int(commit)), "sdsat_accept_nucleus")

    def kv_commit(self, kv: KV, new_len, b: int):
        self._bind_stream()
        _check(_lib().sdsat_kv_commit(self.handle, kv.handle, _ptr(new_len), b), "sdsat_kv_commit")

    def kv_lengths(self, kv: KV, b: int = None):
        """The committed lengths as an int32 CUDA tensor [b] (queued on the current stream)."""
        import torch
        b = kv.batch if b is None else b
        out = torch.empty(b, dtype=torch.int32, device="cuda")
        self._bind_stream()
        _check(_lib().sdsat_kv_lengths(self.handle, kv.handle, _ptr(out), b), "sdsat_kv_lengths")
        return out

    def kv_emitted(self, kv: KV, reset: bool = False):
        """Tokens emitted per sequence so far (int64 CUDA tensor [batch])."""
        import torch
        out = torch.empty(kv.batch, dtype=torch.int64, device="cuda")
        self._bind_stream()
        _check(_lib().sdsat_kv_emitted(self.handle, kv.handle, _ptr(out), kv.batch, int(reset)), "sdsat_kv_emitted")
        return out

    def profile_begin(self, max_launches: int):
        _check(_lib().sdsat_profile_begin(self.handle, max_launches), "sdsat_profile_begin")

    def profile_end(self) -> dict:
        """{kernel class: (launches, total_ms)} of the launches since profile_begin."""
        self._bind_stream()
        buf = (KernelStat * 32)()
        n = ctypes.c_int(0)
        _check(_lib().sdsat_profile_end(self.handle, buf, 32, ctypes.byref(n)), "sdsat_profile_end")
        return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms)) for i in range(n.value)}

    def trace_begin(self, max_records: int):
        _check(_lib().sdsat_trace_begin(self.handle, max_records), "sdsat_trace_begin")

    def trace_end(self, max_records: int):
        """Device timeline records: list of dicts with the kernel class name, launch seq, block,
        smid, flags and the %globaltimer stamps entry / wait / marks (3) / exit."""
        import numpy as np
        buf = np.zeros((max_records, TRACE_WORDS), dtype=np.uint64)
        n = ctypes.c_int(0)
        self._bind_stream()
        _check(_lib().sdsat_trace_end(self.handle, buf.ctypes.data, max_records, ctypes.byref(n)), "sdsat_trace_end")
        out = []
        for r in buf[:n.value]:
            tag, blk = int(r[0]) >> 32, int(r[0]) & 0xFFFFFFFF
            out.append(dict(kernel=_lib().sdsat_kernel_class_name(tag >> 24).decode(), seq=tag & 0xFFFFFF,
                            block=blk, smid=int(r[1]) & 0xFFFFFFFF, flags=int(r[1]) >> 32, entry=int(r[2]),
                            wait=int(r[3]), marks=(int(r[4]), int(r[5]), int(r[6])), exit=int(r[7])))
        return out

    def build_block(self, kv: KV, mode: int, prev_out, prev_acc, tokens_out, b: int, q: int,
                    draft_table=None, table_stride: int = 0):
        self._bind_stream()
        _check(_lib().sdsat_build_block(self.handle, kv.handle, mode, _ptr(prev_out), _ptr(prev_acc),
                                        _ptr(draft_table), table_stride, b, q, _ptr(tokens_out)),
               "sdsat_build_block")

    # ---- tree-structured draft step 2 (Sec. 2.1.2) ----
    def block_forward_tree(self, kv: KV, tokens, parent, logits, b: int, q: int):
        self._bind_stream()
        _check(_lib().sdsat_block_forward_tree(self.handle, kv.handle, _ptr(tokens), _ptr(parent), b, q,
                                               _ptr(logits)), "sdsat_block_forward_tree")

    def accept_tree(self, kv: KV, logits, tokens, parent, b: int, q: int, accepted_len, out_tokens, path=None,
                    temperature: float = 0.0, top_p: float = 1.0, seed: int = 0, top_k: int = 0,
                    commit: bool = True):
        self._bind_stream()
        _check(_lib().sdsat_accept_tree(self.handle, kv.handle, _ptr(logits), _ptr(tokens), _ptr(parent), b, q,
                                        temperature, top_p, seed, top_k, _ptr(accepted_len), _ptr(out_tokens),
                                        _ptr(path), int(commit)), "sdsat_accept_tree")

    def build_tree_block(self, kv: KV, mode: int, prev_out, prev_q: int, prev_acc, tokens_out, b: int, k: int,
                         draft_tables=None, width: int = 1, table_stride: int = 0):
        self._bind_stream()
        _check(_lib().sdsat_build_tree_block(self.handle, kv.handle, mode, _ptr(prev_out), prev_q, _ptr(prev_acc),
                                             _ptr(draft_tables), width, table_stride, b, k, _ptr(tokens_out)),
               "sdsat_build_tree_block")

    # ---- pipelined variant ----
    def build_pipelined_block(self, kv: KV, prev_out, prev_acc, mode, n_verify, tokens_out, b: int, k: int,
                              draft_table=None, table_stride: int = 0):
        self._bind_stream()
        _check(_lib().sdsat_build_pipelined_block(self.handle, kv.handle, _ptr(prev_out), _ptr(prev_acc), _ptr(mode),
                                                  _ptr(n_verify), _ptr(draft_table), table_stride, b, k,
                                                  _ptr(tokens_out)), "sdsat_build_pipelined_block")

    def accept_pipelined(self, kv: KV, logits, tokens, n_verify, b: int, q: int, accepted_len, out_tokens,
                         temperature: float = 0.0, top_p: float = 1.0, seed: int = 0, top_k: int = 0,
                         commit: bool = True):
        self._bind_stream()
        _check(_lib().sdsat_accept_pipelined(self.handle, kv.handle, _ptr(logits), _ptr(tokens), _ptr(n_verify), b, q,
                                             temperature, top_p, seed, top_k, _ptr(accepted_len), _ptr(out_tokens),
                                             int(commit)), "sdsat_accept_pipelined")

    def prefill(self, kv: KV, seq: int, tokens):
        self._bind_stream()
        _check(_lib().sdsat_prefill(self.handle, kv.handle, seq, _ptr(tokens), tokens.numel()), "sdsat_prefill")

    def get_error(self) -> int:
        """Synchronise; return and clear the device error bits."""
        self._bind_stream()
        f = ctypes.c_uint32(0)
        st = _lib().sdsat_get_error(self.handle, ctypes.byref(f))
        if st not in (0, 5):
            raise SdsatError(st, "sdsat_get_error")
        return f.value

    # ---- single kernels ----
    def op_gemm(self, x, w, y):
        self._bind_stream()
        M, K = x.shape
        N = w.shape[0]
        _check(_lib().sdsat_op_gemm(self.handle, _ptr(x), M, K, _ptr(w), N, _ptr(y)), "sdsat_op_gemm")

    def op_attention(self, q, k, v, lens, b: int, qn: int, H: int, hd: int, cap: int, out):
        self._bind_stream()
        _check(_lib().sdsat_op_attention(self.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(lens), b, qn, H, hd, cap,
                                         _ptr(out)), "sdsat_op_attention")

    def op_prefix_attention(self, q, k, v, table, shared, lens, b: int, qn: int, H: int, Hk: int, hd: int, out, anc=None):
        """q, out [b*qn][H*hd] fp32 or bf16 (rows any distance apart); k, v bf16 [pages][Hk][PAGE][hd]; table int32
        [b][columns]; shared (leading columns equal to sequence 0's, may be None) and lens int32 [b]; anc int32 [b*qn]
        block-row masks of a tree block."""
        self._bind_stream()
        (qp, q_ld, kind, q_rows, q_cols), (op, out_ld, kind_out, out_rows, out_cols) = _rows(q), _rows(out)
        if kind != kind_out:
            raise ValueError("q and out are of different types")
        (sequences, columns), pages = table.shape, k.size(0)
        if sequences < b or q_rows < b * qn or out_rows < b * qn:
            raise ValueError("fewer rows than b or b * qn")
        if H > 0 and Hk > 0 and H % Hk == 0 and hd in (64, 128):   # (the library refuses other heads)
            if q_cols < H * hd or out_cols < H * hd:
                raise ValueError("fewer columns than H * hd")
            want = (pages, Hk, PAGE, hd)
            if k.shape != want or v.shape != want:
                raise ValueError("expected pages of [Hk][%d][hd]" % PAGE)
        _check(_lib().sdsat_op_prefix_attention(self.handle, qp, q_ld, _array(k, _bf16, 0), _array(v, _bf16, 0), pages,
                                                _array(table, _i32, 0), columns, _array(shared, _i32, b), _array(lens, _i32, b),
                                                _array(anc, _i32, b * qn), b, qn, H, Hk, hd, op, out_ld, kind),
               "sdsat_op_prefix_attention")

    def op_logprobs(self, logits, tokens=None, logp=None, entropy=None, rank=None, top_ids=None, top_logp=None,
                    temperature: float = 1.0):
        """logits [rows][vocab] fp32 or bf16 (rows any distance apart); tokens, rank int32 and logp, entropy fp32 [rows];
        top_ids int32 and top_logp fp32 [rows][n]."""
        self._bind_stream()
        lp, ld, kind, rows, vocab = _rows(logits)
        n = 0 if top_ids is None else top_ids.size(1)
        if n and top_logp is not None and top_logp.size(1) != n:
            raise ValueError("top_ids and top_logp are of different widths")
        _check(_lib().sdsat_op_logprobs(self.handle, lp, ld, kind, rows, vocab, _array(tokens, _i32, rows), temperature, n,
                                        _array(logp, _f32, rows), _array(entropy, _f32, rows), _array(rank, _i32, rows),
                                        _array(top_ids, _i32, rows * n), _array(top_logp, _f32, rows * n)), "sdsat_op_logprobs")

    # ---- ragged batches on pages: rows starts[s] .. starts[s + 1] - 1 are sequence s's new ones ----
    def rope(self, dims: int, max_position: int, theta: float = 1e4, interleaved: bool = False, scaling: str = None,
             factor: float = 1.0, low: float = 1.0, high: float = 32.0, original: int = 0, magnitude: float = 1.0) -> Rope:
        """The rotation of the first `dims` dimensions of a head; scaling None, "linear" or "parts" (see sdsat.h)."""
        if scaling not in ROPE_SCALING:
            raise ValueError("scaling: expected one of %s" % list(ROPE_SCALING))
        self._bind_stream()
        return Rope(self, RopeConfig(dims, int(interleaved), max_position, ROPE_SCALING[scaling], original, 0, theta, factor, low,
                                     high, magnitude))

    def op_rotary_append(self, rope: Rope, q, k, v, q_out, k_pages, v_pages, table, lens, starts, H: int, Hk: int, hd: int,
                         positions=None, q_gain=None, k_gain=None, eps: float = 1e-5, refs=None):
        """q, q_out [rows][H*hd], k and v [rows][Hk*hd], all fp32 or all bf16 (rows any distance apart); k_pages, v_pages bf16
        [pages][Hk][PAGE][hd]; table int32 [b][columns]; lens int32 [b]; starts int32 [b + 1]; positions int32 [rows];
        gains bf16 [hd]; refs int32 [pages]."""
        if _calls is None:
            _types()
        _check(_calls.rotary_append(self.handle, rope.handle, q, k, v, q_out, k_pages, v_pages, table, lens, starts, H, Hk, hd,
                                     positions, q_gain, k_gain, eps, refs), "sdsat_op_rotary_append")

    def op_chunk_attention(self, q, k_pages, v_pages, table, lens, starts, H: int, Hk: int, hd: int, out):
        """q, out [rows][H*hd], both fp32 or bf16 (rows any distance apart); k_pages, v_pages bf16 [pages][Hk][PAGE][hd];
        table int32 [b][columns]; lens int32 [b]; starts int32 [b + 1]."""
        if _calls is None:
            _types()
        _check(_calls.chunk_attention(self.handle, q, k_pages, v_pages, table, lens, starts, H, Hk, hd, out), "sdsat_op_chunk_attention")

    def op_adjust_logits(self, logits, out, q: int = 1, history=None, history_lens=None, prompt_lens=None, tokens=None, anc=None,
                         repetition=None, frequency=None, presence=None, bias_ids=None, bias=None, allowed=None):
        """logits, out [b*q][vocab], both fp32 or bf16 (rows any distance apart); history int32 [b][n]; history_lens, prompt_lens
        int32 [b]; tokens, anc int32 [b*q]; repetition, frequency, presence fp32 [b]; bias_ids int32 and bias fp32 [b][m];
        allowed int32 [b*q][words of 32 ids]."""
        if _calls is None:
            _types()
        _check(_calls.adjust_logits(self.handle, logits, out, q, history, history_lens, prompt_lens, tokens, anc, repetition,
                                     frequency, presence, bias_ids, bias, allowed), "sdsat_op_adjust_logits")

    def debug_workspace(self, which: int, rows: int):
        """Last-layer workspace of the last forward: 0 h, 1 q, 2 attention out, 3 SwiGLU act."""
        import torch
        s = self.shape
        cols = [s.d_model, s.n_heads * s.head_dim, s.n_heads * s.head_dim, s.ffn_dim][which]
        out = torch.empty(rows, cols, device="cuda")
        self._bind_stream()
        _check(_lib().sdsat_debug_workspace(self.handle, which, rows, _ptr(out)), "sdsat_debug_workspace")
        return out

    def debug_wait_timeout(self):
        """Queue a kernel whose bounded wait runs out (device bit TIMEOUT after ~2 s)."""
        self._bind_stream()
        _check(_lib().sdsat_debug_wait_timeout(self.handle), "sdsat_debug_wait_timeout")

    def op_exp(self, x, y):
        self._bind_stream()
        _check(_lib().sdsat_op_exp(self.handle, _ptr(x), _ptr(y), x.numel()), "sdsat_op_exp")

    def close(self):
        if getattr(self, "handle", None):
            _lib().sdsat_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
