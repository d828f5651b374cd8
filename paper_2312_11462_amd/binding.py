"""ctypes binding of libcsd.so: same names as the C ABI, torch tensors in, torch tensors out.

Only marshalling happens here; every step of the verify path runs in the HIP kernels.
`import torch` must come before the library is loaded so that the library binds to the HIP
runtime PyTorch already brought into the process (one runtime, shared streams and pointers).
"""
from __future__ import annotations

import ctypes as C
import math
import operator
import os
import struct
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libcsd.so")

EXPORTS = ["csd_version", "csd_last_hip_error", "csd_model_create", "csd_model_destroy", "csd_kv_bytes",
           "csd_kv_write", "csd_kv_read", "csd_cross_kv_init", "csd_bigram_fit", "csd_bigram_draft", "csd_maxgram_draft", "csd_verify_block",
           "csd_accept", "csd_verify_accept", "csd_verify_accept_static", "csd_review_ctx", "csd_bigram_draft_append", "csd_cascade_gate", "csd_verify_tree", "csd_tree_accept", "csd_tree_commit",
           "csd_paged_write", "csd_paged_read", "csd_paged_attention", "csd_paged_commit", "csd_paged_cross_attention", "csd_pages_plan", "csd_pages_release", "csd_pages_share", "csd_sample", "csd_filter_probs", "csd_stream_capture", "csd_debug_set_trace", "csd_debug_path", "csd_debug_gemm_plan", "csd_debug_tall_plan", "csd_debug_copy", "csd_debug_read", "csd_debug_mfma",
           "csd_prof_enable", "csd_prof_read"]

_STATUS = {-1: "CSD_EINVAL", -2: "CSD_ESHAPE", -3: "CSD_ENULL", -4: "CSD_EHIP", -5: "CSD_EUNSUPPORTED"}


class CsdError(RuntimeError):
    def __init__(self, what, status, hip=0):
        super().__init__(f"{what}: {_STATUS.get(status, status)}" + (f" (hipError {hip})" if status == -4 else ""))
        self.status = status


class Cfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("arch", "dtype", "n_layers", "d_model", "n_heads", "head_dim", "d_ffn", "vocab",
                 "max_batch", "max_seq", "max_block", "enc_len")] + \
               [("rms_eps", C.c_float), ("rope_theta", C.c_float)]


class Review(C.Structure):
    """csd_review: device pointers of one review with device-resident control."""
    _fields_ = [("ctx", C.c_void_p), ("ctx_stride", C.c_int32), ("ctx_len", C.c_void_p), ("cache_len", C.c_void_p),
                ("prefix_len", C.c_void_p), ("q_tab", C.c_void_p), ("q_onehot_tab", C.c_void_p), ("q_base", C.c_void_p),
                ("q_stride", C.c_int32), ("u_acc_tab", C.c_void_p), ("u_samp_tab", C.c_void_p), ("out_q_tab", C.c_void_p),
                ("out_onehot_tab", C.c_void_p), ("out_base", C.c_void_p), ("out_stride", C.c_int32),
                ("lower_cache_len", C.c_void_p * 4), ("n_lower", C.c_int32), ("n_accepted", C.c_void_p),
                ("next_token", C.c_void_p), ("status", C.c_void_p), ("ext_rows", C.c_void_p)]


class PagedPool(C.Structure):
    """csd_paged_kv: a paged cache and the page table of a call."""
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_pages", "page_rows", "n_kv_heads", "head_dim", "dtype")] + \
               [(n, C.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "table")] + [("table_stride", C.c_int32)]


class PageTable(C.Structure):
    """csd_pages: which sequence holds which pages."""
    _fields_ = [(n, C.c_int32) for n in ("n_pages", "page_rows", "n_sequences", "table_stride")] + \
               [(n, C.c_void_p) for n in ("table", "held", "free_pages", "n_free", "users")]


class Filter(C.Structure):
    """csd_filter: the parameters of draws from logits."""
    _fields_ = [(n, C.c_void_p) for n in ("temperature", "top_k", "top_p", "min_p")] + \
               [("temperature_all", C.c_float), ("top_k_all", C.c_int32), ("top_p_all", C.c_float), ("min_p_all", C.c_float), ("rows_each", C.c_int32)]


_P, _I, _L = C.c_void_p, C.c_int32, C.c_int64
# the paged calls are short: ctypes converts plain integers by these, without an object per argument
_ARGTYPES = {"csd_paged_write": [_P, _I, _P, _P, _I, _I, _P, _L, _P, _L, _I, _P],
             "csd_paged_read": [_P, _I, _P, _P, _I, _I, _P, _L, _P, _L, _I, _P],
             "csd_paged_attention": [_P, _I, _P, _P, _P, _I, _I, _I, _P, _L, _I, _I, C.c_float, _P, _P, _P],
             "csd_paged_commit": [_P, _P, _P, _P, _I, _I, _P],
             "csd_paged_cross_attention": [_P, _I, _P, _P, _I, _I, _I, _P, _L, _I, _I, C.c_float, _P, _P, _P],
             "csd_pages_plan": [_P, _P, _P, _I, _P, _P, _P, _P, _P, _P],
             "csd_pages_release": [_P, _P, _P],
             "csd_pages_share": [_P, _P, _P, _P],
             "csd_sample": [_P, _P, _L, _I, _I, _I, _P, _P, _P, _P],
             "csd_filter_probs": [_P, _P, _L, _I, _I, _I, _P, _P],
             "csd_stream_capture": [_P, _P]}
PAGED_WORKSPACE_BYTES, PAGED_WORKSPACE_ZERO_BYTES = 72 << 20, 64 << 10
_ROWS = {torch.float32: 0, torch.bfloat16: 1}     # types of dense rows

_lib = None


def library_path() -> str:
    return _LIB_PATH


def lib():
    """The loaded library; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
        L = C.CDLL(_LIB_PATH)
        L.csd_version.restype = C.c_char_p
        L.csd_kv_bytes.restype = C.c_size_t
        L.csd_kv_bytes.argtypes = [C.c_void_p]
        for n in EXPORTS:
            if n not in ("csd_version", "csd_kv_bytes"):
                getattr(L, n).restype = C.c_int32
        for n, types in _ARGTYPES.items():
            getattr(L, n).argtypes = types
        _lib = L
    return _lib


def _chk(rc, what):
    if rc != 0:
        raise CsdError(what, rc, lib().csd_last_hip_error())


def _ptr(t, dtype=None):
    if t is None:
        return C.c_void_p(0)
    if not t.is_cuda:
        raise ValueError("device tensor required")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError("contiguous tensor required")
    return C.c_void_p(t.data_ptr())


# (not a public name: a build of torch without it takes the public way)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


# (likewise: the public way also looks whether the runtime is up, which it is once there is a tensor)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", None) or torch.cuda.is_current_stream_capturing


def _stream():
    """The current device's current stream.  Its handle alone: torch.cuda.current_stream() makes an object around it, 2.8 us a call
    against 0.2, which the smallest calls (10 us of kernels) waited for."""
    return C.c_void_p(_raw_stream(torch.cuda.current_device()))


class Model:
    """csd_model plus the KV cache tensor the caller owns."""

    def __init__(self, shape, weights, max_batch=1, max_seq=2048, max_block=16):
        dtype = 1 if shape.dtype == "bf16" else 0
        self.shape = shape
        self.cfg = Cfg(shape.arch, dtype, shape.n_layers, shape.d_model, shape.n_heads, shape.head_dim,
                       shape.d_ffn, shape.vocab, max_batch, max_seq, max_block, getattr(shape, "enc_len", 0),
                       shape.rms_eps, shape.rope_theta)
        want = torch.bfloat16 if dtype == 1 else torch.float32
        ptrs = []
        for i, w in enumerate(weights):
            bias_table = shape.arch == 1 and i == len(weights) - 1       # relative-position bias: always fp32
            ptrs.append(_ptr(w, want if (w.ndim == 2 and not bias_table) else torch.float32).value)
        arr = (C.c_void_p * len(ptrs))(*ptrs)
        self._h = C.c_void_p()
        _chk(lib().csd_model_create(C.byref(self.cfg), arr, len(ptrs), _stream(), C.byref(self._h)), "csd_model_create")
        torch.cuda.current_stream().synchronize()     # the caller's weights may now be freed
        self.kv = torch.zeros(lib().csd_kv_bytes(self._h), dtype=torch.uint8, device="cuda")
        self.max_batch, self.max_seq, self.max_block = max_batch, max_seq, max_block

    def close(self):
        if getattr(self, "_h", None):
            torch.cuda.synchronize()
            lib().csd_model_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def cross_kv_init(self, enc_out):
        """arch 1: enc_out [B][enc_len][d] fp32 on the device -> cross-attention keys/values in the cache."""
        _chk(lib().csd_cross_kv_init(self._h, _ptr(self.kv), _ptr(enc_out, torch.float32), enc_out.shape[0], _stream()),
             "csd_cross_kv_init")

    def kv_write(self, layer, b, pos0, K, V):
        n = K.shape[0]
        _chk(lib().csd_kv_write(self._h, _ptr(self.kv), layer, b, pos0, n, _ptr(K, torch.float32),
                                _ptr(V, torch.float32), _stream()), "csd_kv_write")

    def kv_read(self, layer, b, pos0, n):
        hd = self.shape.n_heads * self.shape.head_dim
        K = torch.empty((n, hd), dtype=torch.float32, device="cuda")
        V = torch.empty((n, hd), dtype=torch.float32, device="cuda")
        _chk(lib().csd_kv_read(self._h, _ptr(self.kv), layer, b, pos0, n, _ptr(K), _ptr(V), _stream()), "csd_kv_read")
        return K, V

    def verify_block(self, tokens, cache_len, temperature=1.0, want_probs=False, logits=None, probs=None):
        """tokens [B][m] int32, cache_len [B] int32 (device) -> logits [B][m][V] (and probs)."""
        B, m = tokens.shape
        V = self.shape.vocab
        if logits is None:
            logits = torch.empty((B, m, V), dtype=torch.float32, device="cuda")
        if want_probs and probs is None:
            probs = torch.empty((B, m, V), dtype=torch.float32, device="cuda")
        _chk(lib().csd_verify_block(self._h, _ptr(self.kv), _ptr(tokens, torch.int32), _ptr(cache_len, torch.int32),
                                    B, m, C.c_float(temperature), _ptr(logits), _ptr(probs), _stream()),
             "csd_verify_block")
        return (logits, probs) if want_probs else logits

    def verify_accept(self, tokens, cache_len, u_acc, u_samp, q=None, q_onehot=None, temperature=1.0,
                      lenience=1.0, mode=0, logits=None, probs=None, n_accepted=None, next_token=None, static=False):
        """static=True: csd_verify_accept_static (scratch in the library's static device array)."""
        B, m = tokens.shape
        if n_accepted is None:
            n_accepted = torch.empty(B, dtype=torch.int32, device="cuda")
        if next_token is None:
            next_token = torch.empty(B, dtype=torch.int32, device="cuda")
        fn = lib().csd_verify_accept_static if static else lib().csd_verify_accept
        _chk(fn(self._h, _ptr(self.kv), _ptr(tokens, torch.int32), _ptr(cache_len, torch.int32),
                B, m, C.c_float(temperature), _ptr(q), _ptr(q_onehot), _ptr(u_acc), _ptr(u_samp),
                C.c_float(lenience), mode, _ptr(logits), _ptr(probs), _ptr(n_accepted),
                _ptr(next_token), _stream()), "csd_verify_accept_static" if static else "csd_verify_accept")
        return n_accepted, next_token

    def verify_tree(self, tokens, parent, cache_len, temperature=1.0, want_probs=False, logits=None, probs=None):
        """csd_verify_tree: tokens, parent [B][m] int32 (device) -> logits [B][m][V] (and probs)."""
        B, m = tokens.shape
        V = self.shape.vocab
        if logits is None:
            logits = torch.empty((B, m, V), dtype=torch.float32, device="cuda")
        if want_probs and probs is None:
            probs = torch.empty((B, m, V), dtype=torch.float32, device="cuda")
        _chk(lib().csd_verify_tree(self._h, _ptr(self.kv), _ptr(tokens, torch.int32), _ptr(parent, torch.int32),
                                   _ptr(cache_len, torch.int32), B, m, C.c_float(temperature), _ptr(logits), _ptr(probs),
                                   _stream()), "csd_verify_tree")
        return (logits, probs) if want_probs else logits

    def tree_commit(self, cache_len, path, n_accepted):
        """csd_tree_commit: the kept rows' K/V move to where a plain block would have stored them."""
        B, m = path.shape
        _chk(lib().csd_tree_commit(self._h, _ptr(self.kv), _ptr(cache_len, torch.int32), _ptr(path, torch.int32),
                                   _ptr(n_accepted, torch.int32), B, m, _stream()), "csd_tree_commit")

    def review_ctx(self, ctx, ctx_len, cache_len, prefix_len, m_max, status, q_tab=None, q_onehot_tab=None, q_base=None,
                   u_acc_tab=None, u_samp_tab=None, out_q_tab=None, out_onehot_tab=None, out_base=None, lower=(),
                   n_accepted=None, next_token=None, ext_rows=None, temperature=1.0, lenience=1.0, mode=0):
        """csd_review_ctx: one review with device-resident control (every tensor stays on the device)."""
        def dp(t):
            return None if t is None else t.data_ptr()
        r = Review()
        r.ctx, r.ctx_stride, r.ctx_len, r.cache_len, r.prefix_len = dp(ctx), ctx.shape[1], dp(ctx_len), dp(cache_len), dp(prefix_len)
        r.q_tab, r.q_onehot_tab, r.q_base = dp(q_tab), dp(q_onehot_tab), dp(q_base)
        r.q_stride = (q_onehot_tab if q_onehot_tab is not None else q_tab).shape[1] if (q_tab is not None or q_onehot_tab is not None) else 0
        r.u_acc_tab, r.u_samp_tab = dp(u_acc_tab), dp(u_samp_tab)
        r.out_q_tab, r.out_onehot_tab, r.out_base = dp(out_q_tab), dp(out_onehot_tab), dp(out_base)
        r.out_stride = (out_onehot_tab if out_onehot_tab is not None else out_q_tab).shape[1] if (out_q_tab is not None or out_onehot_tab is not None) else 0
        for i, t in enumerate(lower):
            r.lower_cache_len[i] = t.data_ptr()
        r.n_lower = len(lower)
        r.n_accepted, r.next_token, r.status, r.ext_rows = dp(n_accepted), dp(next_token), dp(status), dp(ext_rows)
        _chk(lib().csd_review_ctx(self._h, _ptr(self.kv), C.byref(r), ctx.shape[0], m_max, C.c_float(temperature),
                                  C.c_float(lenience), mode, _stream()), "csd_review_ctx")

    def set_trace(self, trace):
        _chk(lib().csd_debug_set_trace(self._h, _ptr(trace)), "csd_debug_set_trace")

    def path(self, B, m):
        return int(lib().csd_debug_path(self._h, B, m))

    def prof_enable(self, on=True):
        _chk(lib().csd_prof_enable(self._h, 1 if on else 0), "csd_prof_enable")

    def prof_read(self, kernel_class, reset=False):
        ms, n = C.c_double(), C.c_int64()
        _chk(lib().csd_prof_read(self._h, kernel_class, C.byref(ms), C.byref(n), 1 if reset else 0), "csd_prof_read")
        return ms.value, n.value


class PagedKv:
    """A paged KV cache: the pools k and v [layers][pages][kv heads][rows of a page][head dim] (torch.float32, bfloat16 or float8_e4m3fn;
    the latter with scale bytes k_scale, v_scale, uint8 of the same shape without the last dimension), which the caller made and owns.

    Every call takes the page table [B][n] int32 (entries outside [0, pages): no rows there) and the ragged rows of a batch: row_start
    [B + 1] int32, and a position [B] int32 for each sequence's first row.  Rows are [rows][heads][head dim], float32 or bfloat16,
    with any distance between rows that is a multiple of 8 elements.  All tensors are on the pools' device, which has to be the current one,
    and the work is enqueued on its current stream.  The attention has a workspace (PAGED_WORKSPACE_BYTES; for bf16 queries, heads of 64 or 128, pools
    of bf16 or e4m3) for every stream that it is called on and for every capture, made at the first call there, so that calls on several streams and graphs that are replayed side by side may overlap.
    A workspace that is given serves all calls, which then must not overlap."""

    def __init__(self, k, v, k_scale=None, v_scale=None, workspace=None):
        types = {torch.float32: 0, torch.bfloat16: 1, torch.float8_e4m3fn: 2}
        if k.ndim != 5 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in types:
            raise ValueError("k and v: [layers][pages][kv heads][rows of a page][head dim], both float32, bfloat16 or float8_e4m3fn")
        if (k.dtype == torch.float8_e4m3fn) != (k_scale is not None) or (k_scale is None) != (v_scale is None):
            raise ValueError("k_scale and v_scale belong to float8_e4m3fn pools")
        self._dev = k.get_device()
        for t in (v, k_scale, v_scale, workspace):
            if t is not None and t.get_device() != self._dev:
                raise ValueError("all tensors of a cache belong on one device")
        if k_scale is not None and (k_scale.shape != k.shape[:-1] or v_scale.shape != k.shape[:-1]):
            raise ValueError("k_scale and v_scale: the pools' shape without the last dimension")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_rows, self.head_dim = k.shape
        self._pool = PagedPool(self.n_layers, self.n_pages, self.page_rows, self.n_kv_heads, self.head_dim, types[k.dtype],
                               _ptr(k).value, _ptr(v).value, _ptr(k_scale, torch.uint8).value, _ptr(v_scale, torch.uint8).value, None, 0)
        self._threads, self._lib, self._device = threading.local(), lib(), k.device
        if workspace is not None and workspace.numel() * workspace.element_size() < PAGED_WORKSPACE_BYTES:
            raise ValueError(f"workspace: {PAGED_WORKSPACE_BYTES} bytes, the first {PAGED_WORKSPACE_ZERO_BYTES} of them zeroed")
        self.workspace = workspace
        self._ws = _ptr(workspace).value
        self._split = self.head_dim in (64, 128) and k.dtype is not torch.float32      # (with bf16 queries: the work of a call may be split, in a workspace)
        self._eager, self._captured = {}, {}              # by stream: (address, tensor), (capture, address, tensor)

    def _workspace_of(self, stream):
        """The address of the current stream's own workspace.  While the stream is captured, that of the capture, from the graph's memory and zeroed
        by the graph; the one of the stream's last capture is let go of (its memory stays with its graph)."""
        if not _capturing():
            held = self._eager.get(stream)
            return (held or self._eager.setdefault(stream, self._new_workspace()))[0]
        capture = C.c_uint64()
        _chk(self._lib.csd_stream_capture(stream, C.addressof(capture)), "csd_stream_capture")
        held = self._captured.get(stream)
        if held is None or held[0] != capture.value:
            held = self._captured[stream] = (capture.value, *self._new_workspace())
        return held[1]

    def _new_workspace(self):
        workspace = torch.empty(PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device=self._device)
        workspace[:PAGED_WORKSPACE_ZERO_BYTES].zero_()
        return workspace.data_ptr(), workspace

    def _mine(self):
        """The call's description of the cache, whose page table a call sets: one per thread."""
        try:
            return self._threads.mine
        except AttributeError:
            pool = PagedPool.from_buffer_copy(self._pool)
            self._threads.mine = pool, C.addressof(pool)
            return self._threads.mine

    def _check(self, **tensors):
        """Raises for what is wrong with a call's tensors.  The methods look at everything in one expression and come here only if it does not hold
        (which strides of dimensions of size one may also cause): checked one by one, in functions, they took as long as the smallest kernels."""
        if _current_device() != self._dev:
            raise ValueError("the cache is on another device than the current one")
        dtype = None
        for name, (t, want) in tensors.items():
            if t.get_device() != self._dev:
                raise ValueError(f"{name}: a tensor on the cache's device is required")
            if isinstance(want, int):                      # int32, so many elements
                if t.dtype is not torch.int32:
                    raise TypeError(f"{name}: expected torch.int32, got {t.dtype}")
                if t.numel() != want or not t.is_contiguous():
                    raise ValueError(f"{name}: {want} contiguous elements are required")
                continue
            if t.dtype not in _ROWS or dtype not in (None, t.dtype):
                raise TypeError(f"{name}: rows are float32 or bfloat16, all of a call alike, got {t.dtype}")
            dtype = t.dtype
            if tuple(t.shape) != want or (want[2] > 1 and t.stride(2) != 1) or (want[1] > 1 and t.stride(1) != want[2]):
                raise ValueError(f"{name}: {list(want)} with contiguous rows is required, got {list(t.shape)} with strides {list(t.stride())}")

    def write(self, layer, table, row_start, cache_len, k_rows, v_rows):
        """csd_paged_write: row r of sequence b becomes position cache_len[b] + r - row_start[b]."""
        dev, i32, d, heads = self._dev, torch.int32, self.head_dim, self.n_kv_heads
        B, n = table.shape
        shape, dtype, ks, vs = k_rows.shape, k_rows.dtype, k_rows.stride(), v_rows.stride()
        rows = shape[0]
        if not (dev == table.get_device() == row_start.get_device() == cache_len.get_device() == k_rows.get_device() == v_rows.get_device()
                and i32 is table.dtype is row_start.dtype is cache_len.dtype and table.is_contiguous() and row_start.is_contiguous()
                and cache_len.is_contiguous() and row_start.numel() == B + 1 and cache_len.numel() == B and dtype in _ROWS
                and v_rows.dtype is dtype and (rows, heads, d) == shape == v_rows.shape and (d, 1) == ks[1:] == vs[1:] and _current_device() == dev):
            self._check(table=(table, B * n), row_start=(row_start, B + 1), cache_len=(cache_len, B), k_rows=(k_rows, (rows, heads, d)),
                        v_rows=(v_rows, (rows, heads, d)))
        pool, ref = self._mine()
        pool.table, pool.table_stride = table.data_ptr(), n
        rc = self._lib.csd_paged_write(ref, layer, row_start.data_ptr(), cache_len.data_ptr(), B, rows, k_rows.data_ptr(),
                                       ks[0] if rows > 1 else heads * d, v_rows.data_ptr(), vs[0] if rows > 1 else heads * d, _ROWS[dtype],
                                       _raw_stream(dev))
        if rc:
            _chk(rc, "csd_paged_write")

    def read(self, layer, table, row_start, cache_len, rows, dtype=torch.float32, out=None):
        """csd_paged_read: (k, v) [rows][kv heads][head dim], row r of sequence b from position cache_len[b] + r - row_start[b].
        out: the two tensors to fill; rows of no sequence are left as they are (undefined in new tensors)."""
        dev, i32, d, heads = self._dev, torch.int32, self.head_dim, self.n_kv_heads
        B, n = table.shape
        if out is None:
            k = torch.empty(rows, heads, d, dtype=dtype, device=self._device)
            v = torch.empty_like(k)
            ok = dtype in _ROWS
        else:
            k, v = out
            dtype = k.dtype
            ok = (dev == k.get_device() == v.get_device() and dtype in _ROWS and v.dtype is dtype and (rows, heads, d) == k.shape == v.shape
                  and (d, 1) == k.stride()[1:] == v.stride()[1:])
        if not (ok and dev == table.get_device() == row_start.get_device() == cache_len.get_device()
                and i32 is table.dtype is row_start.dtype is cache_len.dtype and table.is_contiguous() and row_start.is_contiguous()
                and cache_len.is_contiguous() and row_start.numel() == B + 1 and cache_len.numel() == B and _current_device() == dev):
            self._check(table=(table, B * n), row_start=(row_start, B + 1), cache_len=(cache_len, B), k=(k, (rows, heads, d)), v=(v, (rows, heads, d)))
        pool, ref = self._mine()
        pool.table, pool.table_stride = table.data_ptr(), n
        rc = self._lib.csd_paged_read(ref, layer, row_start.data_ptr(), cache_len.data_ptr(), B, rows, k.data_ptr(),
                                      k.stride(0) if rows > 1 else heads * d, v.data_ptr(), v.stride(0) if rows > 1 else heads * d, _ROWS[dtype],
                                      _raw_stream(dev))
        if rc:
            _chk(rc, "csd_paged_read")
        return k, v

    def attention(self, layer, table, row_start, cache_len, q, scale, max_rows=None, parent=None, out=None):
        """csd_paged_attention: q [rows][heads][head dim] -> out, contiguous and of q's type; rows of no sequence are left as they are
        (undefined in a new tensor).  max_rows: at least the rows of the longest sequence of the batch (default: all rows of the call, for
        several trees 64 at most; the kernels are chosen by it, so single tokens and short blocks are served best where it is given);
        parent: tree blocks, of 64 rows at most."""
        dev, i32, d = self._dev, torch.int32, self.head_dim
        B, n = table.shape
        rows, heads, width = q.shape
        dtype, qs = q.dtype, q.stride()
        if not (dev == table.get_device() == row_start.get_device() == cache_len.get_device() == q.get_device()
                and i32 is table.dtype is row_start.dtype is cache_len.dtype and table.is_contiguous() and row_start.is_contiguous()
                and cache_len.is_contiguous() and row_start.numel() == B + 1 and cache_len.numel() == B and dtype in _ROWS and width == d
                and qs[1:] == (d, 1) and _current_device() == dev):
            self._check(table=(table, B * n), row_start=(row_start, B + 1), cache_len=(cache_len, B), q=(q, (rows, heads, d)))
        if out is None:
            out = torch.empty(rows, heads, d, dtype=dtype, device=self._device)
        elif not (out.dtype is dtype and out.shape == q.shape and out.get_device() == dev and out.is_contiguous()):
            self._check(q=(q, (rows, heads, d)), out=(out, (rows, heads, d)))
            raise ValueError("out: a contiguous tensor is required")
        up = None
        if parent is not None:
            self._check(parent=(parent, rows))
            up = parent.data_ptr()
            if max_rows is None and B > 1:
                max_rows = min(rows, 64) or 1
        pool, ref = self._mine()
        pool.table, pool.table_stride = table.data_ptr(), n
        stream = _raw_stream(dev)
        rc = self._lib.csd_paged_attention(ref, layer, row_start.data_ptr(), cache_len.data_ptr(), up, B, rows,
                                           (rows or 1) if max_rows is None else max_rows, q.data_ptr(), qs[0] if rows > 1 else heads * d, heads,
                                           _ROWS[dtype], scale, out.data_ptr(),
                                           self._ws or (self._workspace_of(stream) if self._split and dtype is torch.bfloat16 else None), stream)
        if rc:
            _chk(rc, "csd_paged_attention")
        return out

    def cross_attention(self, layer, table, row_start, enc_len, q, scale, max_rows=None, out=None):
        """csd_paged_cross_attention: every row of sequence b attends the enc_len[b] rows that its table names (an encoder's projected states, written once with
        `write`); q, out, scale and max_rows as for `attention`."""
        dev, i32, d = self._dev, torch.int32, self.head_dim
        B, n = table.shape
        rows, heads, width = q.shape
        dtype, qs = q.dtype, q.stride()
        if not (dev == table.get_device() == row_start.get_device() == enc_len.get_device() == q.get_device()
                and i32 is table.dtype is row_start.dtype is enc_len.dtype and table.is_contiguous() and row_start.is_contiguous()
                and enc_len.is_contiguous() and row_start.numel() == B + 1 and enc_len.numel() == B and dtype in _ROWS and width == d
                and qs[1:] == (d, 1) and _current_device() == dev):
            self._check(table=(table, B * n), row_start=(row_start, B + 1), enc_len=(enc_len, B), q=(q, (rows, heads, d)))
        if out is None:
            out = torch.empty(rows, heads, d, dtype=dtype, device=self._device)
        elif not (out.dtype is dtype and out.shape == q.shape and out.get_device() == dev and out.is_contiguous()):
            self._check(q=(q, (rows, heads, d)), out=(out, (rows, heads, d)))
            raise ValueError("out: a contiguous tensor is required")
        pool, ref = self._mine()
        pool.table, pool.table_stride = table.data_ptr(), n
        stream = _raw_stream(dev)
        rc = self._lib.csd_paged_cross_attention(ref, layer, row_start.data_ptr(), enc_len.data_ptr(), B, rows, (rows or 1) if max_rows is None else max_rows,
                                                 q.data_ptr(), qs[0] if rows > 1 else heads * d, heads, _ROWS[dtype], scale, out.data_ptr(),
                                                 self._ws or (self._workspace_of(stream) if self._split and dtype is torch.bfloat16 else None), stream)
        if rc:
            _chk(rc, "csd_paged_cross_attention")
        return out

    def commit(self, table, cache_len, path, n_accepted):
        """csd_paged_commit: the kept rows of a tree block, path[b][: n_accepted[b]], to positions cache_len[b] + 1 .., in all layers."""
        dev, i32 = self._dev, torch.int32
        B, n = table.shape
        sequences, m = path.shape
        if not (dev == table.get_device() == path.get_device() == cache_len.get_device() == n_accepted.get_device()
                and i32 is table.dtype is path.dtype is cache_len.dtype is n_accepted.dtype and table.is_contiguous() and path.is_contiguous()
                and cache_len.is_contiguous() and n_accepted.is_contiguous() and B == sequences == cache_len.numel() == n_accepted.numel()
                and _current_device() == dev):
            self._check(table=(table, B * n), cache_len=(cache_len, B), path=(path, B * m), n_accepted=(n_accepted, B))
        pool, ref = self._mine()
        pool.table, pool.table_stride = table.data_ptr(), n
        rc = self._lib.csd_paged_commit(ref, cache_len.data_ptr(), path.data_ptr(), n_accepted.data_ptr(), B, m, _raw_stream(dev))
        if rc:
            _chk(rc, "csd_paged_commit")


class Pages:
    """Which sequence holds which pages of a paged cache, on the device (csd_pages): table [sequences][entries], held [sequences], free [pages], n_free [1], users
    [pages], all int32, contiguous and on one device; the caller made and owns them, and may read them between calls.  `Pages.new` makes them for
    sequences that hold nothing.  The calls enqueue on the current stream of the arrays' device, which has to be the current one, and change the arrays in place:
    calls on the same arrays must not overlap."""

    def __init__(self, table, held, free, n_free, users, page_rows):
        self._dev, self._device = table.get_device(), table.device
        if table.ndim != 2 or users.shape != free.shape:
            raise ValueError("table: [sequences][entries]; free and users: [pages]")
        self.n_sequences, n = table.shape
        self.n_pages, self.page_rows = free.numel(), page_rows
        for name, t, count in (("table", table, self.n_sequences * n), ("held", held, self.n_sequences), ("free", free, self.n_pages),
                               ("n_free", n_free, 1), ("users", users, self.n_pages)):
            self._check(name, t, count)
        self.table, self.held, self.free, self.n_free, self.users = table, held, free, n_free, users
        self._lib = lib()
        self._arrays = PageTable(self.n_pages, page_rows, self.n_sequences, n, *(t.data_ptr() for t in (table, held, free, n_free, users)))
        self._ref = C.addressof(self._arrays)

    @classmethod
    def new(cls, n_pages, page_rows, sequences, entries, device="cuda"):
        """For so many sequences of up to `entries` pages each, none of which holds any yet; pages are taken from 0 on."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.full((sequences, entries), -1, **i32), torch.zeros(sequences, **i32), torch.arange(n_pages - 1, -1, -1, **i32),
                   torch.full((1,), n_pages, **i32), torch.zeros(n_pages, **i32), page_rows)

    def _check(self, name, t, count):
        if t.get_device() != self._dev or self._dev < 0:
            raise ValueError(f"{name}: a tensor on the arrays' device is required")
        if t.dtype is not torch.int32:
            raise TypeError(f"{name}: expected torch.int32, got {t.dtype}")
        if t.numel() != count or not t.is_contiguous():
            raise ValueError(f"{name}: {count} contiguous elements are required")

    def _given(self, **tensors):
        """Raises for what is wrong with a call's tensors (the methods look at them in one expression, and come here if it does not hold)."""
        if _current_device() != self._dev:
            raise ValueError("the arrays are on another device than the current one")
        for name, t in tensors.items():
            self._check(name, t, self.n_sequences)

    def plan(self, cache_len, new_rows, rows):
        """csd_pages_plan: (row_start [sequences + 1], sequence [rows], position [rows], slot [rows] int64, served [sequences]); rows: the most rows of the step.
        A sequence whose new rows would lie in a page that others use too is not served."""
        n, dev = self.n_sequences, self._dev
        if not (dev == cache_len.get_device() == new_rows.get_device() and torch.int32 is cache_len.dtype is new_rows.dtype and cache_len.is_contiguous()
                and new_rows.is_contiguous() and n == cache_len.numel() == new_rows.numel() and _current_device() == dev):
            self._given(cache_len=cache_len, new_rows=new_rows)
        # (one tensor for all that is int32: a tensor made is a microsecond, as much as a step's kernel spends on its lengths)
        row_start, sequence, position, served = torch.empty(2 * (n + rows) + 1, dtype=torch.int32, device=self._device).split((n + 1, rows, rows, n))
        slot = torch.empty(rows, dtype=torch.int64, device=self._device)
        rc = self._lib.csd_pages_plan(self._ref, cache_len.data_ptr(), new_rows.data_ptr(), rows, row_start.data_ptr(), sequence.data_ptr(),
                                      position.data_ptr(), slot.data_ptr(), served.data_ptr(), _raw_stream(dev))
        if rc:
            _chk(rc, "csd_pages_plan")
        return row_start, sequence, position, slot, served

    def release(self, keep_len):
        """csd_pages_release: sequence b keeps its first keep_len[b] rows (0: it has ended; negative: it is left alone)."""
        dev = self._dev
        if not (dev == keep_len.get_device() and keep_len.dtype is torch.int32 and keep_len.is_contiguous() and keep_len.numel() == self.n_sequences
                and _current_device() == dev):
            self._given(keep_len=keep_len)
        rc = self._lib.csd_pages_release(self._ref, keep_len.data_ptr(), _raw_stream(dev))
        if rc:
            _chk(rc, "csd_pages_release")

    def share(self, source, length):
        """csd_pages_share: sequences that hold nothing take over the whole pages of the first length[b] rows of source[b] (negative: none).  Shared pages are
        not written: one that is cut inside them, the source too, has to release back to the page's first row before it gets new rows."""
        self._given(source=source, length=length)
        rc = self._lib.csd_pages_share(self._ref, source.data_ptr(), length.data_ptr(), _raw_stream(self._dev))
        if rc:
            _chk(rc, "csd_pages_share")


# csd_filter as bytes: four addresses, the numbers beside them, the rows that share an entry
_FILTER = struct.Struct("@4PfiffI")


def _filter(logits, temperature, top_k, top_p, min_p):
    """(csd_filter as a buffer, rows, elements between rows) of a call; raises for what is wrong with its tensors."""
    dev, shape = logits.get_device(), logits.shape
    if dev < 0:
        raise ValueError("logits: a device tensor is required")
    if _current_device() != dev:
        raise ValueError("logits: on another device than the current one")
    if logits.dtype not in _ROWS:
        raise TypeError(f"logits are float32 or bfloat16, got {logits.dtype}")
    if len(shape) == 2 and logits.stride(1) == 1:
        rows, V = shape
        step = logits.stride(0) if rows > 1 else V
    else:
        rows, step = _rows_of(shape, logits.stride())
    addresses, numbers, sets = [None] * 4, [1.0, 0, 1.0, 0.0], 0
    for i, value in enumerate((temperature, top_k, top_p, min_p)):
        if value is None:
            continue
        if isinstance(value, torch.Tensor):
            n = value.numel()
            if value.get_device() != dev:
                raise ValueError(f"{_PARAMETERS[i]}: a tensor on the logits' device is required")
            if value.dtype is not (torch.int32 if i == 1 else torch.float32):
                raise TypeError(f"{_PARAMETERS[i]}: expected {torch.int32 if i == 1 else torch.float32}, got {value.dtype}")
            if not value.is_contiguous() or (rows and (n == 0 or rows % n)) or sets not in (0, n):
                raise ValueError(f"{_PARAMETERS[i]}: contiguous, one entry for each row or for each of the same number of consecutive rows, all parameters alike")
            sets = n
            addresses[i] = value.data_ptr()
        else:
            numbers[i] = value
    buffer = C.create_string_buffer(_FILTER.size)
    each = rows // sets or 1 if sets else 1
    try:
        _FILTER.pack_into(buffer, 0, *(a or 0 for a in addresses), *numbers, each)
    except (struct.error, OverflowError):
        _FILTER.pack_into(buffer, 0, *(a or 0 for a in addresses), *_in_range(numbers), each)
    return buffer, rows, step


def _in_range(numbers):
    """Parameters that csd_filter's types do not hold, as ones that mean the same: a top_k beyond int32, the others beyond fp32; raises for what is no such number."""
    out = []
    for name, value in zip(_PARAMETERS, numbers):
        try:
            if name == "top_k":
                out.append(min(max(operator.index(value), 0), 2 ** 31 - 1))
            else:
                value = float(value)
                out.append(value if math.isinf(value) else max(min(value, _FP32_MAX), -_FP32_MAX))
        except (TypeError, ValueError, OverflowError):
            raise TypeError(f"{name}: expected {'a whole number' if name == 'top_k' else 'a number'}, got {value!r}") from None
    return out


_PARAMETERS = "temperature", "top_k", "top_p", "min_p"
_FP32_MAX = 3.4028234663852886e38


def _rows_of(shape, stride):
    """(rows, elements between rows) of logits [..., V] whose leading dimensions are one run of equal steps."""
    if not shape or shape[-1] == 0:
        raise ValueError("logits: [..., V] with V >= 1 is required")
    if 0 in shape:
        return 0, shape[-1]
    rows, step = 1, shape[-1]
    for size, by in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if size > 1:
            if rows == 1:
                step = by
            elif by != step * rows:
                raise ValueError("logits: rows at equal distances are required")
        rows *= size
    if shape[-1] > 1 and stride[-1] != 1:
        raise ValueError("logits: contiguous rows are required")
    return rows, step


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, probs=None, out=None):
    """csd_sample: logits [..., V] float32 or bfloat16, u [...] float32 in [0, 1) -> tokens [...] int32 (-1 for a row without a logit above -inf).  The parameters are numbers,
    or tensors with an entry for every row or for every so many consecutive rows (a sequence's block); None: not set.  probs: a float32
    tensor [..., V] that takes the probabilities too."""
    f, rows, step = _filter(logits, temperature, top_k, top_p, min_p)
    shape, dev = logits.shape, logits.get_device()
    if not (u.shape == shape[:-1] and u.dtype is torch.float32 and u.get_device() == dev and u.is_contiguous()):
        _given("u", u, shape[:-1], torch.float32, logits)
    if out is None:
        out = torch.empty_like(u, dtype=torch.int32)
    else:
        _given("out", out, shape[:-1], torch.int32, logits)
    if probs is not None:
        _given("probs", probs, shape, torch.float32, logits)
    rc = lib().csd_sample(f, logits.data_ptr(), step, _ROWS[logits.dtype], rows, shape[-1], u.data_ptr(), out.data_ptr(),
                          None if probs is None else probs.data_ptr(), _raw_stream(dev))
    if rc:
        _chk(rc, "csd_sample")
    return out


def filter_probs(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None):
    """csd_filter_probs: the probabilities [..., V] float32 of the draws that `sample` makes with these parameters, as `accept` and `tree_accept` take them."""
    f, rows, step = _filter(logits, temperature, top_k, top_p, min_p)
    if out is None:
        out = torch.empty_like(logits, dtype=torch.float32, memory_format=torch.contiguous_format)
    else:
        _given("out", out, logits.shape, torch.float32, logits)
    rc = lib().csd_filter_probs(f, logits.data_ptr(), step, _ROWS[logits.dtype], rows, logits.shape[-1], out.data_ptr(), _raw_stream(logits.get_device()))
    if rc:
        _chk(rc, "csd_filter_probs")
    return out


def _given(name, t, shape, dtype, like):
    if t.get_device() != like.get_device():
        raise ValueError(f"{name}: a tensor on the logits' device is required")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: {list(shape)}, contiguous, is required")


def debug_copy(dst, src):
    """Streaming copy of src into dst (same byte size, a multiple of 16): counter calibration."""
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("debug_copy: size mismatch")
    _chk(lib().csd_debug_copy(C.c_void_p(dst.data_ptr()), C.c_void_p(src.data_ptr()), C.c_size_t(nbytes), _stream()),
         "csd_debug_copy")


def debug_read(src, sink):
    """Streaming read of src (byte size a multiple of 16); sink: uint32/int32 device tensor of >= 2048 words."""
    nbytes = src.numel() * src.element_size()
    _chk(lib().csd_debug_read(C.c_void_p(src.data_ptr()), C.c_size_t(nbytes), C.c_void_p(sink.data_ptr()), _stream()),
         "csd_debug_read")


def debug_mfma(iters, sink):
    """4096 waves x iters x 8 matrix instructions (16x16x32 bf16) on registers; returns the flops issued."""
    _chk(lib().csd_debug_mfma(C.c_int64(iters), C.c_void_p(sink.data_ptr()), _stream()), "csd_debug_mfma")
    return 4096 * iters * 8 * 16384


def bigram_fit(tokens, vocab, next_table):
    """In-place fit of next_table [vocab] int32 (pre-filled with the default successors)."""
    _chk(lib().csd_bigram_fit(_ptr(tokens, torch.int32), tokens.shape[0], vocab, _ptr(next_table, torch.int32),
                              _stream()), "csd_bigram_fit")
    return next_table


def bigram_draft(ctx, ctx_len, next_table, k, max_match=0, want_match_len=True, out=None):
    if ctx.ndim == 1:
        ctx = ctx[None, :]
    B, stride = ctx.shape
    if out is None:
        out = torch.empty((B, k), dtype=torch.int32, device="cuda")
    elif tuple(out.shape) != (B, k):
        raise ValueError("out must be [B][k]")
    mlen = torch.empty(B, dtype=torch.int32, device="cuda") if want_match_len else None
    _chk(lib().csd_bigram_draft(_ptr(ctx, torch.int32), _ptr(ctx_len, torch.int32), B, stride,
                                _ptr(next_table, torch.int32), next_table.shape[0], k, max_match, _ptr(out),
                                _ptr(mlen), _stream()), "csd_bigram_draft")
    return (out, mlen) if want_match_len else out


def maxgram_draft(haystack, haystack_len, needle, needle_len, next_table, k, max_match=0):
    """Max-Gram with a haystack of its own: returns (tokens [B][k], match_len [B], n_copied [B])."""
    B, hs = haystack.shape
    out = torch.empty((B, k), dtype=torch.int32, device="cuda")
    mlen = torch.empty(B, dtype=torch.int32, device="cuda")
    ncp = torch.empty(B, dtype=torch.int32, device="cuda")
    _chk(lib().csd_maxgram_draft(_ptr(haystack, torch.int32), _ptr(haystack_len, torch.int32), hs, _ptr(needle, torch.int32),
                                 _ptr(needle_len, torch.int32), needle.shape[1], B, _ptr(next_table, torch.int32),
                                 next_table.shape[0], k, max_match, _ptr(out), _ptr(mlen), _ptr(ncp), _stream()),
         "csd_maxgram_draft")
    return out, mlen, ncp


def tree_accept(p, tokens, parent, u=None, mode=0):
    """csd_tree_accept: p [B][m][V] -> (n_accepted [B], path [B][m], next_token [B])."""
    B, m, V = p.shape
    n_acc = torch.empty(B, dtype=torch.int32, device="cuda")
    path = torch.full((B, m), -1, dtype=torch.int32, device="cuda")
    nxt = torch.empty(B, dtype=torch.int32, device="cuda")
    _chk(lib().csd_tree_accept(_ptr(p, torch.float32), _ptr(tokens, torch.int32), _ptr(parent, torch.int32), _ptr(u), B, m, V,
                               mode, _ptr(n_acc), _ptr(path), _ptr(nxt), _stream()), "csd_tree_accept")
    return n_acc, path, nxt


def bigram_draft_append(ctx, ctx_len, next_table, k, max_match=0, gate=None, q_onehot_tab=None, q_base=None):
    """csd_bigram_draft_append: Max-Gram drafts written at the end of the device-side sequences."""
    _chk(lib().csd_bigram_draft_append(_ptr(ctx, torch.int32), ctx.shape[1], _ptr(ctx_len, torch.int32), ctx.shape[0],
                                       _ptr(next_table, torch.int32), next_table.shape[0], k, max_match, _ptr(gate),
                                       _ptr(q_onehot_tab), _ptr(q_base), q_onehot_tab.shape[1] if q_onehot_tab is not None else 0,
                                       _stream()), "csd_bigram_draft_append")


def cascade_gate(ctx_len, gate_out, loop_start=None, need=0, parent_gate=None):
    """csd_cascade_gate: the loop condition of Algorithm 1 evaluated on the device."""
    _chk(lib().csd_cascade_gate(_ptr(ctx_len, torch.int32), _ptr(loop_start), need, _ptr(parent_gate), ctx_len.shape[0],
                                _ptr(gate_out, torch.int32), _stream()), "csd_cascade_gate")


def accept(p, q, draft, u_acc, u_samp, lenience=1.0, mode=0, q_onehot=None):
    B, k1, V = p.shape
    k = k1 - 1
    n_acc = torch.empty(B, dtype=torch.int32, device="cuda")
    nxt = torch.empty(B, dtype=torch.int32, device="cuda")
    _chk(lib().csd_accept(_ptr(p, torch.float32), _ptr(q), _ptr(q_onehot), _ptr(draft), _ptr(u_acc), _ptr(u_samp),
                          B, k, V, C.c_float(lenience), mode, _ptr(n_acc), _ptr(nxt), _stream()), "csd_accept")
    return n_acc, nxt
