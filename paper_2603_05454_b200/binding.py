"""ctypes binding with the same names as include/lsp.h.  Argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.environ.get("LSP_LIB") or os.path.join(_HERE, "liblsp_b200.so")   # LSP_LIB: another build of the library

FLAG_SNAPPED, FLAG_FALLBACK, FLAG_RANGE_UNACHIEVABLE = 1, 2, 4
FLAG_RUN_TO_END, FLAG_NEAR_THRESHOLD, FLAG_NEAR_TIE = 8, 16, 32
PAGED_BAD_LEN, PAGED_BAD_PAGE, PAGED_BAD_ROWS = 1, 2, 4        # bits of a paged cache's status word

EXPORTS = ["lsp_workspace_bytes", "lsp_kv_cache_bytes", "lsp_init", "lsp_set_sched", "lsp_set_option",
           "lsp_begin", "lsp_denoise_step", "lsp_commit", "lsp_generate", "lsp_generate_host", "lsp_active", "lsp_score_rows",
           "lsp_get_scores", "lsp_head_scan", "lsp_scan", "lsp_op_linear", "lsp_op_attention", "lsp_last_timing", "lsp_get_counters", "lsp_reset_counters",
           "lsp_linear_static", "lsp_paged_append", "lsp_paged_attention_workspace", "lsp_paged_attention",
           "lsp_paged_evict_workspace", "lsp_paged_evict", "lsp_last_error", "lsp_destroy"]


class LSPError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"lsp error {code}: {msg}")
        self.code = code


class ModelCfg(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab")] + \
               [("rms_eps", C.c_float), ("rope_theta", C.c_float), ("dtype", C.c_int), ("mask_id", C.c_int)]


class SchedCfgC(C.Structure):
    _fields_ = [("score", C.c_int), ("mode", C.c_int), ("tau", C.c_float), ("alpha", C.c_float), ("beta", C.c_float),
                ("l_min", C.c_int), ("snap_window", C.c_int), ("fixed_k", C.c_int), ("delim_bitmap", C.c_void_p),
                ("exclude_mask_logit", C.c_int), ("flag_tol", C.c_float), ("tie_tol", C.c_float), ("topology", C.c_int)]


class WeightsC(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("final_norm", C.c_void_p), ("w_head", C.c_void_p)] + \
               [(n, C.POINTER(C.c_void_p)) for n in ("attn_norm", "w_qkv", "w_o", "ffn_norm", "w_gate", "w_up", "w_down")]


class StepRec(C.Structure):
    _fields_ = [("step", C.c_int), ("n_before", C.c_int), ("rows", C.c_int), ("l_run", C.c_int), ("l_commit", C.c_int),
                ("tau_used", C.c_float), ("flags", C.c_uint), ("ms", C.c_float), ("flips", C.c_int), ("flip_base", C.c_int)]


class PagedKV(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_table", C.c_void_p), ("status", C.c_void_p),
                ("page_stride", C.c_longlong), ("row_stride", C.c_longlong), ("head_stride", C.c_longlong)] + \
               [(n, C.c_int) for n in ("n_pages", "page_size", "max_pages", "batch", "n_kv_heads", "head_dim", "dtype")]


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2603_05454_b200.build` "
                          "(there is no CPU or PyTorch fallback)")
    l = C.CDLL(_LIB_PATH)
    l.lsp_workspace_bytes.restype = C.c_size_t
    l.lsp_workspace_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int, C.c_int]
    l.lsp_kv_cache_bytes.restype = C.c_size_t
    l.lsp_kv_cache_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int, C.c_int]
    l.lsp_init.argtypes = [C.POINTER(C.c_void_p), C.POINTER(ModelCfg), C.POINTER(SchedCfgC), C.POINTER(WeightsC),
                           C.c_void_p, C.c_void_p, C.c_size_t, C.c_int, C.c_int, C.c_void_p]
    l.lsp_set_sched.argtypes = [C.c_void_p, C.POINTER(SchedCfgC)]
    l.lsp_set_option.argtypes = [C.c_void_p, C.c_int, C.c_int]
    l.lsp_debug_set.argtypes = [C.c_void_p, C.c_int, C.c_int]      # internal (csrc/lsp_tuning.h), not in EXPORTS
    l.lsp_debug_wait_selftest.argtypes = [C.c_void_p, C.c_int]
    l.lsp_begin.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int]
    l.lsp_denoise_step.argtypes = [C.c_void_p, C.POINTER(StepRec)]
    l.lsp_commit.argtypes = [C.c_void_p, C.c_void_p]
    l.lsp_generate.argtypes = [C.c_void_p, C.POINTER(StepRec), C.c_int, C.POINTER(C.c_int)]
    l.lsp_generate_host.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                    C.POINTER(StepRec), C.c_int, C.POINTER(C.c_int)]
    l.lsp_active.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int)]
    l.lsp_score_rows.argtypes = [C.c_void_p]
    l.lsp_get_scores.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    l.lsp_head_scan.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int] + [C.c_void_p] * 4
    l.lsp_scan.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int] + [C.c_void_p] * 4
    l.lsp_op_linear.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int]
    l.lsp_op_attention.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_int]
    l.lsp_last_timing.argtypes = [C.c_void_p, C.c_void_p]
    l.lsp_get_counters.argtypes = [C.c_void_p, C.c_void_p]
    l.lsp_reset_counters.argtypes = [C.c_void_p]
    l.lsp_linear_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_char_p,
                                    C.c_size_t]
    pkv, vp, i, ll, sz, cs = C.POINTER(PagedKV), C.c_void_p, C.c_int, C.c_longlong, C.c_size_t, C.c_char_p
    l.lsp_paged_append.argtypes = [pkv, vp, vp, ll, vp, vp, i, i, vp, vp, vp, vp, vp, vp, cs, sz]
    l.lsp_paged_attention_workspace.restype = sz
    l.lsp_paged_attention_workspace.argtypes = [pkv, i, i, i]
    l.lsp_paged_attention.argtypes = [pkv, vp, ll, i, vp, vp, i, i, C.c_float, vp, ll, vp, vp, vp, vp, sz, vp, cs, sz]
    l.lsp_paged_evict_workspace.restype = sz
    l.lsp_paged_evict_workspace.argtypes = [pkv, i]
    l.lsp_paged_evict.argtypes = [pkv, vp, vp, vp, vp, i, i, i, vp, vp, vp, vp, sz, vp, cs, sz]
    l.lsp_last_error.restype = C.c_char_p
    l.lsp_last_error.argtypes = [C.c_void_p]
    l.lsp_destroy.argtypes = [C.c_void_p]
    return l


lib = _load()


@dataclass
class SchedCfg:
    score: int = 0            # 0 = max-prob, 1 = logit margin
    mode: int = 0             # 0 fixed tau, 1 adaptive, 2 fixed-k
    tau: float = 0.9
    alpha: float = 0.25
    beta: float = 0.50
    l_min: int = 1
    snap_window: int = 16
    fixed_k: int = 1
    delim_bitmap: Optional[torch.Tensor] = None   # uint8 CUDA tensor, vocab bits
    exclude_mask_logit: int = 1
    flag_tol: float = 0.0
    tie_tol: float = 0.0
    topology: int = 0         # 0 prefix (LSP), 1 scattered acceptance (baseline)

    def to_c(self) -> SchedCfgC:
        p = self.delim_bitmap.data_ptr() if self.delim_bitmap is not None else None
        return SchedCfgC(self.score, self.mode, self.tau, self.alpha, self.beta, self.l_min, self.snap_window,
                         self.fixed_k, p, self.exclude_mask_logit, self.flag_tol, self.tie_tol, self.topology)


def _ptr_array(tensors: Sequence[torch.Tensor]):
    arr = (C.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])
    return arr


class LSPDecoder:
    """Owns the device buffers (allocated through torch) and a library context.

    shape: any object with the fields of lsp_model_cfg (n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ffn,
    vocab, rms_eps, rope_theta, dtype in {"fp32","bf16"}, mask_id).
    weights: dict with CUDA tensors embed, w_head, final_norm and a list "layers" of dicts with attn_norm, w_q,
    w_k, w_v (or w_qkv), w_o, ffn_norm, w_gate, w_up, w_down; linear weights are [out_features, in_features].
    """

    def __init__(self, shape, weights, sched: SchedCfg, max_batch: int, max_len: int, device="cuda:0", stream=None):
        self.device = torch.device(device)
        self.shape = shape
        self.tdtype = torch.float32 if shape.dtype == "fp32" else torch.bfloat16
        self.mc = ModelCfg(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads, shape.head_dim,
                           shape.d_ffn, shape.vocab, shape.rms_eps, shape.rope_theta,
                           0 if shape.dtype == "fp32" else 1, shape.mask_id)
        self.max_batch, self.max_len = max_batch, max_len
        ws = lib.lsp_workspace_bytes(C.byref(self.mc), max_batch, max_len)
        kv = lib.lsp_kv_cache_bytes(C.byref(self.mc), max_batch, max_len)
        if ws == 0 or kv == 0:
            raise LSPError(-2, "unsupported model shape")
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=self.device)
        self.kv_cache = torch.zeros(kv, dtype=torch.uint8, device=self.device)
        self._keep = []
        layers = []
        for lw in weights["layers"]:
            lw = dict(lw)
            if "w_qkv" not in lw:
                lw["w_qkv"] = torch.cat([lw["w_q"], lw["w_k"], lw["w_v"]], dim=0).contiguous()
            layers.append(lw)
        self._layers = layers
        self._w = weights
        names = ("attn_norm", "w_qkv", "w_o", "ffn_norm", "w_gate", "w_up", "w_down")
        arrs = {n: _ptr_array([lw[n] for lw in layers]) for n in names}
        self._keep.append(arrs)
        wc = WeightsC(weights["embed"].data_ptr(), weights["final_norm"].data_ptr(), weights["w_head"].data_ptr(),
                      *[C.cast(arrs[n], C.POINTER(C.c_void_p)) for n in names])
        self.sched = sched
        sc = sched.to_c()
        self.stream = stream
        sptr = stream.cuda_stream if stream is not None else torch.cuda.current_stream(self.device).cuda_stream
        self._h = C.c_void_p()
        with torch.cuda.device(self.device):
            rc = lib.lsp_init(C.byref(self._h), C.byref(self.mc), C.byref(sc), C.byref(wc), self.kv_cache.data_ptr(),
                              self.workspace.data_ptr(), ws, max_batch, max_len, sptr)
        if rc != 0:
            raise LSPError(rc, "lsp_init failed")
        self.batch = 0

    # -- helpers
    def _check(self, rc):
        if rc != 0:
            raise LSPError(rc, lib.lsp_last_error(self._h).decode())

    def close(self):
        if self._h:
            lib.lsp_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def layer_weights(self):
        """Per-layer weight tensors as the library holds them (w_qkv is the packed [q; k; v] projection)."""
        return self._layers

    def set_sched(self, sched: SchedCfg):
        self.sched = sched
        sc = sched.to_c()
        self._check(lib.lsp_set_sched(self._h, C.byref(sc)))

    def set_option(self, key: int, value: int):
        self._check(lib.lsp_set_option(self._h, key, value))

    def debug_set(self, key: int, value: int):
        """Internal tuning and benchmark knobs (csrc/lsp_tuning.h); not part of the public interface."""
        self._check(lib.lsp_debug_set(self._h, key, value))

    def wait_selftest(self, limit_us: int = 200):
        """Internal (csrc/lsp_tuning.h): lets a bounded device-side wait run out; raises LSPError(-6)."""
        self._check(lib.lsp_debug_wait_selftest(self._h, limit_us))

    # -- Algorithm 1
    def begin(self, tokens: torch.Tensor, prompt_len, gen_len):
        assert tokens.dtype == torch.int32 and tokens.is_cuda and tokens.dim() == 2 and tokens.is_contiguous()
        batch = tokens.shape[0]
        pl = np.ascontiguousarray(prompt_len, dtype=np.int32)
        gl = np.ascontiguousarray(gen_len, dtype=np.int32)
        if pl.shape != (batch,) or gl.shape != (batch,):
            raise ValueError(f"prompt_len and gen_len need one entry per row of tokens ({batch})")
        self._check(lib.lsp_begin(self._h, tokens.data_ptr(), tokens.shape[1], pl.ctypes.data, gl.ctypes.data, batch))
        self.tokens = tokens          # the library state changed only now (a rejected call leaves the old decode in place)
        self.batch = batch

    def denoise_step(self):
        recs = (StepRec * self.batch)()
        self._check(lib.lsp_denoise_step(self._h, recs))
        return [_rec(r) for r in recs]

    def commit(self, L=None):
        if L is None:
            self._check(lib.lsp_commit(self._h, None))
        else:
            a = np.ascontiguousarray(L, dtype=np.int32)
            if a.shape != (self.batch,):
                raise ValueError(f"L needs one entry per sequence ({self.batch})")
            self._check(lib.lsp_commit(self._h, a.ctypes.data))

    def generate(self, max_recs: int = 0):
        n = C.c_int(0)
        recs = (StepRec * max_recs)() if max_recs else None
        self._check(lib.lsp_generate(self._h, recs, max_recs, C.byref(n)))
        out = [_rec(r) for r in recs][: n.value * self.batch] if recs is not None else []
        return n.value, out

    def generate_host(self, tokens_dev: torch.Tensor, tokens_in: torch.Tensor, tokens_out: torch.Tensor, prompt_len,
                      gen_len, max_recs: int = 0):
        """Algorithm 1 from host memory: tokens_in / tokens_out are CPU int32 tensors [batch, stride] (pinned or
        not), tokens_dev the device buffer of the same shape the decode runs in."""
        assert tokens_dev.dtype == torch.int32 and tokens_dev.is_cuda and tokens_dev.is_contiguous()
        for t in (tokens_in, tokens_out):
            assert t.dtype == torch.int32 and not t.is_cuda and t.is_contiguous() and t.shape == tokens_dev.shape
        batch = tokens_dev.shape[0]
        pl = np.ascontiguousarray(prompt_len, dtype=np.int32)
        gl = np.ascontiguousarray(gen_len, dtype=np.int32)
        if pl.shape != (batch,) or gl.shape != (batch,):
            raise ValueError(f"prompt_len and gen_len need one entry per row of tokens ({batch})")
        self.tokens = tokens_dev
        self.batch = batch
        n = C.c_int(0)
        recs = (StepRec * max_recs)() if max_recs else None
        self._check(lib.lsp_generate_host(self._h, tokens_dev.data_ptr(), tokens_dev.shape[1], tokens_in.data_ptr(),
                                          tokens_out.data_ptr(), pl.ctypes.data, gl.ctypes.data, self.batch, recs,
                                          max_recs, C.byref(n)))
        out = [_rec(r) for r in recs][: n.value * self.batch] if recs is not None else []
        return n.value, out

    def active(self):
        a = np.zeros(self.batch, dtype=np.int32)
        u = C.c_int(0)
        self._check(lib.lsp_active(self._h, a.ctypes.data, C.byref(u)))
        return a, u.value

    def scores(self):
        n = lib.lsp_score_rows(self._h)
        y = np.zeros(n, dtype=np.int32)
        p = np.zeros(n, dtype=np.float32)
        m = np.zeros(n, dtype=np.float32)
        self._check(lib.lsp_get_scores(self._h, y.ctypes.data, p.ctypes.data, m.ctypes.data))
        return y, p, m

    def _scan_out(self, batch):
        return (np.zeros(batch, np.int32), np.zeros(batch, np.int32), np.zeros(batch, np.uint32), np.zeros(batch, np.float32))

    def head_scan(self, hidden: torch.Tensor, seq_offsets):
        assert hidden.is_cuda and hidden.is_contiguous() and hidden.dtype == self.tdtype
        so = np.ascontiguousarray(seq_offsets, dtype=np.int32)
        batch = len(so) - 1
        lr, lc, fl, tu = self._scan_out(batch)
        self._check(lib.lsp_head_scan(self._h, hidden.data_ptr(), so.ctypes.data, batch, lr.ctypes.data, lc.ctypes.data,
                                      fl.ctypes.data, tu.ctypes.data))
        return dict(L_run=lr, L_commit=lc, flags=fl, tau_used=tu)

    def scan(self, score: torch.Tensor, yhat: torch.Tensor, margin: Optional[torch.Tensor], seq_offsets):
        assert score.dtype == torch.float32 and yhat.dtype == torch.int32 and score.is_cuda and yhat.is_cuda
        so = np.ascontiguousarray(seq_offsets, dtype=np.int32)
        batch = len(so) - 1
        lr, lc, fl, tu = self._scan_out(batch)
        self._check(lib.lsp_scan(self._h, score.data_ptr(), yhat.data_ptr(), margin.data_ptr() if margin is not None else None,
                                 so.ctypes.data, batch, lr.ctypes.data, lc.ctypes.data, fl.ctypes.data, tu.ctypes.data))
        return dict(L_run=lr, L_commit=lc, flags=fl, tau_used=tu)

    def op_linear(self, op: int, A: torch.Tensor, W: torch.Tensor, W2: Optional[torch.Tensor], out: torch.Tensor):
        M, K = A.shape
        N = W.shape[0]
        self._check(lib.lsp_op_linear(self._h, op, A.data_ptr(), W.data_ptr(), W2.data_ptr() if W2 is not None else None,
                                      out.data_ptr(), M, N, K))
        return out

    def op_attention(self, layer: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, out: torch.Tensor,
                     cache_len, rows):
        """One layer's suffix-over-prefix attention on packed rows; the cached K/V are read from kv_view()."""
        cl = np.ascontiguousarray(cache_len, dtype=np.int32)
        rw = np.ascontiguousarray(rows, dtype=np.int32)
        assert cl.shape == rw.shape and q.shape[0] == int(rw.sum()) == k_new.shape[0] == v_new.shape[0] == out.shape[0]
        for t in (q, k_new, v_new, out):
            assert t.is_cuda and t.is_contiguous() and t.dtype == self.tdtype
        self._check(lib.lsp_op_attention(self._h, layer, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), out.data_ptr(),
                                         cl.ctypes.data, rw.ctypes.data, len(cl)))
        return out

    def last_timing(self):
        a = np.zeros(8, dtype=np.float32)
        self._check(lib.lsp_last_timing(self._h, a.ctypes.data))
        return a

    def counters(self):
        a = np.zeros(18, dtype=np.float64)
        self._check(lib.lsp_get_counters(self._h, a.ctypes.data))
        return dict(zip(("launches", "gemm_bytes", "gemm_flops", "attn_bytes", "append_bytes", "head_bytes",
                         "head_flops", "steps", "launches_misc", "launches_gemm", "launches_attn", "launches_head",
                         "launches_scan", "launches_commit", "attn_flops", "tokens", "attn_kernel", "attn_cluster"),
                        a.tolist()))

    def reset_counters(self):
        self._check(lib.lsp_reset_counters(self._h))

    # views of the caller-visible state (device memory owned here)
    def kv_view(self):
        s = self.shape
        return self.kv_cache.view(self.tdtype).view(s.n_layers, 2, self.max_batch, self.max_len, s.n_kv_heads, s.head_dim)


def linear_static(A: torch.Tensor, W: torch.Tensor, out: torch.Tensor, stream=None):
    """out = A W^T through lsp_linear_static: no context, no workspace; the library's static scratch is used.
    A [M, K], W [N, K], out [M, N]: contiguous bfloat16 CUDA tensors on the current device."""
    M, K = A.shape
    N = W.shape[0]
    sptr = stream.cuda_stream if stream is not None else torch.cuda.current_stream(A.device).cuda_stream
    buf = C.create_string_buffer(256)
    with torch.cuda.device(A.device):
        rc = lib.lsp_linear_static(A.data_ptr(), W.data_ptr(), out.data_ptr(), M, N, K, sptr, buf, len(buf))
    if rc != 0:
        raise LSPError(rc, buf.value.decode())
    return out


class PagedKVCache:
    """One layer's keys and values in pages (lsp_paged_*): append, attention of new rows, eviction by gathered weight.

    k_pool, v_pool: [n_pages, page_size, n_kv_heads, head_dim] CUDA tensors (bfloat16 or float32) with the same strides, heads
    contiguous; any view with 16-byte strides will do, a decoder's own planes among them.  page_table: int32 CUDA tensor [batch, max_pages],
    contiguous; without it page p of sequence b is page b * max_pages + p (batch then tells max_pages = n_pages // batch).
    All tensors are borrowed; page_table may be rewritten between calls.  The object owns the status word that check() reads and the workspace: for any
    eviction, and for attention of at most n_rows packed rows, by default max_rows for every sequence; with `weights` for attention that gathers
    them, 4 bytes for every row, query head and slot of a sequence's pages (16 x 8 rows of 32 heads over 32768 slots: 0.5 GB).

    Every call enqueues on the current stream of the pools' device, or on `stream`.  It costs the host 8 to 13 us: capture a step's calls into a graph where
    they take less on the device.  Calls of one object must not overlap on the device: give each stream, and each captured graph that may run
    beside others, an object of its own over the same pools.  An object is ready for any stream once it is made (the constructor waits for its
    stream).  One made in a stream capture belongs to that graph: its calls are those of the capture, and others raise.  It may be dropped while calls
    on torch's streams are still running; keep it for those on an external stream, and for the replays of a graph that holds its calls.
    """

    def __init__(self, k_pool: torch.Tensor, v_pool: torch.Tensor, page_table: Optional[torch.Tensor] = None, *, n_heads: int,
                 batch: Optional[int] = None, max_rows: int = 1, n_rows: Optional[int] = None, weights: bool = False):
        if k_pool.dim() != 4 or v_pool.shape != k_pool.shape or v_pool.stride() != k_pool.stride() or v_pool.dtype != k_pool.dtype:
            raise ValueError("k_pool and v_pool need one shape [n_pages, page_size, n_kv_heads, head_dim], one type and one layout")
        if not (k_pool.is_cuda and v_pool.device == k_pool.device) or k_pool.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("the pools must be float32 or bfloat16 tensors of one CUDA device")
        if k_pool.shape[3] > 1 and k_pool.stride(3) != 1:
            raise ValueError("the elements of a head must be contiguous")
        n_pages, page_size, n_kv, dh = k_pool.shape
        self.device, self.dtype, self._index = k_pool.device, k_pool.dtype, k_pool.get_device()
        if page_table is not None:
            if page_table.dim() != 2:
                raise ValueError("page_table must be [batch, max_pages]")
            self._tensor("page_table", page_table, torch.int32, page_table.shape)
            self.batch, self.max_pages = page_table.shape
            if batch not in (None, self.batch):
                raise ValueError(f"page_table has {self.batch} sequences, not {batch}")
        else:
            self.batch = batch or 1
            self.max_pages = n_pages // self.batch
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv, dh
        self.max_rows = max_rows
        self.capacity = self.max_pages * page_size
        self._per_seq, self._per_slot = torch.Size((self.batch,)), torch.Size((self.batch, n_kv, self.capacity))
        self._offsets = torch.Size((self.batch + 1,))
        self._q_width, self._kv_width, self._scale = n_heads * dh, n_kv * dh, dh ** -0.5
        self.k_pool, self.v_pool, self.page_table = k_pool, v_pool, page_table
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._kv = PagedKV(k_pool.data_ptr(), v_pool.data_ptr(), page_table.data_ptr() if page_table is not None else None,
                           self.status.data_ptr(), k_pool.stride(0), k_pool.stride(1), k_pool.stride(2), n_pages, page_size,
                           self.max_pages, self.batch, n_kv, dh, 0 if k_pool.dtype == torch.float32 else 1)
        self._ref = C.byref(self._kv)
        self._err = C.create_string_buffer(256)
        rows = self.batch * max_rows if n_rows is None else n_rows
        need = lib.lsp_paged_attention_workspace(self._ref, n_heads, rows, int(weights))
        if need == 0:
            # the library's own words for what is wrong with the description
            self._check(lib.lsp_paged_evict(self._ref, None, None, None, None, 1, 0, 0, None, None, None, None, 0, None, self._err, 256))
        # (an eviction moves most where half of the slots go)
        need = max(need, lib.lsp_paged_evict_workspace(self._ref, max(1, self.capacity // 2)))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
        self.workspace[:4096].zero_()          # arrival counters
        self._ws, self._ws_bytes = self.workspace.data_ptr(), need
        # Counters and status are clear ahead of any call, whatever stream it takes: waited for here; in a capture, which forbids that, by each
        # further stream of it.
        made_on = torch.cuda.current_stream(self.device)
        self._streams, self._cleared = {made_on.cuda_stream}, None
        with torch.cuda.device(self.device):
            if torch.cuda.is_current_stream_capturing():
                self._cleared = torch.cuda.Event()
                self._cleared.record(made_on)
            else:
                made_on.synchronize()

    # (the checks run with every call of a few microseconds: each is one comparison of what torch hands out as it is)
    def _tensor(self, name, t, dtype, shape):
        """Address of a contiguous tensor; None for None."""
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self._index or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {list(shape)} on {self.device}")
        return t.data_ptr()

    def _rows(self, name, t, width):
        """Address, count and distance of packed rows [n_rows, width]."""
        shape, stride = t.shape, t.stride()
        if t.dtype is not self.dtype or len(shape) != 2 or shape[1] != width or stride[1] != 1 or t.get_device() != self._index:
            raise ValueError(f"{name} must be a {self.dtype} tensor of shape [rows, {width}] on {self.device}, elements of a row contiguous")
        return t.data_ptr(), shape[0], stride[0] if shape[0] > 1 else max(stride[0], width)

    def _row_off(self, row_off, n_rows, max_rows):
        """Address of the offsets and the bound of a sequence's rows."""
        if row_off is not None:
            return self._tensor("row_off", row_off, torch.int32, self._offsets), max_rows or self.max_rows
        if n_rows % self.batch or n_rows == 0:
            raise ValueError(f"without row_off every one of the {self.batch} sequences has as many rows: {n_rows} rows do not divide")
        return None, n_rows // self.batch

    def _check(self, rc):
        if rc != 0:
            raise LSPError(rc, self._err.value.decode())

    def _meet(self, stream, sptr):
        """Ahead of the first call on a stream that the object was not made on."""
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        if self._cleared is not None:
            stream.wait_event(self._cleared)
        # The allocator gives the object's memory out again only behind what the stream has been handed by then.  (Not a stream that torch did not
        # make, whose id is its address: it may be gone by then, and the allocator would still ask it.)
        if isinstance(stream, torch.cuda.Stream) and (sptr == 0 or stream.stream_id != sptr):
            self.workspace.record_stream(stream)
            self.status.record_stream(stream)
        self._streams.add(sptr)

    def _call(self, stream, fn, *args):
        sptr = torch._C._cuda_getCurrentRawStream(self._index) if stream is None else stream.cuda_stream
        if sptr not in self._streams:
            self._meet(stream, sptr)
        if torch._C._cuda_getDevice() == self._index:
            rc = fn(self._ref, *args, sptr, self._err, 256)
        else:
            with torch.cuda.device(self.device):
                rc = fn(self._ref, *args, sptr, self._err, 256)
        if rc != 0:
            self._check(rc)

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor, lens: torch.Tensor, lens_out: torch.Tensor, *, row_off=None,
               max_rows: Optional[int] = None, weights=None, pos=None, seen=None, seen_out=None, stream=None):
        """Writes packed rows k_new, v_new [n_rows, n_kv_heads * head_dim] behind the lens[b] cached ones (lsp_paged_append)."""
        kp, n, ld = self._rows("k_new", k_new, self._kv_width)
        vp, nv, ldv = self._rows("v_new", v_new, self._kv_width)
        if nv != n or ldv != ld:
            raise ValueError("k_new and v_new need one shape and one row stride")
        off, most = self._row_off(row_off, n, max_rows)
        i32, b, tensor = torch.int32, self._per_seq, self._tensor
        self._call(stream, lib.lsp_paged_append, kp, vp, ld, tensor("lens", lens, i32, b), off, most, n, tensor("lens_out", lens_out, i32, b),
                   tensor("weights", weights, torch.float32, self._per_slot), tensor("pos", pos, i32, self._per_slot), tensor("seen", seen, i32, b),
                   tensor("seen_out", seen_out, i32, b))
        return lens_out

    def attention(self, q: torch.Tensor, lens: torch.Tensor, out: torch.Tensor, *, row_off=None, max_rows: Optional[int] = None,
                  scale: Optional[float] = None, lse=None, weights_in=None, weights_out=None, stream=None):
        """Attention of packed rows q [n_rows, n_heads * head_dim] over their sequences' slots (lsp_paged_attention); scale: 1 / sqrt(head_dim)."""
        qp, n, ldq = self._rows("q", q, self._q_width)
        op, no, ldo = self._rows("out", out, self._q_width)
        if no != n:
            raise ValueError(f"q has {n} rows, out {no}")
        off, most = self._row_off(row_off, n, max_rows)
        f32, tensor = torch.float32, self._tensor
        self._call(stream, lib.lsp_paged_attention, qp, ldq, self.n_heads, tensor("lens", lens, torch.int32, self._per_seq), off, most, n,
                   self._scale if scale is None else scale, op, ldo, None if lse is None else tensor("lse", lse, f32, (n, self.n_heads)),
                   tensor("weights_in", weights_in, f32, self._per_slot), tensor("weights_out", weights_out, f32, self._per_slot),
                   self._ws, self._ws_bytes)
        return out

    def evict(self, weights: torch.Tensor, lens: torch.Tensor, budget: int, weights_out: torch.Tensor, lens_out: torch.Tensor, *,
              n_sink: int = 0, n_recent: int = 0, pos=None, pos_out=None, seen=None, stream=None):
        """Thins every sequence to at most budget slots per KV head (lsp_paged_evict).  seen: positions of each sequence so far (the append's seen_out);
        needed with n_recent for a sequence that was thinned before, since without it the number of slots is taken, and positions lie beyond that."""
        i32, f32, b, slots, tensor = torch.int32, torch.float32, self._per_seq, self._per_slot, self._tensor
        self._call(stream, lib.lsp_paged_evict, tensor("weights", weights, f32, slots), tensor("pos", pos, i32, slots), tensor("lens", lens, i32, b),
                   tensor("seen", seen, i32, b), budget, n_sink, n_recent, tensor("weights_out", weights_out, f32, slots),
                   tensor("pos_out", pos_out, i32, slots), tensor("lens_out", lens_out, i32, b), self._ws, self._ws_bytes)
        return lens_out

    def check(self):
        """Waits for the device and raises LSPError (LSP_ERR_STATE) with the status bits if a call since the last check met lengths, table
        entries or row offsets out of range; clears them."""
        torch.cuda.synchronize(self.device)
        bits = int(self.status.item())
        if bits:
            self.status.zero_()
            torch.cuda.synchronize(self.device)        # (ahead of the next call, on whatever stream)
            words = [w for bit, w in ((PAGED_BAD_LEN, "a length outside the sequence's pages"), (PAGED_BAD_PAGE, "a table entry outside the pool"),
                                      (PAGED_BAD_ROWS, "row offsets out of range")) if bits & bit]
            raise LSPError(-4, f"paged cache: {', '.join(words)} (status {bits})")


def _rec(r: StepRec):
    return dict(step=r.step, n_before=r.n_before, rows=r.rows, L_run=r.l_run, L_commit=r.l_commit,
                tau_used=r.tau_used, flags=r.flags, ms=r.ms, flips=r.flips, flip_base=r.flip_base)
