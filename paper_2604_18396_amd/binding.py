"""Thin ctypes binding of libriver.so (include/river.h).

Argument marshalling only: every step of the decode path runs in the library's HIP
kernels.  torch is used for device memory and the stream.  If the library has not
been built, loading raises: there is no fallback of any kind.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os

import numpy as np
import torch

from . import build as _build
from .configs import MATRICES, ModelConfig

RIVER_OK, RIVER_EINVAL, RIVER_ENOSPC, RIVER_ESTATE, RIVER_EHIP = 0, -1, -2, -3, -4
EXEC_KERNELS, EXEC_PERSISTENT = 0, 1
DBG_HIDDEN, DBG_LOGITS, DBG_KCACHE, DBG_VCACHE, DBG_TRACE, DBG_BATCH_HIDDEN, DBG_BATCH_LOGITS = 0, 1, 2, 3, 4, 5, 6
EXIT_PER_SEQUENCE, EXIT_BATCH_MIN = 0, 1

EXPORTS = ("river_quantize_w4", "river_workspace_bytes", "river_create", "river_create_static", "river_prefill",
           "river_decode_step", "river_decode_batch", "river_read_batch_records", "river_read_records",
           "river_rewind", "river_position", "river_seq_position",
           "river_get_debug", "river_fill_cache", "river_last_error", "river_destroy",
           "river_rope_frequencies", "river_rope_store", "river_paged_attention_workspace", "river_paged_attention",
           "river_copy_pages", "river_pool_create", "river_pool_destroy", "river_pool_extend", "river_pool_fork",
           "river_pool_rewind", "river_pool_trim", "river_pool_compact", "river_pool_flush", "river_pool_length",
           "river_pool_free_pages", "river_pool_row", "river_save_pages", "river_load_pages",
           "river_build_batch", "river_store_slots", "river_prefix_attention_workspace", "river_prefix_attention")
TICKETS = 1024
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}
ROPE_HIGH = {"bands": 4.0, "ramp": 32.0}        # turns from which on a frequency stays as it is, where models do not say otherwise


class RiverError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"river error {code}: {msg}")
        self.code = code


class river_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab")] + \
               [("rope_base", C.c_float), ("rms_eps", C.c_float), ("dtype", C.c_int32),
                ("max_batch", C.c_int32), ("max_seq", C.c_int32), ("min_exit_layer", C.c_int32),
                ("tau", C.c_float), ("river_bits", C.c_int32), ("river_group", C.c_int32),
                ("exec_mode", C.c_int32), ("spin_limit", C.c_int32), ("prefill_gemm_min_tokens", C.c_int32),
                ("batch_exit_rule", C.c_int32), ("kv_dtype", C.c_int32)]


_PP = C.POINTER(C.c_void_p)


class river_weights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)] + \
               [(n, _PP) for n in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up",
                                   "w_down")]


class river_qweights(C.Structure):
    _fields_ = [("codes", _PP * 7), ("scale", _PP * 7), ("zero", _PP * 7)]


class river_pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64), ("page_stride", C.c_int64)] + \
               [(n, C.c_int32) for n in ("n_layers", "n_pages", "page_size", "n_kv_heads", "head_dim", "dtype", "kv_dtype")]


class river_batch(C.Structure):
    _fields_ = [("table", C.c_void_p), ("lens", C.c_void_p), ("q_start", C.c_void_p)] + \
               [(n, C.c_int32) for n in ("n_seq", "n_tokens", "max_pages", "table_stride", "max_new", "max_len")]


class river_prefixes(C.Structure):
    _fields_ = [("table", C.c_void_p), ("lens", C.c_void_p), ("seq_start", C.c_void_p)] + \
               [(n, C.c_int32) for n in ("n_groups", "max_pages", "table_stride", "max_len", "max_seqs")]


class river_tables(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("table", "lens", "lens_out", "free_pages", "n_free", "n_free_out", "n_shared")] + \
               [(n, C.c_int32) for n in ("n_seq", "max_pages", "table_stride", "n_pages", "page_size")]


class river_rope(C.Structure):
    _fields_ = [("inv_freq", C.c_void_p), ("rot_dim", C.c_int32), ("layout", C.c_int32), ("mscale", C.c_float)]


_lib = None


def load():
    """Load libriver.so; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = os.environ.get("RIVER_LIB_PATH", _build.LIB)      # e.g. the diagnostics build
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it first "
                          "(python -c 'import __graft_entry__ as g; g.build()')")
    L = C.CDLL(path)
    L.river_quantize_w4.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_int32,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    L.river_workspace_bytes.argtypes = [C.POINTER(river_config)]
    L.river_workspace_bytes.restype = C.c_size_t
    L.river_create.argtypes = [C.POINTER(river_config), C.POINTER(river_weights),
                               C.POINTER(river_qweights), C.c_void_p, C.c_size_t, C.c_void_p,
                               C.POINTER(C.c_void_p)]
    L.river_create_static.argtypes = L.river_create.argtypes
    L.river_prefill.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_int32,
                                C.POINTER(C.c_int32), C.c_void_p]
    L.river_decode_step.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                    C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.c_void_p]
    L.river_decode_batch.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_void_p]
    L.river_read_batch_records.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
    L.river_seq_position.argtypes = [C.c_void_p, C.c_int32]
    L.river_read_records.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
    L.river_rewind.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
    L.river_position.argtypes = [C.c_void_p]
    L.river_get_debug.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t]
    L.river_fill_cache.argtypes = [C.c_void_p, C.c_int32]
    L.river_last_error.argtypes = [C.c_void_p]
    L.river_last_error.restype = C.c_char_p
    L.river_destroy.argtypes = [C.c_void_p]
    i32, i64, f64, ptr, pages, batch = C.c_int32, C.c_int64, C.c_double, C.c_void_p, C.POINTER(river_pages), C.POINTER(river_batch)
    L.river_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, ptr, C.POINTER(C.c_float)]
    L.river_rope_store.argtypes = [pages, i32, batch, C.POINTER(river_rope), i32, ptr, i64, ptr, i64, ptr, i64, ptr, i64, ptr]
    L.river_paged_attention_workspace.argtypes = [pages, batch, i32, i32, i32, C.POINTER(C.c_size_t)]
    L.river_paged_attention.argtypes = [pages, i32, batch, i32, ptr, i64, C.c_float, i32, i32, ptr, i64, ptr, C.c_size_t, ptr, ptr]
    L.river_copy_pages.argtypes = [pages, ptr, ptr, i32, ptr]
    L.river_pool_create.argtypes = [i32, i32, i32, i32, C.POINTER(ptr)]
    for name, more in (("destroy", []), ("extend", [i32, i32]), ("fork", [i32, i32]), ("rewind", [i32, i32]), ("trim", [i32, i32, i32]),
                       ("compact", []), ("flush", [pages, ptr, ptr]), ("length", [i32]), ("free_pages", []), ("row", [i32, ptr])):
        getattr(L, "river_pool_" + name).argtypes = [ptr, *more]
    prefixes = C.POINTER(river_prefixes)
    L.river_build_batch.argtypes = [C.POINTER(river_tables), ptr, i32, ptr, ptr, ptr, ptr, ptr]
    L.river_store_slots.argtypes = [pages, i32, ptr, i32, ptr, i64, ptr, i64, ptr]
    L.river_prefix_attention_workspace.argtypes = [pages, batch, prefixes, i32, C.POINTER(C.c_size_t)]
    L.river_prefix_attention.argtypes = [pages, i32, batch, prefixes, i32, ptr, i64, C.c_float, ptr, i64, ptr, C.c_size_t, ptr, ptr]
    L.river_save_pages.argtypes = [ptr, i32, i32, i32, pages, ptr, i32]
    L.river_load_pages.argtypes = [ptr, i32, i32, i32, pages, ptr, i32]
    _lib = L
    return L


def default_exec_mode(cfg: ModelConfig) -> int:
    """One launch per token where the library offers it (bf16), else one launch per phase."""
    return EXEC_PERSISTENT if cfg.dtype == 1 else EXEC_KERNELS


def make_config(cfg: ModelConfig, exec_mode: int | None = None, spin_limit: int = 0,
                prefill_gemm_min_tokens: int = 0, max_batch: int = 1, batch_exit_rule: int = 0) -> river_config:
    if exec_mode is None:
        exec_mode = default_exec_mode(cfg)
    return river_config(cfg.n_layers, cfg.d_model, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim,
                        cfg.d_ffn, cfg.vocab, cfg.rope_base, cfg.rms_eps, cfg.dtype, max_batch, cfg.max_seq,
                        cfg.min_exit_layer, cfg.tau, 4, cfg.river_group, exec_mode, spin_limit,
                        prefill_gemm_min_tokens, batch_exit_rule, cfg.kv_dtype)


def _stream_ptr() -> int:
    return torch.cuda.current_stream().cuda_stream


def river_quantize_w4(w: torch.Tensor, group: int):
    """Device tensor [rows, cols] (fp32 / bf16) -> (codes u8 [rows, cols/2], scale, zero)."""
    assert w.is_cuda and w.is_contiguous() and w.dim() == 2
    rows, cols = w.shape
    gpr = -(-cols // group)
    codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device=w.device)
    scale = torch.empty((rows, gpr), dtype=w.dtype, device=w.device)
    zero = torch.empty((rows, gpr), dtype=w.dtype, device=w.device)
    dt = 1 if w.dtype == torch.bfloat16 else 0
    rc = load().river_quantize_w4(w.data_ptr(), rows, cols, group, dt, codes.data_ptr(),
                                  scale.data_ptr(), zero.data_ptr(), _stream_ptr())
    if rc:
        raise RiverError(rc, "river_quantize_w4")
    return codes, scale, zero


def upload_weights(weights: dict, device="cuda:0") -> dict:
    """CPU weight dict (inputs.make_weights) -> same structure on the device."""
    out = {k: weights[k].to(device) for k in ("tok_emb", "final_norm", "lm_head")}
    out["layers"] = [{k: v.to(device) for k, v in blk.items()} for blk in weights["layers"]]
    return out


def offload_backbone(dev_weights: dict, from_block: int) -> dict:
    """Backbone Offloading: the seven matrices of backbone blocks from_block+1..L (1-based: the
    blocks a token only reaches when its exit position exceeds from_block) are moved out of
    HBM into pinned host memory, which the GPU reads in place over the host link when a token
    does reach them; norm gains, embedding, head and the whole river stay in HBM.  Build the
    river first (quantize_river reads the matrices on the device).  Returns a new weight dict."""
    out = {k: dev_weights[k] for k in ("tok_emb", "final_norm", "lm_head")}
    out["layers"] = []
    for l, blk in enumerate(dev_weights["layers"]):
        if l < from_block:
            out["layers"].append(blk)
            continue
        nb = {}
        for k, v in blk.items():
            if k in MATRICES:
                host = torch.empty(v.shape, dtype=v.dtype, pin_memory=True)
                host.copy_(v)
                nb[k] = host
            else:
                nb[k] = v
        out["layers"].append(nb)
    torch.cuda.synchronize()
    return out


def quantize_river(cfg: ModelConfig, dev_weights: dict) -> list:
    """River construction on the device for every block (list of {name: (codes, scale, zero)})."""
    return [{m: river_quantize_w4(blk[m], cfg.river_group) for m in MATRICES}
            for blk in dev_weights["layers"]]


class River:
    """One decode context (river_create .. river_destroy)."""

    def __init__(self, cfg: ModelConfig, dev_weights: dict, dev_river: list | None,
                 exec_mode: int | None = None, spin_limit: int = 0, static_scratch: bool = False,
                 prefill_gemm_min_tokens: int = 0, max_batch: int = 1, batch_exit_rule: int = 0):
        """static_scratch=True goes through river_create_static (no device allocation inside
        the library: activations and barrier counters in the library's static device array)."""
        L = load()
        self.cfg = cfg
        self._c = make_config(cfg, exec_mode, spin_limit, prefill_gemm_min_tokens, max_batch, batch_exit_rule)
        self.max_batch = max_batch
        self._keep = [dev_weights, dev_river]
        n = cfg.n_layers
        w = river_weights()
        w.tok_emb = dev_weights["tok_emb"].data_ptr()
        w.final_norm = dev_weights["final_norm"].data_ptr()
        w.lm_head = dev_weights["lm_head"].data_ptr()
        for name in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down"):
            arr = (C.c_void_p * n)(*[blk[name].data_ptr() for blk in dev_weights["layers"]])
            self._keep.append(arr)
            setattr(w, name, C.cast(arr, _PP))
        q = None
        if dev_river is not None:
            q = river_qweights()
            for j, m in enumerate(MATRICES):
                for k, field in enumerate(("codes", "scale", "zero")):
                    arr = (C.c_void_p * n)(*[(r[m][k].data_ptr() if r is not None else None)
                                             for r in dev_river])
                    self._keep.append(arr)
                    getattr(q, field)[j] = C.cast(arr, _PP)
        nbytes = L.river_workspace_bytes(C.byref(self._c))
        if nbytes == 0:
            raise RiverError(RIVER_EINVAL, "invalid configuration")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev_weights["tok_emb"].device)
        self.workspace_bytes = nbytes
        self._stream = torch.cuda.current_stream()             # the context's, from now on
        h = C.c_void_p()
        create = L.river_create_static if static_scratch else L.river_create
        rc = create(C.byref(self._c), C.byref(w), C.byref(q) if q is not None else None,
                    self.workspace.data_ptr(), nbytes, self._stream.cuda_stream, C.byref(h))
        if rc:
            raise RiverError(rc, L.river_last_error(None).decode())
        self._h = h

    def _check(self, rc: int):
        if rc:
            raise RiverError(rc, load().river_last_error(self._h).decode())

    def close(self):
        if getattr(self, "_h", None):
            load().river_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def prefill(self, tokens, exit_layer: int | None = None, out_logits: torch.Tensor | None = None,
                seq: int = 0) -> int:
        """Prefill phase at the unified depth exit_layer (None: the full depth L).
        out_logits: optional device fp32 [vocab] tensor that receives the last position's logits.
        seq: the sequence of a batched context."""
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        out = C.c_int32()
        if out_logits is not None:
            assert out_logits.is_cuda and out_logits.dtype == torch.float32 and out_logits.is_contiguous()
            assert out_logits.numel() == self.cfg.vocab
        self._check(load().river_prefill(self._h, seq, t.ctypes.data, len(t),
                                         -1 if exit_layer is None else int(exit_layer), C.byref(out),
                                         out_logits.data_ptr() if out_logits is not None else None))
        return out.value

    def decode_step(self, token: int | None = None, forced_exit: int | None = None, sync: bool = True):
        """sync=True -> (next_token, exit_position, sims[L]); sync=False queues the step only."""
        tin = C.byref(C.c_int32(int(token))) if token is not None else None
        fe = C.byref(C.c_int32(int(forced_exit))) if forced_exit is not None else None
        if not sync:
            self._check(load().river_decode_step(self._h, tin, fe, None, None, None))
            return None
        tok, e = C.c_int32(), C.c_int32()
        sims = np.empty(self.cfg.n_layers, dtype=np.float32)
        self._check(load().river_decode_step(self._h, tin, fe, C.byref(tok), C.byref(e),
                                             sims.ctypes.data))
        return tok.value, e.value, sims

    def decode_batch(self, n_seq: int, tokens=None, forced_exits=None, sync: bool = True):
        """One step of a batched context.  sync=True -> (tokens[n], exit_positions[n], sims[n, L])."""
        tin = np.ascontiguousarray(tokens, dtype=np.int32) if tokens is not None else None
        fe = (np.ascontiguousarray([-1 if f is None else int(f) for f in forced_exits], dtype=np.int32)
              if forced_exits is not None else None)
        a = tin.ctypes.data if tin is not None else None
        b = fe.ctypes.data if fe is not None else None
        if not sync:
            self._check(load().river_decode_batch(self._h, n_seq, a, b, None, None, None))
            return None
        toks = np.empty(n_seq, dtype=np.int32)
        es = np.empty(n_seq, dtype=np.int32)
        sims = np.empty((n_seq, self.cfg.n_layers), dtype=np.float32)
        self._check(load().river_decode_batch(self._h, n_seq, a, b, toks.ctypes.data, es.ctypes.data,
                                              sims.ctypes.data))
        return toks, es, sims

    def read_batch_records(self, n_steps: int, n_seq: int):
        toks = np.empty((n_steps, n_seq), dtype=np.int32)
        es = np.empty((n_steps, n_seq), dtype=np.int32)
        self._check(load().river_read_batch_records(self._h, n_steps, n_seq, toks.ctypes.data, es.ctypes.data))
        return toks, es

    def seq_pos(self, seq: int) -> int:
        return load().river_seq_position(self._h, seq)

    def batch_hidden(self) -> np.ndarray:
        """[L+1, max_batch, d] hidden states of the last batched step."""
        out = np.empty((self.cfg.n_layers + 1, self.max_batch, self.cfg.d_model), dtype=np.float32)
        self._check(load().river_get_debug(self._h, DBG_BATCH_HIDDEN, out.ctypes.data, out.nbytes))
        return out

    def batch_logits(self) -> np.ndarray:
        out = np.empty((self.max_batch, self.cfg.vocab), dtype=np.float32)
        self._check(load().river_get_debug(self._h, DBG_BATCH_LOGITS, out.ctypes.data, out.nbytes))
        return out

    def save_pages(self, pages: "Pages", row: torch.Tensor, n: int, first: int = 0, seq: int = 0):
        """Positions first .. first + n - 1 of the sequence to the pages that `row` (device int32) names.  On the context's stream, behind
        what the current one has queued; what is queued there afterwards comes behind the call."""
        self._check_pages(pages, row)
        with self._in_order():
            self._check(load().river_save_pages(self._h, seq, first, n, pages.ref, row.data_ptr(), row.numel()))

    def load_pages(self, pages: "Pages", row: torch.Tensor, n: int, next_token: int, seq: int = 0):
        """Positions 0 .. n - 1 of the sequence from pages; next_token is what its next step consumes by default.  Streams as in
        save_pages."""
        self._check_pages(pages, row)
        with self._in_order():
            self._check(load().river_load_pages(self._h, seq, n, int(next_token), pages.ref, row.data_ptr(), row.numel()))

    @contextlib.contextmanager
    def _in_order(self):
        with torch.cuda.device(self._stream.device):
            here = torch.cuda.current_stream()
            if here == self._stream:
                yield
                return
            self._stream.wait_stream(here)
            try:
                yield
            finally:
                here.wait_stream(self._stream)

    def _check_pages(self, pages: "Pages", row: torch.Tensor):
        _check_on(pages.device, torch.int32, row=row)
        assert row.dim() == 1 and row.is_contiguous()
        if pages.index != self.workspace.get_device():
            raise ValueError("pages and context are on different devices")

    def read_records(self, n: int):
        toks = np.empty(n, dtype=np.int32)
        es = np.empty(n, dtype=np.int32)
        sims = np.empty((n, self.cfg.n_layers), dtype=np.float32)
        self._check(load().river_read_records(self._h, n, toks.ctypes.data, es.ctypes.data,
                                              sims.ctypes.data))
        return toks, es, sims

    def rewind(self, new_len: int, seq: int = 0):
        self._check(load().river_rewind(self._h, seq, new_len))

    @property
    def pos(self) -> int:
        return load().river_position(self._h)

    def hidden(self) -> np.ndarray:
        out = np.empty((self.cfg.n_layers + 1, self.cfg.d_model), dtype=np.float32)
        self._check(load().river_get_debug(self._h, DBG_HIDDEN, out.ctypes.data, out.nbytes))
        return out

    def logits(self) -> np.ndarray:
        out = np.empty(self.cfg.vocab, dtype=np.float32)
        self._check(load().river_get_debug(self._h, DBG_LOGITS, out.ctypes.data, out.nbytes))
        return out

    def _cache(self, what) -> np.ndarray:
        c = self.cfg
        kvd = c.n_kv_heads * c.head_dim
        shape = (c.n_layers, c.max_seq, kvd) if self.max_batch == 1 else (self.max_batch, c.n_layers, c.max_seq, kvd)
        if c.dtype == 1:
            raw = np.empty(shape, dtype=np.uint16)
            self._check(load().river_get_debug(self._h, what, raw.ctypes.data, raw.nbytes))
            if c.kv_dtype == 1:
                return raw.view(np.float16).astype(np.float32)         # IEEE half words -> fp32 values
            return (raw.astype(np.uint32) << 16).view(np.float32)      # bf16 words -> fp32 values
        raw = np.empty(shape, dtype=np.float32)
        self._check(load().river_get_debug(self._h, what, raw.ctypes.data, raw.nbytes))
        return raw

    def kcache(self) -> np.ndarray:
        return self._cache(DBG_KCACHE)

    def vcache(self) -> np.ndarray:
        return self._cache(DBG_VCACHE)

    def trace(self, workgroups: int) -> np.ndarray:
        """[5L, 2, workgroups] barrier arrive/release device times (diagnostics build only)."""
        n = 5 * self.cfg.n_layers * 2 * workgroups
        out = np.empty(n + 64, dtype=np.uint64)
        self._check(load().river_get_debug(self._h, DBG_TRACE, out.ctypes.data, out.nbytes))
        self.marks = out[n:].astype(np.int64)
        return out[:n].reshape(5 * self.cfg.n_layers, 2, workgroups)

    def fill_cache(self, byte: int):
        self._check(load().river_fill_cache(self._h, byte))


# ------------------------------------------------------------------ paged key-value cache

def _check_call(rc: int) -> int:
    if rc < 0:
        raise RiverError(rc, load().river_last_error(None).decode())
    return rc


def _check_on(device, dtype, **tensors):
    for name, t in tensors.items():
        if t.device != device or t.dtype != dtype:
            raise ValueError(f"{name}: {dtype} on {device} is needed, not {t.dtype} on {t.device}")


# (the device's number and its stream's handle without the torch.cuda objects around them, which take longer than a small call; a torch
# that is built without a GPU has neither, and imports this module all the same)
_device = getattr(torch._C, "_cuda_getDevice", None)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


class _Fixed:
    """What the library was told of once stays as it is: another tensor or bound needs another object."""

    _made = False

    def __setattr__(self, name, value):
        if self._made:
            raise AttributeError(f"{type(self).__name__}.{name} cannot be changed: make another {type(self).__name__}")
        object.__setattr__(self, name, value)


class Pages(_Fixed):
    """A paged cache: k and v [n_layers, n_pages, n_kv_heads, page_size, head_dim] (the last three dimensions
    contiguous, the strides of k and v alike), in the dtype of the activations (fp32, bf16) or, with bf16 ones, fp16."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, dtype: torch.dtype | None = None):
        dtype = k.dtype if dtype is None else dtype
        if not k.is_cuda or k.dim() != 5 or k.shape != v.shape or k.stride() != v.stride() or v.device != k.device or v.dtype != k.dtype:
            raise ValueError("k and v: device tensors [layers, pages, heads, page_size, head_dim] of one shape, type and layout")
        layers, pages, heads, size, hd = k.shape
        if k.stride()[2:] != (size * hd, hd, 1):
            raise ValueError("a page's heads, positions and elements must be contiguous")
        if (dtype, k.dtype) not in ((torch.float32,) * 2, (torch.bfloat16,) * 2, (torch.bfloat16, torch.float16)):
            raise ValueError(f"no cache of {k.dtype} for {dtype}")
        self.k, self.v, self.dtype, self.device, self.index = k, v, dtype, k.device, k.device.index
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        self.c = river_pages(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), layers, pages, size, heads, hd,
                             0 if dtype == torch.float32 else 1, 1 if k.dtype == torch.float16 else 0)
        self.ref = C.byref(self.c)
        self.shape_key = (heads, size, hd, dtype)
        self._made = True


class Batch(_Fixed):
    """The sequences of a call: table [n_seq, max_pages], lens [n_seq] and q_start [n_seq + 1] (None: one new token per
    sequence), int32 on the device and read there at every call.  max_new and max_len bound a sequence's new tokens (further ones
    are left out of the attention) and positions (more are still right); the attention divides its work by them, so that bounds
    near what is there are fastest.  Default: a call's tokens, and what the table holds."""

    def __init__(self, table: torch.Tensor, lens: torch.Tensor, q_start: torch.Tensor | None = None, max_new: int | None = None,
                 max_len: int | None = None):
        _check_on(table.device, torch.int32, table=table, lens=lens, **({} if q_start is None else {"q_start": q_start}))
        n = lens.numel()
        if not table.is_cuda or table.dim() != 2 or table.shape[0] != n or table.shape[1] < 1 or lens.dim() != 1:
            raise ValueError("table [n_seq, max_pages] and lens [n_seq] on the device")
        if (table.shape[1] > 1 and table.stride(1) != 1) or (n > 1 and table.stride(0) < table.shape[1]) or not lens.is_contiguous():
            raise ValueError("rows of the table and lens must be contiguous")
        if q_start is not None and (q_start.shape != (n + 1,) or not q_start.is_contiguous()):
            raise ValueError("q_start [n_seq + 1]")
        if q_start is None and max_new not in (None, 1):
            raise ValueError("without q_start every sequence has one new token")
        self.table, self.lens, self.q_start, self.index, self.n_seq = table, lens, q_start, table.get_device(), n
        self.max_len, self.max_new = max_len, max_new
        self._calls, self._bytes = {}, {}       # the C struct, and the workspace's size, of a shape of call
        self._made = True

    def bind(self, n_tokens: int, pages: Pages):
        """The call's C struct (one per number of tokens and page size: never changed once made)."""
        if pages.index != self.index:
            raise ValueError("pages and batch are on different devices")
        got = self._calls.get((n_tokens, pages.page_size))
        if got is None:
            most = self.table.shape[1]
            c = river_batch(self.table.data_ptr(), self.lens.data_ptr(), None if self.q_start is None else self.q_start.data_ptr(), self.n_seq,
                            n_tokens, most, self.table.stride(0) if self.n_seq > 1 else most,
                            n_tokens if self.max_new is None else self.max_new,
                            min(2**31 - 1, most * pages.page_size) if self.max_len is None else self.max_len)
            if len(self._calls) >= 256:
                self._calls.clear()
                self._bytes.clear()
            got = self._calls[(n_tokens, pages.page_size)] = C.byref(c)
        return got


class Rope(_Fixed):
    """Rotary positions: inv_freq float64 [rot_dim / 2] on the device (river_rope_frequencies has the usual ones), layout "half" or "interleaved"."""

    def __init__(self, inv_freq: torch.Tensor, layout: str = "half", mscale: float = 1.0):
        if not inv_freq.is_cuda or inv_freq.dtype != torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
            raise ValueError("inv_freq: float64 [rot_dim / 2] on the device")
        self.inv_freq, self.index = inv_freq, inv_freq.get_device()
        self.c = river_rope(inv_freq.data_ptr(), 2 * inv_freq.numel(), ROPE_LAYOUTS[layout], mscale)
        self.ref = C.byref(self.c)
        self._made = True


def river_rope_frequencies(rot_dim: int, base: float, scaling: str = "plain", factor: float = 1.0, original_len: float = 0.0,
                           low: float | None = None, high: float | None = None):
    """(frequencies as a numpy array of float64, what cosines and sines are multiplied with).  low and high: turns between which
    "bands" (default 1 and 4) and "ramp" (1 and 32) pass from scaled to unscaled frequencies."""
    low, high = 1.0 if low is None else low, ROPE_HIGH.get(scaling, 32.0) if high is None else high
    f, m = np.empty(max(rot_dim // 2, 1), dtype=np.float64), C.c_float()
    _check_call(load().river_rope_frequencies(rot_dim, base, ROPE_SCALINGS[scaling], factor, original_len, low, high, f.ctypes.data,
                                              C.byref(m)))
    return f, m.value


def _rows(name: str, t: torch.Tensor, pages: Pages, heads: int | None = None) -> int:
    """[n_tokens, heads, head_dim] with contiguous heads: the stride between tokens."""
    shape = t.shape
    if t.dtype is not pages.dtype or t.get_device() != pages.index or len(shape) != 3 or shape[2] != pages.head_dim:
        raise ValueError(f"{name}: {pages.dtype} [n_tokens, heads, {pages.head_dim}] on {pages.device}")
    n, h, hd = shape
    between, head, one = t.stride()
    if (heads is not None and h != heads) or one != 1 or (h > 1 and head != hd):
        raise ValueError(f"{name}: wrong number of heads, or a token's heads are not contiguous")
    return between if n > 1 else h * hd


def _out(q: torch.Tensor, out: torch.Tensor | None, pages: Pages):
    """The place of the result (a new tensor where none is given) and the stride between its tokens."""
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        return out, q.shape[1] * q.shape[2]
    if out.shape != q.shape:
        raise ValueError("out must have q's shape")
    return out, _rows("out", out, pages)


def river_rope_store(pages: Pages, layer: int, batch: Batch, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rope: Rope,
                     out: torch.Tensor | None = None) -> torch.Tensor:
    """Rotates q and k [n_tokens, heads, head_dim] at the new tokens' positions and stores k and v in the pages.  Returns the
    rotated queries: `out`, which may be q, or a new tensor (rows of tokens that belong to no sequence are not written).  For inference:
    autograd does not see it."""
    if pages.index != _device():        # the library takes the current device and the stream that it is given
        with torch.cuda.device(pages.index):
            return river_rope_store(pages, layer, batch, q, k, v, rope, out)
    n = q.shape[0]
    qs, ks, vs = _rows("q", q, pages), _rows("k", k, pages, pages.n_kv_heads), _rows("v", v, pages, pages.n_kv_heads)
    if k.shape[0] != n or v.shape[0] != n or rope.index != pages.index:
        raise ValueError("q, k and v must have the same tokens, and the frequencies their device")
    out, os_ = _out(q, out, pages)
    _check_call(load().river_rope_store(pages.ref, layer, batch.bind(n, pages), rope.ref, q.shape[1], q.data_ptr(), qs, k.data_ptr(), ks,
                                        v.data_ptr(), vs, out.data_ptr(), os_, _stream(pages.index)))
    return out


def river_paged_attention(pages: Pages, layer: int, batch: Batch, q: torch.Tensor, window: int = 0, sinks: int = 0,
                          scale: float = 0.0, out: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of the new tokens' queries [n_tokens, heads, head_dim] over their sequences' pages.  Rows of `out` (or of the new
    tensor that is returned) whose tokens belong to no sequence are not written.  For inference: autograd does not see it."""
    if pages.index != _device():
        with torch.cuda.device(pages.index):
            return river_paged_attention(pages, layer, batch, q, window, sinks, scale, out)
    qs = _rows("q", q, pages)
    out, os_ = _out(q, out, pages)
    L, (n, heads, _) = load(), q.shape
    ref = batch.bind(n, pages)
    key = (pages.shape_key, n, heads, window, sinks)
    nbytes = batch._bytes.get(key)
    if nbytes is None:
        got = C.c_size_t()
        _check_call(L.river_paged_attention_workspace(pages.ref, ref, heads, window, sinks, C.byref(got)))
        if len(batch._bytes) >= 256:
            batch._bytes.clear()
        nbytes = batch._bytes[key] = got.value
    stream, ws, tickets = _stream(pages.index), None, None
    if nbytes:
        # (from torch's allocator, call by call: the memory of a captured call belongs to its graph, and no two streams share it)
        memory = torch.empty(nbytes, dtype=torch.uint8, device=pages.device)
        ws, tickets = memory.data_ptr(), _tickets(pages.index, stream)
    _check_call(L.river_paged_attention(pages.ref, layer, ref, heads, q.data_ptr(), qs, scale, window, sinks, out.data_ptr(), os_, ws, nbytes,
                                        tickets, stream))
    return out


_ticket_tensors = {}


def _tickets(index: int, stream: int):
    """The attention's tickets for a stream: its calls run one after the other, so one set serves them all.  None while a graph is
    captured, which may be replayed on any stream at any time."""
    if torch._C._cuda_isCurrentStreamCapturing():
        return None
    t = _ticket_tensors.get((index, stream))
    if t is None:
        # (two threads that call for the first time at once get the one tensor that stays: another would be freed under a call's kernel)
        t = _ticket_tensors.setdefault((index, stream), torch.zeros(TICKETS, dtype=torch.int32, device=f"cuda:{index}"))
    return t.data_ptr()


def _page_list(x) -> np.ndarray:
    if isinstance(x, np.ndarray) and x.dtype == np.int32 and x.ndim == 1 and x.flags.c_contiguous:
        return x
    a = np.ascontiguousarray(x)
    if a.ndim != 1 or (a.size and a.dtype.kind not in "iu"):
        raise ValueError("a list of page numbers")
    if a.size and (a.min() < -2**31 or a.max() >= 2**31):
        raise ValueError("page number out of range")
    return a.astype(np.int32, copy=False)


def river_copy_pages(pages: Pages, src, dst):
    """Copies pages src[i] -> dst[i] (host lists) in every layer, as if one after the other."""
    s, d = _page_list(src), _page_list(dst)
    if s.size != d.size:
        raise ValueError("as many destinations as sources")
    if pages.index != _device():
        with torch.cuda.device(pages.index):
            return river_copy_pages(pages, s, d)
    _check_call(load().river_copy_pages(pages.ref, s.ctypes.data, d.ctypes.data, s.size, _stream(pages.index)))


class PagePool:
    """Which sequence has which pages (river_pool_*).  lens and table are views of `state`, which flush keeps current on
    the device; a Batch over their rows serves every step."""

    def __init__(self, n_pages: int, page_size: int, max_seqs: int, max_pages: int, device="cuda:0"):
        h = C.c_void_p()
        _check_call(load().river_pool_create(n_pages, page_size, max_seqs, max_pages, C.byref(h)))
        self._h, self.max_seqs, self.max_pages = h, max_seqs, max_pages
        self.state = torch.empty(max_seqs * (max_pages + 1), dtype=torch.int32, device=device)
        self.index = self.state.device.index
        self.lens, self.table = self.state[:max_seqs], self.state[max_seqs:].view(max_seqs, max_pages)

    def close(self):
        if getattr(self, "_h", None):
            load().river_pool_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def extend(self, seq: int, n_new: int):
        _check_call(load().river_pool_extend(self._h, seq, n_new))

    def fork(self, src: int, dst: int):
        _check_call(load().river_pool_fork(self._h, src, dst))

    def rewind(self, seq: int, new_len: int):
        _check_call(load().river_pool_rewind(self._h, seq, new_len))

    def free(self, seq: int):
        self.rewind(seq, 0)

    def trim(self, seq: int, window: int, sinks: int = 0):
        _check_call(load().river_pool_trim(self._h, seq, window, sinks))

    def compact(self) -> int:
        return _check_call(load().river_pool_compact(self._h))

    def flush(self, pages: Pages | None = None):
        """Queued copies and changed entries, on the device's current stream."""
        if pages is not None and pages.device != self.state.device:
            raise ValueError("pages and pool are on different devices")
        if self.index != _device():
            with torch.cuda.device(self.index):
                return self.flush(pages)
        _check_call(load().river_pool_flush(self._h, None if pages is None else pages.ref, self.state.data_ptr(), _stream(self.index)))

    def length(self, seq: int) -> int:
        return _check_call(load().river_pool_length(self._h, seq))

    @property
    def free_pages(self) -> int:
        return _check_call(load().river_pool_free_pages(self._h))

    def row(self, seq: int) -> np.ndarray:
        out = np.empty(self.max_pages, dtype=np.int32)
        _check_call(load().river_pool_row(self._h, seq, out.ctypes.data))
        return out


# The C entry points under their own names (the class above is the same calls with
# the context kept in an object).
def river_create(cfg, dev_weights, dev_river, exec_mode=None, spin_limit=0) -> River:
    return River(cfg, dev_weights, dev_river, exec_mode, spin_limit)


def river_create_static(cfg, dev_weights, dev_river, exec_mode=None, spin_limit=0) -> River:
    return River(cfg, dev_weights, dev_river, exec_mode, spin_limit, static_scratch=True)


def river_prefill(ctx: River, tokens, exit_layer=None, out_logits=None) -> int:
    return ctx.prefill(tokens, exit_layer, out_logits)


def river_decode_step(ctx: River, token=None, forced_exit=None, sync=True):
    return ctx.decode_step(token, forced_exit, sync)


def river_decode_batch(ctx: River, n_seq: int, tokens=None, forced_exits=None, sync=True):
    return ctx.decode_batch(n_seq, tokens, forced_exits, sync)


def river_read_batch_records(ctx: River, n_steps: int, n_seq: int):
    return ctx.read_batch_records(n_steps, n_seq)


def river_read_records(ctx: River, n: int):
    return ctx.read_records(n)


def river_rewind(ctx: River, new_len: int):
    ctx.rewind(new_len)


def river_destroy(ctx: River):
    ctx.close()


# ------------------------------------------------------------------ a step laid out on the device, common prefixes

class Prefixes(_Fixed):
    """Prefixes that sequences of a Batch have in common: table [n_groups, max_pages], lens [n_groups] and seq_start [n_groups + 1], int32
    on the device and read there at every call: sequences seq_start[g] .. seq_start[g + 1] - 1 have the first lens[g] positions in the pages of
    row g.  max_len and max_seqs bound the prefixes' positions and a group's sequences (more are still right); the attention divides
    its work by them.  Default: what the table holds, and all sequences of the call."""

    def __init__(self, table: torch.Tensor, lens: torch.Tensor, seq_start: torch.Tensor, max_len: int | None = None, max_seqs: int | None = None):
        _check_on(table.device, torch.int32, table=table, lens=lens, seq_start=seq_start)
        n = lens.numel()
        if not table.is_cuda or table.dim() != 2 or table.shape[0] != n or table.shape[1] < 1 or lens.dim() != 1:
            raise ValueError("table [n_groups, max_pages] and lens [n_groups] on the device")
        if (table.shape[1] > 1 and table.stride(1) != 1) or (n > 1 and table.stride(0) < table.shape[1]) or not lens.is_contiguous():
            raise ValueError("rows of the table and lens must be contiguous")
        if seq_start.shape != (n + 1,) or not seq_start.is_contiguous():
            raise ValueError("seq_start [n_groups + 1]")
        self.table, self.lens, self.seq_start, self.index, self.n_groups = table, lens, seq_start, table.get_device(), n
        self.max_len, self.max_seqs = max_len, max_seqs
        self.shape_key = (n, table.shape[1], max_len, max_seqs)
        self._calls = {}                        # the C struct of a number of sequences and page size
        self._made = True

    def bind(self, n_seq: int, page_size: int):
        got = self._calls.get((n_seq, page_size))
        if got is None:
            most = self.table.shape[1]
            if len(self._calls) >= 256:
                self._calls.clear()
            got = self._calls[(n_seq, page_size)] = C.byref(river_prefixes(
                self.table.data_ptr(), self.lens.data_ptr(), self.seq_start.data_ptr(), self.n_groups, most,
                self.table.stride(0) if self.n_groups > 1 else most,
                min(2**31 - 1, most * page_size) if self.max_len is None else self.max_len, n_seq if self.max_seqs is None else self.max_seqs))
        return got


def river_prefix_attention(pages: Pages, layer: int, batch: Batch, prefixes: Prefixes, q: torch.Tensor, scale: float = 0.0,
                           out: torch.Tensor | None = None) -> torch.Tensor:
    """river_paged_attention, without a window, of sequences that go on from common prefixes, whose pages are read once for a group.  Rows of `out`
    (or of the new tensor that is returned) whose tokens belong to no sequence are not written.  For inference: autograd does not see it."""
    if pages.index != _device():
        with torch.cuda.device(pages.index):
            return river_prefix_attention(pages, layer, batch, prefixes, q, scale, out)
    if prefixes.index != pages.index:
        raise ValueError("pages and prefixes are on different devices")
    qs = _rows("q", q, pages)
    out, os_ = _out(q, out, pages)
    L, (n, heads, _) = load(), q.shape
    ref, shared = batch.bind(n, pages), prefixes.bind(batch.n_seq, pages.page_size)
    key = (pages.shape_key, n, heads, prefixes.shape_key)
    nbytes = batch._bytes.get(key)
    if nbytes is None:
        got = C.c_size_t()
        _check_call(L.river_prefix_attention_workspace(pages.ref, ref, shared, heads, C.byref(got)))
        if len(batch._bytes) >= 256:
            batch._bytes.clear()
        nbytes = batch._bytes[key] = got.value
    stream, ws, tickets = _stream(pages.index), None, None
    if nbytes:
        memory = torch.empty(nbytes, dtype=torch.uint8, device=pages.device)        # (call by call: see river_paged_attention)
        ws, tickets = memory.data_ptr(), _tickets(pages.index, stream)
    _check_call(L.river_prefix_attention(pages.ref, layer, ref, shared, heads, q.data_ptr(), qs, scale, out.data_ptr(), os_, ws, nbytes,
                                         tickets, stream))
    return out


def river_store_slots(pages: Pages, layer: int, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor):
    """Stores k and v [n_tokens, heads, head_dim] as they are to slots [n_tokens] (int64: page * page_size + place in the page, below 0: left
    out; none of them twice).  For inference: autograd does not see it."""
    if pages.index != _device():
        with torch.cuda.device(pages.index):
            return river_store_slots(pages, layer, slots, k, v)
    ks, vs, n = _rows("k", k, pages, pages.n_kv_heads), _rows("v", v, pages, pages.n_kv_heads), k.shape[0]
    if v.shape[0] != n or slots.shape != (n,) or slots.dtype is not torch.int64 or slots.get_device() != pages.index or not slots.is_contiguous():
        raise ValueError("slots: int64 [n_tokens] on the pages' device, and as many keys and values")
    _check_call(load().river_store_slots(pages.ref, layer, slots.data_ptr(), n, k.data_ptr(), ks, v.data_ptr(), vs, _stream(pages.index)))


class Tables(_Fixed):
    """A page table that lives on the device alone, and its free list: table [n_seq, max_pages], lens [n_seq], free_pages [n_pages], n_free [1]
    and, where rows begin with pages of somebody else, n_shared [n_seq]; all int32, the caller's, and changed by river_build_batch.  lens_out
    and n_free_out: where it writes lengths and count instead (a step laid out ahead of being taken).  A sequence that has given back positions
    in its first n_shared pages and asks again writes over those entries, or into those pages: lower its n_shared, and copy the page in which it ends,
    before it does."""

    def __init__(self, table: torch.Tensor, lens: torch.Tensor, free_pages: torch.Tensor, n_free: torch.Tensor, page_size: int,
                 n_shared: torch.Tensor | None = None, lens_out: torch.Tensor | None = None, n_free_out: torch.Tensor | None = None):
        lens_out, n_free_out = lens if lens_out is None else lens_out, n_free if n_free_out is None else n_free_out
        vectors = dict(lens=lens, lens_out=lens_out, free_pages=free_pages, n_free=n_free, n_free_out=n_free_out,
                       **({} if n_shared is None else {"n_shared": n_shared}))
        _check_on(table.device, torch.int32, table=table, **vectors)
        n = lens.numel()
        if not table.is_cuda or table.dim() != 2 or table.shape[0] != n or table.shape[1] < 1:
            raise ValueError("table [n_seq, max_pages] and lens [n_seq] on the device")
        if (table.shape[1] > 1 and table.stride(1) != 1) or (n > 1 and table.stride(0) < table.shape[1]):
            raise ValueError("rows of the table must be contiguous")
        for name, t in vectors.items():
            if t.dim() != 1 or not t.is_contiguous() or (name in ("lens_out", "n_shared") and t.numel() != n) or (name[:6] == "n_free" and t.numel() != 1):
                raise ValueError(f"{name}: one number, or as many as there are sequences, contiguous")
        self.table, self.lens, self.lens_out, self.free_pages, self.n_free, self.n_free_out, self.n_shared = (
            table, lens, lens_out, free_pages, n_free, n_free_out, n_shared)
        self.n_seq, self.page_size, self.device, self.index = n, page_size, table.device, table.get_device()
        self.c = river_tables(table.data_ptr(), lens.data_ptr(), lens_out.data_ptr(), free_pages.data_ptr(), n_free.data_ptr(), n_free_out.data_ptr(),
                              None if n_shared is None else n_shared.data_ptr(), n, table.shape[1], table.stride(0) if n > 1 else table.shape[1],
                              free_pages.numel(), page_size)
        self.ref = C.byref(self.c)
        self._made = True

    @classmethod
    def empty(cls, n_pages: int, page_size: int, max_seqs: int, max_pages: int, device="cuda:0", n_shared: torch.Tensor | None = None) -> "Tables":
        """No positions, all pages free, the lowest given out first."""
        free = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
        return cls(torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=device), torch.zeros(max_seqs, dtype=torch.int32, device=device),
                   free, torch.full((1,), n_pages, dtype=torch.int32, device=device), page_size, n_shared)


def _vector(name: str, t: torch.Tensor | None, dtype: torch.dtype, n: int | None, index: int):
    """The address of a contiguous vector on the device, of n numbers (None: of any number)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != index or t.dim() != 1 or (n is not None and t.numel() != n) or not t.is_contiguous():
        raise ValueError(f"{name}: contiguous {dtype} [{'n_tokens' if n is None else n}] on the tables' device")
    return t.data_ptr()


def river_build_batch(tables: Tables, n_new: torch.Tensor, q_start: torch.Tensor, slots: torch.Tensor | None = None,
                      positions: torch.Tensor | None = None, refused: torch.Tensor | None = None, n_tokens: int | None = None):
    """Lays a step out: sequence s gets n_new[s] positions more (or gives back -n_new[s]), all of them or none.  Written: q_start [n_seq + 1],
    and where given slots (int64) and positions (int32) [n_tokens] of the new tokens, refused [1] (sequences that asked and got nothing).  n_tokens: no
    more new tokens than these in the call (default: the room in slots or positions, else 2^22)."""
    if tables.index != _device():
        with torch.cuda.device(tables.index):
            return river_build_batch(tables, n_new, q_start, slots, positions, refused, n_tokens)
    if n_tokens is None:
        n_tokens = slots.numel() if slots is not None else positions.numel() if positions is not None else 1 << 22
    i, n = tables.index, tables.n_seq
    _check_call(load().river_build_batch(tables.ref, _vector("n_new", n_new, torch.int32, n, i), n_tokens,
                                         _vector("q_start", q_start, torch.int32, n + 1, i), _vector("slots", slots, torch.int64, n_tokens, i),
                                         _vector("positions", positions, torch.int32, n_tokens, i), _vector("refused", refused, torch.int32, 1, i),
                                         _stream(i)))
