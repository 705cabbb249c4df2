"""Thin Python binding of libsps_b200.so (the C ABI of include/sps.h).

Argument marshalling only: torch supplies device memory and streams, every step of the path runs in
the library's CUDA kernels.  There is no CPU fallback: if the library is missing or there is no CUDA
device, calls raise.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

from . import build as _build

SPS_OK, SPS_EINVAL, SPS_ENOMEM, SPS_ECUDA, SPS_ERANGE, SPS_ESTATE, SPS_ETIMEOUT = 0, -1, -2, -3, -4, -5, -6
SPS_MAX_K = 15
FLAG_RESAMPLED, FLAG_BONUS, FLAG_FALLBACK = 1, 2, 4
CFG_NO_GRAPH = 1
CFG_TENSOR_PARALLEL = 2
LAYER_KEYS = ("attn_norm", "ffn_norm", "wq", "wk", "wv", "wo", "w_up", "w_down")
SCALED_KEYS = ("wq", "wk", "wv", "wo", "w_up", "w_down")   # matrices that carry row scales when weights are int8


class SpsError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"sps error {code}: {msg}")
        self.code = code


class sps_model_cfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("d_head", C.c_int32),
                ("d_ff", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("rms_eps", C.c_float),
                ("rope_base", C.c_float), ("n_kv_heads", C.c_int32)]


class sps_cfg(C.Structure):
    _fields_ = [("target", sps_model_cfg), ("draft", sps_model_cfg), ("max_seq", C.c_int32), ("max_batch", C.c_int32),
                ("max_K", C.c_int32), ("device", C.c_int32), ("stream", C.c_void_p), ("flags", C.c_uint32)]


class sps_weights(C.Structure):
    _fields_ = [("tok_embed", C.c_void_p), ("unembed", C.c_void_p), ("final_norm", C.c_void_p)] + \
               [(k, C.POINTER(C.c_void_p)) for k in LAYER_KEYS] + [("unembed_scale", C.c_void_p)] + \
               [(k + "_scale", C.POINTER(C.c_void_p)) for k in SCALED_KEYS]


class sps_stats(C.Structure):
    _fields_ = [("loops", C.c_int32), ("draft_calls", C.c_int32), ("emitted", C.c_int32), ("accepted", C.c_int32),
                ("resampled", C.c_int32), ("bonus", C.c_int32), ("fallback", C.c_int32), ("overshoot", C.c_int32),
                ("hist_emitted", C.c_int32 * (SPS_MAX_K + 2)), ("ms_prefill", C.c_float), ("ms_decode", C.c_float),
                ("ms_draft", C.c_float), ("ms_verify", C.c_float), ("ms_accept", C.c_float), ("kernel_launches", C.c_int32)]

    def as_dict(self):
        d = {k: getattr(self, k) for k, _ in self._fields_ if k != "hist_emitted"}
        d["hist_emitted"] = list(self.hist_emitted)
        return d


class sps_rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64), ("dtype", C.c_int32), ("heads", C.c_int32)]


class sps_rotary_plan(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("rot_dim", C.c_int32), ("layout", C.c_int32), ("gain", C.c_float)]


class sps_paged_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("pos_stride", C.c_int64),
                ("dtype", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("d_head", C.c_int32)]


class sps_paged_batch(C.Structure):
    _fields_ = [("q_start", C.c_void_p), ("kv_len", C.c_void_p), ("pages", C.c_void_p), ("status", C.c_void_p),
                ("B", C.c_int32), ("pages_ld", C.c_int32), ("max_q", C.c_int32)]


class sps_page_pool(C.Structure):
    _fields_ = [("refs", C.c_void_p), ("status", C.c_void_p), ("n_pages", C.c_int32), ("page_size", C.c_int32)]


class sps_page_table(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("held", C.c_void_p), ("len", C.c_void_p), ("B", C.c_int32), ("ld", C.c_int32)]


class sps_page_moves(C.Structure):
    _fields_ = [("list", C.c_void_p), ("count", C.c_void_p), ("capacity", C.c_int32)]


_lib = None


def lib_path() -> str:
    return _build.LIB


def lib():
    """Load the CUDA library, building it first if the sources are newer.  Raises if that fails."""
    global _lib
    if _lib is None:
        path = _build.build()
        L = C.CDLL(path)
        vp, i32, u32, u64, f32, i64 = C.c_void_p, C.c_int32, C.c_uint32, C.c_uint64, C.c_float, C.c_int64
        L.sps_create.argtypes = [C.POINTER(sps_weights), C.POINTER(sps_weights), C.POINTER(sps_cfg), C.POINTER(vp)]
        L.sps_destroy.argtypes = [vp]
        L.sps_last_error.argtypes = [vp]
        L.sps_last_error.restype = C.c_char_p
        L.sps_generate.argtypes = [vp, vp, i32, i32, i32, f32, u64, vp, C.POINTER(sps_stats)]
        L.sps_generate_batch.argtypes = [vp, vp, i32, i32, i32, i32, f32, u64, vp, C.POINTER(sps_stats)]
        L.sps_reset.argtypes = [vp]
        L.sps_prefill.argtypes = [vp, vp, i32]
        L.sps_step.argtypes = [vp, i32, f32, u64, u32, vp, vp, vp]
        L.sps_last_logits.argtypes = [vp, i32, vp, vp, vp]
        L.sps_last_loop_trace.argtypes = [vp, vp, vp, vp, i32, vp]
        L.sps_set_forced_acceptance.argtypes = [vp, f32]
        L.sps_verify.argtypes = [vp, vp, i32, vp, C.POINTER(f32)]
        L.sps_score.argtypes = [vp, i32, vp, i32, vp, C.POINTER(f32)]
        L.sps_accept.argtypes = [vp, vp, vp, i32, i32, i32, f32, u64, u32, vp, vp, vp, vp]
        L.sps_sample.argtypes = [vp, i32, i32, f32, u64, u32, u32, vp, vp]
        L.sps_set_sampling.argtypes = [vp, i32, f32]
        L.sps_generate_adaptive.argtypes = [vp, vp, i32, i32, i32, i32, f32, u64, vp, C.POINTER(sps_stats)]
        L.sps_accept_filtered.argtypes = [vp, vp, vp, i32, i32, i32, f32, i32, f32, u64, u32, vp, vp, vp, vp]
        L.sps_sample_filtered.argtypes = [vp, i32, i32, f32, i32, f32, u64, u32, u32, vp, vp]
        L.sps_linear.argtypes = [vp, i32, vp, i32, i32, i32, vp, vp, vp, C.POINTER(f32)]
        L.sps_linear_scaled.argtypes = [vp, i32, vp, vp, i32, i32, i32, vp, vp, vp, C.POINTER(f32)]
        L.sps_linear_wide.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, C.POINTER(f32)]
        L.sps_linear_wide_workspace_bytes.argtypes = [i32, i32]
        L.sps_linear_wide_workspace_bytes.restype = i64
        L.sps_linear_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.sps_linear_workspace_bytes.restype = i64
        L.sps_philox.argtypes = [vp, vp, i32, vp, vp]
        L.sps_linear_static.argtypes = [vp, i32, vp, i32, i32, i32, vp, vp]
        L.sps_linear_static_max_floats.restype = i64
        L.sps_linear_static_floats_needed.argtypes = [i32, i32, i32, i32]
        L.sps_linear_static_floats_needed.restype = i64
        L.sps_prefill_batch.argtypes = [vp, vp, vp, i32, i32]
        L.sps_set_sequence_index0.argtypes = [vp, u32]
        L.sps_debug_set_wait.argtypes = [i64, i32]
        L.sps_tp_buffers.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), C.POINTER(i64), C.POINTER(i64)]
        L.sps_tp_attach.argtypes = [vp, i32, i32, vp, vp]
        L.sps_tp_group_prefill.argtypes = [vp, i32, vp, i32]
        L.sps_tp_group_score.argtypes = [vp, i32, i32, vp, i32, vp, C.POINTER(f32)]
        L.sps_tp_group_generate.argtypes = [vp, i32, vp, i32, i32, i32, f32, u64, vp, C.POINTER(sps_stats)]
        f64 = C.c_double
        L.sps_rotary_frequencies.argtypes = [i32, f64, i32, f64, i32, f64, f64, vp]
        L.sps_rotary.argtypes = [vp, vp, vp, i32, i32, vp, i32, vp]
        L.sps_paged_append.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp]
        L.sps_paged_attention.argtypes = [vp, vp, i32, vp, vp, f32, vp, vp, vp]
        L.sps_paged_attention_workspace_bytes.argtypes = [vp, i32, i32]
        L.sps_paged_attention_workspace_bytes.restype = i64
        L.sps_paged_fork.argtypes = [vp, vp, vp, vp, vp]
        L.sps_paged_reserve.argtypes = [vp, vp, vp, vp, vp, vp, vp]
        L.sps_paged_pool_workspace_bytes.argtypes = [i32]
        L.sps_paged_pool_workspace_bytes.restype = i64
        L.sps_paged_compact.argtypes = [vp, vp, vp, vp, vp, vp, vp]
        L.sps_paged_copy.argtypes = [vp, i32, vp, vp]
        L.sps_beam_select.argtypes = [vp, i32, i64, i32, i32, i32, f64, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp]
        L.sps_beam_select_workspace_bytes.argtypes = [i32, i32, i32]
        L.sps_beam_select_workspace_bytes.restype = i64
        _lib = L
    return _lib


def _check(rc, h=None):
    if rc != SPS_OK:
        msg = lib().sps_last_error(h)
        raise SpsError(rc, msg.decode() if msg else "")


def _np_ptr(a):
    return a.ctypes.data_as(C.c_void_p)


def _model_cfg(c: dict) -> sps_model_cfg:
    return sps_model_cfg(c["n_layers"], c["d_model"], c["n_heads"], c["d_head"], c["d_ff"], c["vocab"], c["dtype"],
                         c.get("rms_eps", 1e-5), c.get("rope_base", 10000.0), c.get("n_kv_heads", 0))


def _weights(w: dict, keep: list) -> sps_weights:
    sw = sps_weights()
    sw.tok_embed, sw.unembed, sw.final_norm = w["tok_embed"].data_ptr(), w["unembed"].data_ptr(), w["final_norm"].data_ptr()
    n = len(w["layers"])
    for k in LAYER_KEYS:
        arr = (C.c_void_p * max(n, 1))(*[lw[k].data_ptr() for lw in w["layers"]])
        keep.append(arr)
        setattr(sw, k, C.cast(arr, C.POINTER(C.c_void_p)))
    if "unembed_scale" in w:      # int8 weights (dtype 2): fp32 row scales beside every matrix
        sw.unembed_scale = w["unembed_scale"].data_ptr()
        for k in SCALED_KEYS:
            arr = (C.c_void_p * max(n, 1))(*[lw[k + "_scale"].data_ptr() for lw in w["layers"]])
            keep.append(arr)
            setattr(sw, k + "_scale", C.cast(arr, C.POINTER(C.c_void_p)))
    return sw


class Handle:
    """sps_create / sps_destroy and the calls that take a handle.  `target_w` / `draft_w` are dicts of
    CUDA torch tensors (tok_embed, unembed, final_norm, layers=[{attn_norm, ffn_norm, wq, wk, wv, wo,
    w_up, w_down}]); they must stay alive as long as the handle."""

    def __init__(self, target_cfg, target_w, draft_cfg=None, draft_w=None, max_seq=1024, max_batch=1, max_K=4,
                 device=0, stream=None, flags=0):
        self._keep = [target_w, draft_w]
        cfg = sps_cfg()
        cfg.target = _model_cfg(target_cfg)
        if draft_cfg is not None:
            cfg.draft = _model_cfg(draft_cfg)
        cfg.max_seq, cfg.max_batch, cfg.max_K, cfg.device = max_seq, max_batch, max_K, device
        cfg.stream = stream
        cfg.flags = flags
        tw = _weights(target_w, self._keep)
        dw = _weights(draft_w, self._keep) if draft_w is not None else None
        h = C.c_void_p()
        rc = lib().sps_create(C.byref(tw), C.byref(dw) if dw is not None else None, C.byref(cfg), C.byref(h))
        _check(rc, None)
        self._h = h
        self.vocab = target_cfg["vocab"]
        self.max_K = max_K
        self.B = 1          # sequences the last prefill set

    def close(self):
        if getattr(self, "_h", None):
            lib().sps_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def sps_generate(self, prompt, n_new, K, temperature, seed):
        p = np.ascontiguousarray(prompt, dtype=np.int32)
        out = np.zeros(n_new, dtype=np.int32)
        st = sps_stats()
        _check(lib().sps_generate(self._h, _np_ptr(p), p.shape[0], n_new, K, temperature, seed, _np_ptr(out), C.byref(st)),
               self._h)
        return out, st.as_dict()

    def sps_generate_adaptive(self, prompt, n_new, K_min, K_max, temperature, seed):
        p = np.ascontiguousarray(prompt, dtype=np.int32)
        out = np.zeros(n_new, dtype=np.int32)
        st = sps_stats()
        _check(lib().sps_generate_adaptive(self._h, _np_ptr(p), p.shape[0], n_new, K_min, K_max, temperature, seed, _np_ptr(out),
                                           C.byref(st)), self._h)
        return out, st.as_dict()

    def sps_generate_batch(self, prompts, n_new, K, temperature, seed):
        p = np.ascontiguousarray(prompts, dtype=np.int32)
        B, P = p.shape
        out = np.zeros((B, n_new), dtype=np.int32)
        st = (sps_stats * B)()
        _check(lib().sps_generate_batch(self._h, _np_ptr(p), B, P, n_new, K, temperature, seed, _np_ptr(out), st), self._h)
        return out, [s.as_dict() for s in st]

    def sps_set_sampling(self, top_k=0, top_p=1.0):
        _check(lib().sps_set_sampling(self._h, int(top_k), float(top_p)), self._h)

    def sps_set_forced_acceptance(self, alpha):
        """Measurement mode: accept every draft with probability alpha (0 = off)."""
        _check(lib().sps_set_forced_acceptance(self._h, float(alpha)), self._h)

    def sps_reset(self):
        _check(lib().sps_reset(self._h), self._h)
        self.B = 1

    def sps_prefill(self, toks):
        t = np.ascontiguousarray(toks, dtype=np.int32)
        _check(lib().sps_prefill(self._h, _np_ptr(t), t.shape[0]), self._h)
        self.B = 1

    def sps_prefill_batch(self, seqs):
        """seqs: list of B int sequences (their own lengths): the sequences so far of a batch."""
        lens = np.array([len(x) for x in seqs], dtype=np.int32)
        ld = int(lens.max())
        t = np.zeros((len(seqs), ld), dtype=np.int32)
        for b, x in enumerate(seqs):
            t[b, :len(x)] = x
        _check(lib().sps_prefill_batch(self._h, _np_ptr(t), _np_ptr(lens), len(seqs), ld), self._h)
        self.B = len(seqs)

    def tp_buffers(self):
        """(inbox pointer, flags pointer, inbox bytes, flags bytes) of a tensor-parallel rank's receive buffers."""
        inbox, flags, nb, nf = C.c_void_p(), C.c_void_p(), C.c_int64(0), C.c_int64(0)
        _check(lib().sps_tp_buffers(self._h, C.byref(inbox), C.byref(flags), C.byref(nb), C.byref(nf)), self._h)
        return inbox.value, flags.value, nb.value, nf.value

    def tp_attach(self, rank, world, peer_inbox, peer_flags):
        """peer_inbox / peer_flags: device addresses (ints) of every rank's buffers as this device sees them."""
        pi = (C.c_void_p * world)(*peer_inbox)
        pf = (C.c_void_p * world)(*peer_flags)
        _check(lib().sps_tp_attach(self._h, rank, world, pi, pf), self._h)

    def sps_set_sequence_index0(self, index0):
        """Sequence b of later generate / step calls uses Philox sequence index index0 + b."""
        _check(lib().sps_set_sequence_index0(self._h, int(index0)), self._h)

    def sps_step(self, K, temperature, seed, step):
        """One loop for every sequence of the last prefill.  Batch 1: (tokens [K+1], n_emitted, flags);
        batch B > 1: (tokens [B, K+1], n_emitted [B], flags [B])."""
        B = self.B
        out = np.full((B, K + 1), -1, dtype=np.int32)
        n = np.zeros(B, dtype=np.int32)
        fl = np.zeros(B, dtype=np.uint32)
        _check(lib().sps_step(self._h, K, temperature, seed, step, _np_ptr(out), _np_ptr(n), _np_ptr(fl)), self._h)
        if B == 1:
            return out[0], int(n[0]), int(fl[0])
        return out, n, fl

    def sps_last_loop_trace(self, cap=4096):
        """(loop_ms, loop_emitted, loop_K) of the last generation, one entry per loop."""
        ms, em, kk = np.zeros(cap, dtype=np.float32), np.zeros(cap, dtype=np.int32), np.zeros(cap, dtype=np.int32)
        n = C.c_int32(0)
        _check(lib().sps_last_loop_trace(self._h, _np_ptr(ms), _np_ptr(em), _np_ptr(kk), cap, C.byref(n)), self._h)
        m = min(n.value, cap)
        return ms[:m], em[:m], kk[:m]

    def sps_last_logits(self, K):
        """(q_logits, p_logits, drafts) of the last step: [K+1, V], [K, V], [K] for batch 1, with a leading B otherwise."""
        B = self.B
        q = np.zeros((B, K + 1, self.vocab), dtype=np.float32)
        p = np.zeros((B, K, self.vocab), dtype=np.float32)
        d = np.zeros((B, K), dtype=np.int32)
        _check(lib().sps_last_logits(self._h, K, _np_ptr(q), _np_ptr(p) if K else None, _np_ptr(d) if K else None), self._h)
        if B == 1:
            return q[0], p[0], d[0]
        return q, p, d

    def sps_verify(self, rows, K, out_logits):
        r = np.ascontiguousarray(rows, dtype=np.int32)
        ms = C.c_float(0)
        _check(lib().sps_verify(self._h, _np_ptr(r), K, out_logits.data_ptr(), C.byref(ms)), self._h)
        return ms.value

    def sps_score(self, which, rows, out_logits):
        r = np.ascontiguousarray(rows, dtype=np.int32)
        ms = C.c_float(0)
        _check(lib().sps_score(self._h, which, _np_ptr(r), r.shape[0], out_logits.data_ptr(), C.byref(ms)), self._h)
        return ms.value


def _stream_ptr(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return stream


def sps_accept(q_logits, p_logits, draft_tokens, temperature, seed, step, out_n_accepted, out_tokens, out_flags,
               stream=None):
    """q_logits [B,K+1,V] fp32, p_logits [B,K,V] fp32, draft_tokens [B,K] int32: CUDA torch tensors;
    outputs CUDA int32 [B], int32 [B,K+1], int32-sized [B].  Enqueues one kernel on `stream`."""
    B, K1, V = q_logits.shape
    K = K1 - 1
    _check(lib().sps_accept(q_logits.data_ptr(), p_logits.data_ptr() if K else None,
                            draft_tokens.data_ptr() if K else None, B, K, V, temperature, seed, step,
                            _stream_ptr(stream), out_n_accepted.data_ptr(), out_tokens.data_ptr(), out_flags.data_ptr()))


def sps_accept_filtered(q_logits, p_logits, draft_tokens, temperature, top_k, top_p, seed, step, out_n_accepted, out_tokens,
                        out_flags, stream=None):
    """sps_accept with top-k / nucleus filtering of both distributions (temperature 0 = greedy)."""
    B, K1, V = q_logits.shape
    K = K1 - 1
    _check(lib().sps_accept_filtered(q_logits.data_ptr(), p_logits.data_ptr() if K else None,
                                     draft_tokens.data_ptr() if K else None, B, K, V, temperature, top_k, top_p, seed, step,
                                     _stream_ptr(stream), out_n_accepted.data_ptr(), out_tokens.data_ptr(),
                                     out_flags.data_ptr()))


def sps_sample_filtered(logits, temperature, top_k, top_p, seed, step, t, out_tokens, stream=None):
    B, V = logits.shape
    _check(lib().sps_sample_filtered(logits.data_ptr(), B, V, temperature, top_k, top_p, seed, step, t, _stream_ptr(stream),
                                     out_tokens.data_ptr()))


def sps_sample(logits, temperature, seed, step, t, out_tokens, stream=None):
    B, V = logits.shape
    _check(lib().sps_sample(logits.data_ptr(), B, V, temperature, seed, step, t, _stream_ptr(stream), out_tokens.data_ptr()))


def sps_linear_workspace_bytes(dtype, M, N, D):
    return int(lib().sps_linear_workspace_bytes(dtype, M, N, D))


def sps_linear(W, X, Y, workspace, stream=None, timed=False):
    """Y[M,N] = X[M,D] W[N,D]^T.  W CUDA fp32 or bf16, X/Y CUDA fp32, workspace CUDA uint8 (zeroed once)."""
    import torch
    dtype = 0 if W.dtype == torch.float32 else 1
    N, D = W.shape
    M = X.shape[0]
    ms = C.c_float(0)
    _check(lib().sps_linear(W.data_ptr(), dtype, X.data_ptr(), M, N, D, Y.data_ptr(), workspace.data_ptr(),
                            _stream_ptr(stream), C.byref(ms) if timed else None))
    return ms.value


def sps_linear_scaled(W, row_scale, X, Y, workspace, stream=None, timed=False):
    """Y[m,n] = row_scale[n] * sum_k X[m,k] W[n,k] with W CUDA int8 [N,D], row_scale CUDA fp32 [N]."""
    N, D = W.shape
    M = X.shape[0]
    ms = C.c_float(0)
    _check(lib().sps_linear_scaled(W.data_ptr(), 2, row_scale.data_ptr(), X.data_ptr(), M, N, D, Y.data_ptr(),
                                   workspace.data_ptr(), _stream_ptr(stream), C.byref(ms) if timed else None))
    return ms.value


def sps_linear_wide_workspace_bytes(N, D):
    return int(lib().sps_linear_wide_workspace_bytes(N, D))


def sps_linear_wide(W, X, Y, workspace, stream=None, timed=False):
    """Y[M,N] = X[M,D] W[N,D]^T for up to 128 rows (the prompt pass): W CUDA bf16, X/Y CUDA fp32."""
    N, D = W.shape
    M = X.shape[0]
    ms = C.c_float(0)
    _check(lib().sps_linear_wide(W.data_ptr(), X.data_ptr(), M, N, D, Y.data_ptr(), workspace.data_ptr(),
                                 _stream_ptr(stream), C.byref(ms) if timed else None))
    return ms.value


def sps_philox(ctr, key, out, stream=None):
    _check(lib().sps_philox(ctr.data_ptr(), key.data_ptr(), ctr.shape[0], _stream_ptr(stream), out.data_ptr()))


def sps_linear_static(W, X, Y, stream=None):
    """Y[M,N] = X[M,D] W[N,D]^T with the scratch held inside the library: for callers that cannot
    allocate device memory (see include/sps.h).  W CUDA fp32 or bf16, X/Y CUDA fp32."""
    import torch
    dtype = 0 if W.dtype == torch.float32 else 1
    N, D = W.shape
    _check(lib().sps_linear_static(W.data_ptr(), dtype, X.data_ptr(), X.shape[0], N, D, Y.data_ptr(), _stream_ptr(stream)))


def sps_linear_static_max_floats():
    return int(lib().sps_linear_static_max_floats())


def sps_linear_static_floats_needed(dtype, M, N, D):
    return int(lib().sps_linear_static_floats_needed(dtype, M, N, D))


def sps_debug_set_wait(limit_us=0, drop_stage=-1):
    """Test hook: bound of the kernels' waits in microseconds (0 = the default 2 s) and the stage the first CTA's copy
    producer leaves out (-1 = none)."""
    _check(lib().sps_debug_set_wait(int(limit_us), int(drop_stage)))


# ---------------------------------------------------------------------------------------------------------------------
# rotary positions and the paged cache (see include/sps.h)
# ---------------------------------------------------------------------------------------------------------------------
PAGED_BAD_PAGE, PAGED_BAD_LENGTH, PAGED_TIMEOUT = 1, 2, 4
ROTARY_LAYOUTS = {"pairs": 0, "halves": 1}
ROTARY_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "bands": 3}


def sps_rotary_frequencies(rot_dim, base=10000.0, scaling="plain", factor=1.0, trained_len=0, low_turns=1.0, high_turns=32.0):
    """The pairs' frequencies as a numpy float64 array [rot_dim / 2] (host arithmetic, no GPU needed)."""
    if scaling not in ROTARY_SCALINGS:
        raise ValueError("scaling is one of %s" % ", ".join(ROTARY_SCALINGS))
    out = np.zeros(max(int(rot_dim) // 2, 1), dtype=np.float64)
    _check(lib().sps_rotary_frequencies(int(rot_dim), base, ROTARY_SCALINGS[scaling], factor, trained_len, low_turns, high_turns, _np_ptr(out)))
    return out


class _Torch:
    """What the calls below need of torch, looked up once (importing this module does not import torch)."""
    codes = None

    @classmethod
    def load(cls):
        import torch
        cls.float64, cls.float32, cls.int32, cls.cuda_device = torch.float64, torch.float32, torch.int32, torch.cuda.device
        cls.current_device, cls.raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        cls.codes = {torch.float32: 0, torch.bfloat16: 1}


def _dtype_of(t):
    if _Torch.codes is None:
        _Torch.load()
    code = _Torch.codes.get(t.dtype)
    if code is None:
        raise ValueError("tensors are float32 or bfloat16, got %s" % t.dtype)
    return code


def _rows_of(t, index):
    """A [rows, heads, d_head] tensor (any strides over contiguous heads) on device `index` as an sps_rows, and its shape."""
    shape = t.shape
    if len(shape) != 3 or t.get_device() != index:
        raise ValueError("rows are [rows, heads, d_head] tensors, all on one CUDA device")
    row, head, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError("a head's elements must be contiguous")
    code = _Torch.codes.get(t.dtype)
    if code is None:
        raise ValueError("tensors are float32 or bfloat16, got %s" % t.dtype)
    return sps_rows(t.data_ptr(), row, head, code, shape[1]), shape


class Rotary:
    """A rotary plan: `freq` CUDA float64 [rot_dim / 2] (e.g. torch.from_numpy(sps_rotary_frequencies(...)).cuda()),
    `layout` "pairs" or "halves", `gain` the factor on the rotated elements."""

    def __init__(self, freq, layout="pairs", gain=1.0):
        if layout not in ROTARY_LAYOUTS:
            raise ValueError("layout is one of %s" % ", ".join(ROTARY_LAYOUTS))
        if _Torch.codes is None:
            _Torch.load()
        if freq.dtype is not _Torch.float64 or freq.dim() != 1 or not freq.is_contiguous() or not freq.is_cuda:
            raise ValueError("freq is a contiguous CUDA float64 vector")
        self.freq, self.layout, self.gain, self.device, self.index = freq, layout, float(gain), freq.device, freq.get_device()
        self._c = sps_rotary_plan(freq.data_ptr(), 2 * freq.shape[0], ROTARY_LAYOUTS[layout], self.gain)
        self._p = C.addressof(self._c)


class PagedCache:
    """One layer's pages: k, v CUDA [n_pages, n_kv_heads, page_size, d_head], fp32 or bf16, of the same strides (any with
    contiguous heads: a [n_pages, page_size, n_kv_heads, d_head] tensor goes in as its transpose(1, 2))."""

    def __init__(self, k, v):
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.device != v.device or not k.is_cuda:
            raise ValueError("k and v are CUDA tensors [n_pages, n_kv_heads, page_size, d_head] of the same shape, strides and dtype")
        if k.stride(3) != 1:
            raise ValueError("a slot's d_head elements must be contiguous")
        self.k, self.v, self.device, self.index = k, v, k.device, k.get_device()
        self.d_head = k.shape[3]
        self._c = sps_paged_cache(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2), _dtype_of(k), k.shape[0], k.shape[2],
                                  k.shape[1], k.shape[3])
        self._p = C.addressof(self._c)


class PagedBatch:
    """The sequences of a call: q_start CUDA int32 [B + 1], kv_len CUDA int32 [B], pages CUDA int32 [B, ...] (rows of the
    page table), read by the kernels when they run.  max_q: the most new rows a sequence brings.  `status` (int32 [1],
    made here unless given) collects PAGED_* bits and is never cleared by the calls."""

    def __init__(self, q_start, kv_len, pages, max_q=1, status=None):
        import torch
        for t in (q_start, kv_len, pages):
            if t.dtype != torch.int32 or t.device != q_start.device or not t.is_cuda:
                raise ValueError("q_start, kv_len and pages are CUDA int32 tensors on one device")
        B = kv_len.shape[0]
        if kv_len.dim() != 1 or q_start.dim() != 1 or q_start.shape[0] != B + 1 or pages.dim() != 2 or pages.shape[0] != B:
            raise ValueError("q_start [B + 1], kv_len [B], pages [B, ...]")
        if not (q_start.is_contiguous() and kv_len.is_contiguous()) or (pages.numel() > 0 and pages.stride(1) != 1 and pages.shape[1] > 1):
            raise ValueError("q_start, kv_len and the rows of pages must be contiguous")
        if B > 1 and pages.stride(0) != pages.shape[1]:
            raise ValueError("the rows of pages must follow one another")
        if status is None:
            status = torch.zeros(1, dtype=torch.int32, device=q_start.device)
        if status.dtype != torch.int32 or status.numel() < 1 or status.device != q_start.device:
            raise ValueError("status is a CUDA int32 tensor of one element")
        self.q_start, self.kv_len, self.pages, self.status = q_start, kv_len, pages, status
        self.device, self.index = q_start.device, q_start.get_device()
        self._c = sps_paged_batch(q_start.data_ptr(), kv_len.data_ptr(), pages.data_ptr(), status.data_ptr(), B, pages.shape[1], int(max_q))
        self._p = C.addressof(self._c)


def _on(index, fn, stream, *args):
    """fn(*args, stream) with device `index` current, on `stream` or that device's current one."""
    if _Torch.current_device() == index:
        rc = fn(*args, _Torch.raw_stream(index) if stream is None else stream)
    else:
        with _Torch.cuda_device(index):
            rc = fn(*args, _Torch.raw_stream(index) if stream is None else stream)
    if rc:
        _check(rc)


def sps_rotary(x, y, positions, plan, transposed=False, stream=None):
    """y = gain R(positions) x over the plan's rotated elements, the others copied; x, y CUDA [rows, heads, d_head], fp32 or
    bf16 (y may be x); positions CUDA int32 [rows].  transposed: gain R^T, the gradient."""
    rx, shape = _rows_of(x, plan.index)
    ry, other = _rows_of(y, plan.index)
    if shape != other or positions.dtype is not _Torch.int32 or positions.dim() != 1 or positions.numel() != shape[0] or \
            not positions.is_contiguous() or positions.get_device() != plan.index:
        raise ValueError("x and y [rows, heads, d_head], positions contiguous int32 [rows], all on one CUDA device")
    _on(plan.index, lib().sps_rotary, stream, plan._p, C.byref(rx), C.byref(ry), shape[0], shape[2], positions.data_ptr(), 1 if transposed else 0)


def sps_paged_append(cache, batch, k, v, plan=None, q=None, q_out=None, stream=None):
    """Keys (rotated under `plan`) and values of the batch's rows into their slots; with q, its rotated rows into q_out.
    k, v CUDA [rows, n_kv_heads, d_head]; q, q_out CUDA [rows, heads, d_head]."""
    index = cache.index
    rk, shape = _rows_of(k, index)
    rv, other = _rows_of(v, index)
    if shape != other or shape[2] != cache.d_head:
        raise ValueError("k and v are [rows, n_kv_heads, d_head]")
    if batch.index != index or (plan is not None and plan.index != index):
        raise ValueError("all tensors must be on one CUDA device")
    rq = ro = None
    if q is not None and q_out is not None:
        rq, qs = _rows_of(q, index)
        ro, other = _rows_of(q_out, index)
        if qs != other or qs[0] != shape[0] or qs[2] != shape[2]:
            raise ValueError("q and q_out are [rows, heads, d_head]")
        rq, ro = C.byref(rq), C.byref(ro)
    elif q is not None or q_out is not None:
        raise ValueError("q and q_out go together")
    _on(index, lib().sps_paged_append, stream, cache._p, batch._p, plan._p if plan is not None else None, shape[0], C.byref(rk), C.byref(rv), rq, ro)


def _workspace_bytes(cache, n_heads, code):
    """On the cache's device: its number of SMs counts."""
    if _Torch.current_device() == cache.index:
        return int(lib().sps_paged_attention_workspace_bytes(cache._p, n_heads, code))
    with _Torch.cuda_device(cache.index):
        return int(lib().sps_paged_attention_workspace_bytes(cache._p, n_heads, code))


def sps_paged_attention_workspace_bytes(cache, n_heads, q_dtype):
    """q_dtype: torch.float32 or torch.bfloat16."""
    n = _workspace_bytes(cache, n_heads, _Torch.codes.get(q_dtype, -1))
    if n < 0:
        _check(SPS_EINVAL)
    return n


def sps_paged_attention(cache, batch, q, out, workspace, scale=0.0, lse=None, stream=None):
    """Causal attention of the batch's rows over their sequences' pages.  q, out CUDA [rows, heads, d_head]; workspace CUDA
    uint8 (zeroed once) of sps_paged_attention_workspace_bytes; scale 0 = 1 / sqrt(d_head); lse CUDA float32 [rows, heads]."""
    index = cache.index
    rq, shape = _rows_of(q, index)
    ro, other = _rows_of(out, index)
    if shape != other or shape[2] != cache.d_head:
        raise ValueError("q and out are [rows, heads, d_head]")
    if batch.index != index or workspace.get_device() != index:
        raise ValueError("all tensors must be on one CUDA device")
    lse_p = None
    if lse is not None:
        if lse.shape != shape[:2] or not lse.is_contiguous() or lse.get_device() != index or lse.dtype is not _Torch.float32:
            raise ValueError("lse is contiguous float32 [rows, heads] on the same device")
        lse_p = lse.data_ptr()
    if workspace.nbytes < _workspace_bytes(cache, shape[1], rq.dtype) or not workspace.is_contiguous():
        raise ValueError("workspace not contiguous, or smaller than sps_paged_attention_workspace_bytes")
    _on(index, lib().sps_paged_attention, stream, cache._p, batch._p, shape[0], C.byref(rq), C.byref(ro), scale, lse_p, workspace.data_ptr())


# ---------------------------------------------------------------------------------------------------------------------
# a paged cache's pages, and the selection of a beam step (see include/sps.h)
# ---------------------------------------------------------------------------------------------------------------------
PAGED_NO_PAGE, PAGED_BAD_ROW = 8, 16


def _ints(t, shape, index, what):
    """A contiguous CUDA int32 tensor of that shape on device `index`."""
    if t.dtype is not _Torch.int32 or t.shape != shape or not t.is_contiguous() or t.get_device() != index:
        raise ValueError("%s is contiguous int32 %s on the same CUDA device" % (what, list(shape)))
    return t.data_ptr()


class PagePool:
    """A pool's state: refs CUDA int32 [n_pages], the table rows that hold each page (all zeros: an empty pool).  `status` (int32
    [1], made here unless given) collects PAGED_* bits and is never cleared by the calls."""

    def __init__(self, refs, page_size, status=None):
        import torch
        if _Torch.codes is None:
            _Torch.load()
        if refs.dim() != 1 or not refs.is_cuda:
            raise ValueError("refs is a CUDA int32 tensor [n_pages]")
        self.refs, self.page_size, self.index = refs, int(page_size), refs.get_device()
        p = _ints(refs, (refs.shape[0],), self.index, "refs")
        self.status = torch.zeros(1, dtype=torch.int32, device=refs.device) if status is None else status
        self._need = lib().sps_paged_pool_workspace_bytes(refs.shape[0])
        self._c = sps_page_pool(p, _ints(self.status, (1,), self.index, "status"), refs.shape[0], self.page_size)
        self._p = C.addressof(self._c)


class PageTable:
    """Rows of pages: pages CUDA int32 [B, ld], held (pages of each row) and lens (tokens) CUDA int32 [B]."""

    def __init__(self, pages, held, lens):
        if _Torch.codes is None:
            _Torch.load()
        if pages.dim() != 2 or not pages.is_cuda:
            raise ValueError("pages is a CUDA int32 tensor [B, ld]")
        B, ld = pages.shape
        self.pages, self.held, self.lens, self.index, self.B = pages, held, lens, pages.get_device(), B
        self._c = sps_page_table(_ints(pages, (B, ld), self.index, "pages"), _ints(held, (B,), self.index, "held"), _ints(lens, (B,), self.index, "lens"), B, ld)
        self._p = C.addressof(self._c)


class PageMoves:
    """Pages to be copied: list CUDA int32 [capacity, 3] of (from, to, slots), count CUDA int32 [1]."""

    def __init__(self, list, count):
        if _Torch.codes is None:
            _Torch.load()
        if list.dim() != 2 or not list.is_cuda:
            raise ValueError("list is a CUDA int32 tensor [capacity, 3]")
        self.list, self.count, self.index = list, count, list.get_device()
        self._c = sps_page_moves(_ints(list, (list.shape[0], 3), self.index, "list"), _ints(count, (1,), self.index, "count"), list.shape[0])
        self._p = C.addressof(self._c)


class PagedLayers:
    """The caches of a model's layers (PagedCache, all of one shape, dtype and strides), as sps_paged_copy takes them."""

    def __init__(self, caches):
        if _Torch.codes is None:
            _Torch.load()
        self.caches = list(caches)
        if not self.caches or any(c.index != self.caches[0].index for c in self.caches):
            raise ValueError("caches of one CUDA device, at least one")
        self.index = self.caches[0].index
        self._c = (sps_paged_cache * len(self.caches))(*[c._c for c in self.caches])
        self._p = C.addressof(self._c)


def sps_paged_pool_workspace_bytes(n_pages):
    n = int(lib().sps_paged_pool_workspace_bytes(n_pages))
    if n < 0:
        _check(SPS_EINVAL)
    return n


def _pool_workspace(pool, workspace):
    if workspace.nbytes < pool._need or workspace.get_device() != pool.index or not workspace.is_contiguous():
        raise ValueError("workspace: on the pool's device, contiguous, of sps_paged_pool_workspace_bytes")
    return workspace.data_ptr()


def sps_paged_fork(pool, src, dst, parents, stream=None):
    """Row i of dst becomes row parents[i] of src (-1: an empty row); dst takes src's place in the pool."""
    index = pool.index
    if src.index != index or dst.index != index:
        raise ValueError("all tensors must be on one CUDA device")
    _on(index, lib().sps_paged_fork, stream, pool._p, src._p, dst._p, _ints(parents, (dst.B,), index, "parents"))


def sps_paged_reserve(pool, table, want, moves, workspace, room=None, stream=None):
    """Every row keeps min(len, want) tokens and gets room for want of them; `moves` are then to be copied.  room (CUDA int32 [B]): the
    tokens that each row may then be written up to, want or, where the pool ran out, those kept."""
    index = pool.index
    if table.index != index or moves.index != index:
        raise ValueError("all tensors must be on one CUDA device")
    _on(index, lib().sps_paged_reserve, stream, pool._p, table._p, _ints(want, (table.B,), index, "want"),
        _ints(room, (table.B,), index, "room") if room is not None else None, moves._p, _pool_workspace(pool, workspace))


def sps_paged_compact(pool, src, dst, refs_out, moves, workspace, stream=None):
    """Pages above the number in use move below it; dst, refs_out and `moves` receive the result (dst may be src, refs_out pool.refs)."""
    index = pool.index
    if src.index != index or dst.index != index or moves.index != index:
        raise ValueError("all tensors must be on one CUDA device")
    _on(index, lib().sps_paged_compact, stream, pool._p, src._p, dst._p, _ints(refs_out, (pool._c.n_pages,), index, "refs_out"), moves._p,
        _pool_workspace(pool, workspace))


def sps_paged_copy(layers, moves, stream=None):
    """The listed pages' first slots, in every layer's keys and values."""
    if moves.index != layers.index:
        raise ValueError("all tensors must be on one CUDA device")
    _on(layers.index, lib().sps_paged_copy, stream, layers._p, len(layers._c), moves._p)


def sps_beam_select_workspace_bytes(B, W, V):
    n = int(lib().sps_beam_select_workspace_bytes(B, W, V))
    if n < 0:
        _check(SPS_EINVAL)
    return n


_beam_bytes = {}   # the workspace that a shape needs


def sps_beam_select(logits, scores, out_scores, out_parents, out_tokens, workspace, done=None, out_done=None, end_token=-1,
                    temperature=1.0, stream=None):
    """The N best continuations of each sequence's beams.  logits CUDA [B, W, V], fp32 or bf16 (rows of any one stride); scores CUDA
    float32 [B, W]; done CUDA int32 [B, W]; out_scores float32, out_parents (rows b W + w), out_tokens, out_done int32, all
    [B, N]; workspace CUDA uint8 of sps_beam_select_workspace_bytes."""
    code = _dtype_of(logits)
    index = logits.get_device()
    shape = logits.shape
    if len(shape) != 3 or index < 0:
        raise ValueError("logits is a CUDA tensor [B, W, V]")
    B, W, V = shape
    sb, sw, sv = logits.stride()
    if (sv != 1 and V > 1) or (W > 1 and B > 1 and sb != W * sw):
        raise ValueError("the rows of logits must be contiguous, one stride apart")
    beams, out = (B, W), out_scores.shape
    ints, f32 = _Torch.int32, _Torch.float32
    if scores.dtype is not f32 or scores.shape != beams or out_scores.dtype is not f32 or len(out) != 2 or out[0] != B or \
            not (scores.is_contiguous() and out_scores.is_contiguous()):
        raise ValueError("scores and out_scores are contiguous float32 [B, W] and [B, N]")
    if out_parents.dtype is not ints or out_parents.shape != out or out_tokens.dtype is not ints or out_tokens.shape != out or \
            not (out_parents.is_contiguous() and out_tokens.is_contiguous()):
        raise ValueError("out_parents and out_tokens are contiguous int32 [B, N]")
    done_p = over_p = None
    if done is not None:
        if done.dtype is not ints or done.shape != beams or not done.is_contiguous() or done.get_device() != index:
            raise ValueError("done is contiguous int32 [B, W] on the logits' device")
        done_p = done.data_ptr()
    if out_done is not None:
        if out_done.dtype is not ints or out_done.shape != out or not out_done.is_contiguous() or out_done.get_device() != index:
            raise ValueError("out_done is contiguous int32 [B, N] on the logits' device")
        over_p = out_done.data_ptr()
    if not (scores.get_device() == out_scores.get_device() == out_parents.get_device() == out_tokens.get_device() == workspace.get_device() == index):
        raise ValueError("all tensors must be on one CUDA device")
    L = lib()
    need = _beam_bytes.get((B, W, V))
    if need is None:
        if len(_beam_bytes) > 1000:
            _beam_bytes.clear()
        need = _beam_bytes[(B, W, V)] = L.sps_beam_select_workspace_bytes(B, W, V)
    if workspace.nbytes < need or not workspace.is_contiguous():
        raise ValueError("workspace not contiguous, or smaller than sps_beam_select_workspace_bytes")
    _on(index, L.sps_beam_select, stream, logits.data_ptr(), code, sw if W > 1 else sb, B, W, V, temperature, scores.data_ptr(), done_p, end_token, out[1],
        out_scores.data_ptr(), out_parents.data_ptr(), out_tokens.data_ptr(), over_p, workspace.data_ptr())
