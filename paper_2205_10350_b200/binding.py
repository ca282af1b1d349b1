"""Thin ctypes binding of the C ABI in include/aggressive_decoding.h.

Argument marshalling only: every step of the decoding path runs inside the CUDA library.  PyTorch
provides device memory (weights, workspace) and the stream.  There is no CPU fallback: if the shared
library is missing, importing this module's loader raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("AD_LIB_PATH", os.path.join(_HERE, "libad_b200.so"))

AD_OK, AD_ERR_ARG, AD_ERR_STATE, AD_ERR_CAPACITY, AD_ERR_TIMEOUT, AD_ERR_CUDA = 0, -1, -2, -3, -4, -5
AD_DTYPE_FP32, AD_DTYPE_BF16 = 0, 1
AD_MODE_IAD, AD_MODE_GAD = 0, 1
AD_CACHE_E4M3, AD_CACHE_INT8 = 0, 1

EXPORTS = [
    "ad_weight_counts", "ad_query_workspace", "ad_create", "ad_destroy", "ad_last_error", "ad_encode",
    "ad_verify_block", "ad_commit", "ad_force_commit", "ad_generate", "ad_draft_block", "ad_get_state", "ad_sync", "ad_set_acceptance",
    "ad_debug_logits", "ad_debug_encoder_memory", "ad_debug_stage_timeline", "ad_debug_profile_verify", "ad_vocab_argmax_scratch_bytes", "ad_vocab_argmax",
    "ad_vocab_argmax_static", "ad_debug_graph_count", "ad_debug_projection_shapes", "ad_debug_wait_probe", "ad_debug_grid_barrier_probe",
    "ad_linear", "ad_cache_append", "ad_cache_read", "ad_cache_attention_scratch_bytes", "ad_cache_attention", "ad_accept_sampled_scratch_bytes",
    "ad_accept_sampled",
]


class ModelCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("d_model", "n_heads", "d_ffn", "vocab", "n_enc", "n_dec", "dtype", "max_batch", "max_src",
                 "max_tgt", "kmax", "bos", "pad", "eos", "mask")] + [("ln_eps", C.c_float), ("has_drafter", C.c_int32)]


class ModelWeights(C.Structure):
    _fields_ = [("matrices", C.c_void_p), ("vectors", C.c_void_p)]


class Weights(C.Structure):
    _fields_ = [("ar", ModelWeights), ("nar", ModelWeights)]


class GenOpts(C.Structure):
    _fields_ = [("mode", C.c_int32), ("k", C.c_int32), ("max_len", C.c_void_p), ("draft_override", C.c_void_p),
                ("override_stride", C.c_int32), ("run_drafter", C.c_int32), ("sync_every", C.c_int32),
                ("use_graph", C.c_int32)]


class Stats(C.Structure):
    _fields_ = [("iterations", C.c_int64), ("row_iterations", C.c_int64), ("accepted", C.c_int64),
                ("offered", C.c_int64), ("device_ms", C.c_float), ("encode_ms", C.c_float),
                ("kernel_launches", C.c_int64)]


class KvCacheStruct(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_codes", "v_codes", "k_scale", "v_scale", "table")] + \
               [(n, C.c_int32) for n in ("table_stride", "n_blocks", "n_kv_heads", "block", "head_dim", "format")]


class AdError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"aggressive_decoding error {code}: {msg}")
        self.code = code


_lib = None


def load():
    """Loads the shared library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with paper_2205_10350_b200.build.build(); "
                          "there is no fallback path")
    lib = C.CDLL(LIB_PATH)
    vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
    cache, i64, f32 = C.POINTER(KvCacheStruct), C.c_int64, C.c_float
    sig = {
        "ad_weight_counts": (C.c_int, [C.POINTER(ModelCfg), C.POINTER(sz), C.POINTER(sz)]),
        "ad_query_workspace": (C.c_int, [C.POINTER(ModelCfg), C.POINTER(sz)]),
        "ad_create": (C.c_int, [C.POINTER(ModelCfg), C.POINTER(Weights), vp, sz, vp, C.POINTER(vp)]),
        "ad_destroy": (C.c_int, [vp]),
        "ad_last_error": (C.c_char_p, [vp]),
        "ad_encode": (C.c_int, [vp, vp, i32, vp, i32, i32]),
        "ad_verify_block": (C.c_int, [vp, vp, vp, vp, vp, i32]),
        "ad_commit": (C.c_int, [vp, vp, i32]),
        "ad_force_commit": (C.c_int, [vp, vp, vp, i32]),
        "ad_generate": (C.c_int, [vp, vp, i32, vp, i32, C.POINTER(GenOpts), vp, i32, vp, C.POINTER(Stats), i32]),
        "ad_draft_block": (C.c_int, [vp, i32, vp, vp, i32]),
        "ad_get_state": (C.c_int, [vp, vp, vp, vp]),
        "ad_sync": (C.c_int, [vp]),
        "ad_set_acceptance": (C.c_int, [vp, C.c_int32, C.c_float]),
        "ad_debug_logits": (C.c_int, [vp, i32, vp, sz]),
        "ad_debug_encoder_memory": (C.c_int, [vp, i32, vp, sz]),
        "ad_debug_stage_timeline": (C.c_int, [vp, vp, i32, vp]),
        "ad_debug_profile_verify": (C.c_int, [vp, vp, vp, vp, vp, i32, vp]),
        "ad_vocab_argmax_scratch_bytes": (sz, [i32, i32]),
        "ad_vocab_argmax": (C.c_int, [vp, vp, i32, i32, i32, i32, vp, vp, sz, vp, vp]),
        "ad_vocab_argmax_static": (C.c_int, [vp, vp, i32, i32, i32, i32, vp, vp, vp]),
        "ad_linear": (C.c_int, [vp, vp, vp, i32, i32, i32, i32, vp, vp, vp]),
        "ad_cache_append": (C.c_int, [cache, vp, vp, i32, i64, vp, vp, i32, i32, i32, vp, vp]),
        "ad_cache_read": (C.c_int, [cache, vp, vp, i32, vp, vp, i32, i32, i32, vp, vp]),
        "ad_cache_attention_scratch_bytes": (sz, [cache, i32, i32, i32, i32, i32]),
        "ad_cache_attention": (C.c_int, [cache, vp, i32, i64, i32, vp, vp, i32, i32, i32, i32, i32, f32, vp, vp, sz, vp, vp]),
        "ad_accept_sampled_scratch_bytes": (sz, [i32, i32, i32]),
        "ad_accept_sampled": (C.c_int, [vp, i64, vp, i64, i32, f32, i32, vp, vp, i32, i32, i32, vp, vp, i32, vp, vp, vp, sz, vp, vp]),
        "ad_debug_graph_count": (C.c_int, [vp, vp]),
        "ad_debug_projection_shapes": (C.c_int, [C.POINTER(ModelCfg), vp, i32, vp]),
        "ad_debug_wait_probe": (C.c_int, [vp, i32, vp, vp]),
        "ad_debug_grid_barrier_probe": (C.c_int, [i32, i32, i32, i32, vp, sz, vp, vp, vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    _lib = lib
    return lib


def _i32(a):
    return np.ascontiguousarray(a, dtype=np.int32)


def pack_weights(shape, w):
    """Lays one model's tensors out as the header documents: matrices [out, in] in one array, vectors in
    another.  Input convention: ``*.W`` is [in, out]."""
    mats, vecs = [w["emb"]], []
    T = lambda a: np.ascontiguousarray(np.asarray(a).T)
    cat = np.concatenate
    for l in range(shape.n_enc):
        p = f"enc.{l}"
        mats += [cat([T(w[f"{p}.self.{n}.W"]) for n in "qkv"], 0), T(w[f"{p}.self.o.W"]), T(w[f"{p}.ffn1.W"]),
                 T(w[f"{p}.ffn2.W"])]
        vecs += [cat([w[f"{p}.self.{n}.b"] for n in "qkv"]), w[f"{p}.self.o.b"], w[f"{p}.ln1.g"], w[f"{p}.ln1.b"],
                 w[f"{p}.ffn1.b"], w[f"{p}.ffn2.b"], w[f"{p}.ln2.g"], w[f"{p}.ln2.b"]]
    for l in range(shape.n_dec):
        p = f"dec.{l}"
        mats += [cat([T(w[f"{p}.self.{n}.W"]) for n in "qkv"], 0), T(w[f"{p}.self.o.W"]), T(w[f"{p}.cross.q.W"]),
                 cat([T(w[f"{p}.cross.{n}.W"]) for n in "kv"], 0), T(w[f"{p}.cross.o.W"]), T(w[f"{p}.ffn1.W"]),
                 T(w[f"{p}.ffn2.W"])]
        vecs += [cat([w[f"{p}.self.{n}.b"] for n in "qkv"]), w[f"{p}.self.o.b"], w[f"{p}.ln1.g"], w[f"{p}.ln1.b"],
                 w[f"{p}.cross.q.b"], cat([w[f"{p}.cross.{n}.b"] for n in "kv"]), w[f"{p}.cross.o.b"],
                 w[f"{p}.ln2.g"], w[f"{p}.ln2.b"], w[f"{p}.ffn1.b"], w[f"{p}.ffn2.b"], w[f"{p}.ln3.g"], w[f"{p}.ln3.b"]]
    m = cat([np.asarray(a, np.float32).ravel() for a in mats])
    v = cat([np.asarray(a, np.float32).ravel() for a in vecs])
    return m, v


class AggressiveDecoder:
    """One handle of the library: a verifier model (and optionally a drafter) with fixed capacities."""

    def __init__(self, shape, weights, nar_weights=None, max_batch=1, max_src=64, max_tgt=64, kmax=64,
                 bos=0, pad=1, eos=2, mask=3, ln_eps=1e-5, device="cuda:0", stream=None):
        import torch
        self.torch = torch
        self.lib = load()
        self.dev = torch.device(device)
        torch.cuda.set_device(self.dev)
        self.shape = shape
        self.bf16 = shape.dtype == "bf16"
        self.cfg = ModelCfg(shape.d_model, shape.n_heads, shape.d_ffn, shape.vocab, shape.n_enc, shape.n_dec,
                            AD_DTYPE_BF16 if self.bf16 else AD_DTYPE_FP32, max_batch, max_src, max_tgt, kmax,
                            bos, pad, eos, mask, ln_eps, 1 if nar_weights is not None else 0)
        self.max_batch, self.max_src, self.max_tgt, self.kmax = max_batch, max_src, max_tgt, kmax
        nm, nv = C.c_size_t(), C.c_size_t()
        self._check(self.lib.ad_weight_counts(C.byref(self.cfg), C.byref(nm), C.byref(nv)), None)
        self._keep = []
        wstruct = Weights()
        for field, ww in (("ar", weights), ("nar", nar_weights)):
            if ww is None:
                continue
            m, v = pack_weights(shape, ww)
            assert m.size == nm.value and v.size == nv.value, (m.size, nm.value, v.size, nv.value)
            mt = torch.from_numpy(m).to(self.dev)
            if self.bf16:
                mt = mt.to(torch.bfloat16)
            vt = torch.from_numpy(v).to(self.dev)
            self._keep += [mt, vt]
            setattr(wstruct, field, ModelWeights(mt.data_ptr(), vt.data_ptr()))
        nbytes = C.c_size_t()
        self._check(self.lib.ad_query_workspace(C.byref(self.cfg), C.byref(nbytes)), None)
        self.workspace_bytes = nbytes.value
        self.workspace = torch.empty(nbytes.value + 1024, dtype=torch.uint8, device=self.dev)
        base = (self.workspace.data_ptr() + 1023) // 1024 * 1024
        self.stream = stream if stream is not None else torch.cuda.Stream(device=self.dev)
        torch.cuda.synchronize(self.dev)   # weight uploads ran on torch's current stream
        sp = C.c_void_p(self.stream.cuda_stream)
        h = C.c_void_p()
        self._check(self.lib.ad_create(C.byref(self.cfg), C.byref(wstruct), C.c_void_p(base), nbytes.value, sp,
                                       C.byref(h)), None)
        self.h = h
        self.B = 0

    # ------------------------------------------------------------------ helpers
    def _check(self, rc, h):
        if rc != AD_OK:
            msg = self.lib.ad_last_error(h)
            raise AdError(rc, msg.decode() if msg else "")

    def close(self):
        if getattr(self, "h", None):
            self.lib.ad_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------------ host-array API
    def encode(self, src, src_len):
        src, src_len = _i32(src), _i32(src_len)
        self.B = src.shape[0]
        self._check(self.lib.ad_encode(self.h, src.ctypes.data, src.shape[1], src_len.ctypes.data, self.B, 1), self.h)

    def verify_block(self, drafts, k):
        """drafts [B, <=kmax] (host), k [B].  Returns (argmax [B, kmax], n_accepted [B])."""
        d = np.full((self.B, self.kmax), -1, np.int32)
        drafts = np.asarray(drafts, np.int32)
        d[:, : drafts.shape[1]] = drafts
        k = _i32(k)
        am = np.zeros((self.B, self.kmax), np.int32)
        n = np.zeros(self.B, np.int32)
        self._check(self.lib.ad_verify_block(self.h, d.ctypes.data, k.ctypes.data, am.ctypes.data, n.ctypes.data, 1), self.h)
        return am, n

    def commit(self, n=None):
        if n is None:
            self._check(self.lib.ad_commit(self.h, None, 1), self.h)
        else:
            n = _i32(n)
            self._check(self.lib.ad_commit(self.h, n.ctypes.data, 1), self.h)

    def force_commit(self, tokens, n):
        t = np.full((self.B, self.kmax), -1, np.int32)
        tokens = np.asarray(tokens, np.int32)
        t[:, : tokens.shape[1]] = tokens
        n = _i32(n)
        self._check(self.lib.ad_force_commit(self.h, t.ctypes.data, n.ctypes.data, 1), self.h)

    def draft_block(self, k_cap):
        d = np.zeros((self.B, self.kmax), np.int32)
        k = np.zeros(self.B, np.int32)
        self._check(self.lib.ad_draft_block(self.h, k_cap, d.ctypes.data, k.ctypes.data, 1), self.h)
        return d, k

    def state(self):
        ln, last, fin = (np.zeros(self.B, np.int32) for _ in range(3))
        self._check(self.lib.ad_get_state(self.h, ln.ctypes.data, last.ctypes.data, fin.ctypes.data), self.h)
        return ln, last, fin

    def sync(self):
        self._check(self.lib.ad_sync(self.h), self.h)

    def set_acceptance(self, beta, tau):
        """beta = 0: exact-match verification; beta >= 1: relaxed top-beta / tau verification."""
        self._check(self.lib.ad_set_acceptance(self.h, int(beta), float(tau)), self.h)

    def debug_logits(self, M, which=0):
        t = self.torch.empty((M, self.shape.vocab), dtype=self.torch.float32, device=self.dev)
        self._check(self.lib.ad_debug_logits(self.h, which, C.c_void_p(t.data_ptr()), t.numel()), self.h)
        self.sync()
        return t.cpu().numpy()

    def profile_verify(self, drafts, k, capacity=512):
        """One verification block with every kernel timed on its own: list of (what, microseconds) in launch order."""
        d = np.full((self.B, self.kmax), -1, np.int32)
        drafts = np.asarray(drafts, np.int32)
        d[:, : drafts.shape[1]] = drafts
        k = _i32(k)
        names = C.create_string_buffer(capacity * 64)
        us = np.zeros(capacity, np.float32)
        n = C.c_int32()
        self._check(self.lib.ad_debug_profile_verify(self.h, d.ctypes.data, k.ctypes.data, names, us.ctypes.data, capacity,
                                                     C.byref(n)), self.h)
        raw = names.raw
        return [(raw[i * 64: (i + 1) * 64].split(b"\0")[0].decode(), float(us[i])) for i in range(n.value)]

    def debug_graph_count(self):
        """Captured graphs that the handle keeps."""
        n = C.c_int32()
        self._check(self.lib.ad_debug_graph_count(self.h, C.byref(n)), self.h)
        return n.value

    def debug_stage_timeline(self):
        """Per-stage (inputs visible, signalled) global-timer stamps of the last persistent decoder pass, in ns."""
        buf = np.zeros(2 * (8 * self.shape.n_dec + 1), np.uint64)
        n = C.c_int32()
        self._check(self.lib.ad_debug_stage_timeline(self.h, buf.ctypes.data, buf.size, C.byref(n)), self.h)
        return buf.reshape(-1, 2)

    def debug_encoder_memory(self, b, src_len):
        t = self.torch.empty((src_len, self.shape.d_model), dtype=self.torch.float32, device=self.dev)
        self._check(self.lib.ad_debug_encoder_memory(self.h, b, C.c_void_p(t.data_ptr()), t.numel()), self.h)
        self.sync()
        return t.cpu().numpy()

    def generate(self, src, src_len, mode="IAD", k=1, max_len=None, draft_override=None, run_drafter=False,
                 sync_every=0, use_graph=True, out=None, out_len=None):
        """Host-array form of ad_generate.  Returns (list of per-row outputs, stats dict)."""
        src, src_len = _i32(src), _i32(src_len)
        B = src.shape[0]
        self.B = B
        opts = GenOpts()
        opts.mode = AD_MODE_GAD if mode == "GAD" else AD_MODE_IAD
        opts.k = k
        keep = []
        if max_len is not None:
            ml = _i32(max_len); keep.append(ml)
            opts.max_len = ml.ctypes.data
        if draft_override is not None:
            ov = _i32(draft_override); keep.append(ov)
            opts.draft_override = ov.ctypes.data
            opts.override_stride = ov.shape[1]
        opts.run_drafter = int(run_drafter)
        opts.sync_every = sync_every
        opts.use_graph = int(use_graph)
        if out is None:
            out = np.zeros((B, self.max_tgt), np.int32)
        if out_len is None:
            out_len = np.zeros(B, np.int32)
        st = Stats()
        self._check(self.lib.ad_generate(self.h, src.ctypes.data, src.shape[1], src_len.ctypes.data, B,
                                         C.byref(opts), out.ctypes.data, out.shape[1], out_len.ctypes.data,
                                         C.byref(st), 1), self.h)
        stats = {f[0]: getattr(st, f[0]) for f in Stats._fields_}
        return [out[b, : out_len[b]].copy() for b in range(B)], stats

    # ------------------------------------------------------------------ device-pointer API (no host copies)
    def generate_device(self, src_t, src_len_t, out_t, out_len_t, mode="IAD", k=1, max_len_t=None,
                        override_t=None, run_drafter=False, sync_every=0, use_graph=True):
        """Same call with every array already resident on the device (torch int32 tensors)."""
        opts = GenOpts()
        opts.mode = AD_MODE_GAD if mode == "GAD" else AD_MODE_IAD
        opts.k = k
        if max_len_t is not None:
            opts.max_len = max_len_t.data_ptr()
        if override_t is not None:
            opts.draft_override = override_t.data_ptr()
            opts.override_stride = override_t.shape[1]
        opts.run_drafter = int(run_drafter)
        opts.sync_every = sync_every
        opts.use_graph = int(use_graph)
        st = Stats()
        B = src_t.shape[0]
        self.B = B
        self._check(self.lib.ad_generate(self.h, C.c_void_p(src_t.data_ptr()), src_t.shape[1],
                                         C.c_void_p(src_len_t.data_ptr()), B, C.byref(opts),
                                         C.c_void_p(out_t.data_ptr()), out_t.shape[1],
                                         C.c_void_p(out_len_t.data_ptr()), C.byref(st), 0), self.h)
        return {f[0]: getattr(st, f[0]) for f in Stats._fields_}

    def verify_block_device(self, drafts_t, k_t, argmax_t, n_t):
        self._check(self.lib.ad_verify_block(self.h, C.c_void_p(drafts_t.data_ptr()), C.c_void_p(k_t.data_ptr()),
                                             C.c_void_p(argmax_t.data_ptr()), C.c_void_p(n_t.data_ptr()), 0), self.h)

    def commit_device(self, n_t=None):
        self._check(self.lib.ad_commit(self.h, C.c_void_p(n_t.data_ptr()) if n_t is not None else None, 0), self.h)


_stream = None          # (device, raw handle, stream object) of the last operator-level call


def _current_stream():
    """(stream object, raw handle) of torch's current stream.  torch.cuda.current_stream() builds an object on every call, a
    tenth of a short operator-level call's time; the raw handle costs next to nothing, so the object is only made anew when the
    handle is another one."""
    import torch
    global _stream
    dev = torch._C._cuda_getDevice()
    raw = torch._C._cuda_getCurrentRawStream(dev)
    last = _stream
    if last is None or last[0] != dev or last[1] != raw:
        last = _stream = (dev, raw, torch.cuda.current_stream())
    return last[2], raw


def vocab_argmax(x_t, emb_t, status_t=None):
    """Operator-level call: arg-max of x @ emb^T per row.  x_t [M, d], emb_t [V, d], both float32 or bfloat16.
    Returns when the result is complete."""
    import torch
    lib = load()
    M, d = x_t.shape
    V = emb_t.shape[0]
    dtype = AD_DTYPE_BF16 if x_t.dtype is torch.bfloat16 else AD_DTYPE_FP32
    nbytes = lib.ad_vocab_argmax_scratch_bytes(V, M)
    scratch = x_t.new_empty(nbytes + 256, dtype=torch.uint8)
    out = x_t.new_empty(M, dtype=torch.int32)
    stream, raw = _current_stream()
    rc = lib.ad_vocab_argmax(x_t.data_ptr(), emb_t.data_ptr(), dtype, M, d, V, out.data_ptr(), (scratch.data_ptr() + 255) // 256 * 256, nbytes,
                             status_t.data_ptr() if status_t is not None else None, raw)
    if rc != AD_OK:
        raise AdError(rc, "ad_vocab_argmax")
    stream.synchronize()
    return out


STATIC_SCRATCH_BYTES = 1 << 20


def vocab_argmax_static(x_t, emb_t, out_t, status_t=None):
    """Projection + arg-max for callers that must not allocate device memory at call time.

    Unlike :func:`vocab_argmax`, nothing is allocated here or inside the library: ``out_t`` (int32, [M]) is
    the caller's, and the scratch is an array built into the library (1 MiB per GPU).  Problems that need
    more are refused with ``AD_ERR_CAPACITY``.  Calls on one GPU share that array, so keep them on one
    stream; make the first call on a device outside any stream capture.  Asynchronous on torch's current
    stream."""
    import torch
    lib = load()
    M, d = x_t.shape
    dtype = AD_DTYPE_BF16 if x_t.dtype is torch.bfloat16 else AD_DTYPE_FP32
    rc = lib.ad_vocab_argmax_static(x_t.data_ptr(), emb_t.data_ptr(), dtype, M, d, emb_t.shape[0], out_t.data_ptr(),
                                    status_t.data_ptr() if status_t is not None else None, _current_stream()[1])
    if rc != AD_OK:
        msg = lib.ad_last_error(None)
        raise AdError(rc, msg.decode() if msg else "ad_vocab_argmax_static")
    return out_t


def linear(x_t, W_t, bias_t=None, status_t=None):
    """Operator-level call: y = x W^T + bias in FP32.  x_t [M, K], W_t [N, K].  Returns when the result is complete."""
    import torch
    lib = load()
    M, K = x_t.shape
    N = W_t.shape[0]
    dtype = AD_DTYPE_BF16 if x_t.dtype is torch.bfloat16 else AD_DTYPE_FP32
    y = x_t.new_empty((M, N), dtype=torch.float32)
    stream, raw = _current_stream()
    rc = lib.ad_linear(x_t.data_ptr(), W_t.data_ptr(), bias_t.data_ptr() if bias_t is not None else None, dtype, M, K, N, y.data_ptr(),
                       status_t.data_ptr() if status_t is not None else None, raw)
    if rc != AD_OK:
        raise AdError(rc, "ad_linear")
    stream.synchronize()
    return y


# ---------------------------------------------------------------------------------------------------------
# 8-bit key/value cache and sampled verification.  These calls are asynchronous on torch's current stream of the tensors' device, allocate
# results and scratch through torch, and can be captured into graphs.
# ---------------------------------------------------------------------------------------------------------
def _refuse(entry, why):
    raise AdError(AD_ERR_ARG, f"{entry}: {why}")


def _raise(lib, rc):
    msg = lib.ad_last_error(None)
    raise AdError(rc, msg.decode() if msg else "")


_TOO_LARGE = "sizes must lie between 0 and 2^31 - 1"


# Torch's names that a call needs, looked up once: an import statement and attribute lookups cost a call as much as its checks.
_INT32 = _FP32 = _BF16 = _get_device = _get_stream = None


def _names():
    import torch
    global _INT32, _FP32, _BF16, _get_device, _get_stream
    _INT32, _FP32, _BF16 = torch.int32, torch.float32, torch.bfloat16
    _get_device, _get_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _vector(t, n, dtype, dev):
    """Whether t is a contiguous vector of n numbers of dtype on CUDA device number dev."""
    return t.dtype is dtype and t.get_device() == dev and t.dim() == 1 and t.numel() == n and t.is_contiguous()


def _matrix(t, shape, dtype, dev):
    return t.dtype is dtype and t.get_device() == dev and t.shape == shape and t.is_contiguous()


def _status_pointer(entry, dev, status_t):
    if status_t is None:
        return None
    if not _vector(status_t, 1, _INT32, dev):
        _refuse(entry, f"the status is one int32 on device {dev}")
    return status_t.data_ptr()


def _call_on(dev, call, *args):
    """call(*args, raw stream) with device number dev current; the stream is torch's current one of that device."""
    if _get_device() == dev:
        return call(*args, _get_stream(dev))
    import torch
    with torch.cuda.device(dev):
        return call(*args, _get_stream(dev))


class KvCache:
    """Key/value cache in 8 bits: blocks of `block` tokens with one scale per head and block (format "e4m3" or "int8").

    table [rows, row_blocks] (int32, on the device) names the blocks of each row; without one, row b owns blocks
    b * row_blocks .. (b + 1) * row_blocks - 1.  `tensors` = (k_codes, v_codes, k_scale, v_scale) adopts existing memory; otherwise
    the cache is allocated here."""

    def __init__(self, n_blocks, n_kv_heads, head_dim, block=32, fmt="e4m3", table=None, row_blocks=None, device="cuda:0", tensors=None):
        import torch
        _names()
        entry = "KvCache"
        if fmt not in ("e4m3", "int8"):
            _refuse(entry, f"unknown format {fmt!r}")
        self.device = torch.device(device)
        if self.device.type != "cuda":
            _refuse(entry, "the cache lives on a CUDA device")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.fmt, self.n_blocks, self.n_kv_heads, self.head_dim, self.block = fmt, int(n_blocks), int(n_kv_heads), int(head_dim), int(block)
        dt = torch.float8_e4m3fn if fmt == "e4m3" else torch.int8
        shape = (self.n_blocks, self.n_kv_heads, self.block, self.head_dim)
        if tensors is None:
            codes = [torch.zeros(shape, dtype=torch.uint8, device=self.device).view(dt) for _ in range(2)]
            tensors = (*codes, *(torch.ones(shape[:2], dtype=torch.float32, device=self.device) for _ in range(2)))
        for t, want, s in zip(tensors, (dt, dt, torch.float32, torch.float32), (shape, shape, shape[:2], shape[:2])):
            if not _matrix(t, s, want, self.device.index):
                _refuse(entry, f"codes are contiguous {dt} {shape}, scales float32 {shape[:2]}, on {self.device}")
        self.k_codes, self.v_codes, self.k_scale, self.v_scale = tensors
        if row_blocks is None:
            row_blocks = table.shape[1] if table is not None else self.n_blocks
        if table is not None and not _matrix(table, (table.shape[0], row_blocks), torch.int32, self.device.index):
            _refuse(entry, f"the table is a contiguous int32 tensor [rows, {row_blocks}] on {self.device}")
        self.table, self.row_blocks = table, int(row_blocks)
        self.struct = KvCacheStruct(self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(),
                                    table.data_ptr() if table is not None else None, self.row_blocks, self.n_blocks, self.n_kv_heads, self.block,
                                    self.head_dim, AD_CACHE_E4M3 if fmt == "e4m3" else AD_CACHE_INT8)
        self._ref, self._dev = C.byref(self.struct), self.device.index
        self._table_rows = table.shape[0] if table is not None else 1 << 30
        self._scratch = {}              # sizes of a call -> bytes of scratch it needs

    def _batch(self, entry, off_t, len_t):
        """Rows of a batch: off_t [B + 1], len_t [B]."""
        B = len_t.numel()
        if not (_vector(len_t, B, _INT32, self._dev) and _vector(off_t, B + 1, _INT32, self._dev)):
            _refuse(entry, f"offsets and lengths are contiguous int32 tensors [B + 1] and [B] on {self.device}, got {tuple(off_t.shape)} and {tuple(len_t.shape)}")
        if self._table_rows < B:
            _refuse(entry, f"the table has {self._table_rows} rows, the batch {B}")
        return B

    def _tokens(self, entry, t, heads):
        """(type, tokens, numbers between them) of t [M, heads, head_dim], whose heads lie next to each other."""
        dtype = AD_DTYPE_BF16 if t.dtype is _BF16 else AD_DTYPE_FP32
        if dtype == AD_DTYPE_FP32 and t.dtype is not _FP32:
            _refuse(entry, f"{t.dtype} is neither float32 nor bfloat16")
        if t.dim() != 3 or t.get_device() != self._dev:
            _refuse(entry, f"wanted [tokens, {heads}, {self.head_dim}] on {self.device}, got {tuple(t.shape)} on {t.device}")
        M, h, d = t.shape
        if h != heads or d != self.head_dim:
            _refuse(entry, f"wanted [tokens, {heads}, {self.head_dim}], got {tuple(t.shape)}")
        between, per_head, one = t.stride()
        if one != 1 or (per_head != d and heads > 1):
            _refuse(entry, "the numbers of a token must lie next to each other")
        return dtype, M, between if M > 1 else heads * d


def cache_append(cache, k_t, v_t, off_t, len_t, max_new, status_t=None):
    """Writes k_t, v_t [M, n_kv_heads, head_dim] (float32 or bfloat16, views of a wider array as well) behind the len_t[b] tokens of every row."""
    entry, lib = "ad_cache_append", _lib or load()
    if max_new >> 31:
        _refuse(entry, _TOO_LARGE)
    B = cache._batch(entry, off_t, len_t)
    tokens = cache._tokens(entry, k_t, cache.n_kv_heads)
    if cache._tokens(entry, v_t, cache.n_kv_heads) != tokens:
        _refuse(entry, "keys and values must agree in type, shape and stride")
    dtype, M, stride = tokens
    rc = _call_on(cache._dev, lib.ad_cache_append, cache._ref, k_t.data_ptr(), v_t.data_ptr(), dtype, stride, off_t.data_ptr(), len_t.data_ptr(), B, M,
                  max_new, _status_pointer(entry, cache._dev, status_t))
    if rc != AD_OK:
        _raise(lib, rc)


def cache_read(cache, off_t, start_t, tokens, max_tokens, dtype=None, status_t=None):
    """Positions start_t[b] .. of every row, off_t[b + 1] - off_t[b] of them: (k, v) [tokens, n_kv_heads, head_dim] in dtype (default bfloat16).
    Tokens that no row covers are left uninitialised."""
    entry, lib = "ad_cache_read", _lib or load()
    if (tokens | max_tokens) >> 31:
        _refuse(entry, _TOO_LARGE)
    B = cache._batch(entry, off_t, start_t)
    dtype = dtype or _BF16
    if dtype is not _BF16 and dtype is not _FP32:
        _refuse(entry, f"{dtype} is neither float32 nor bfloat16")
    shape = (tokens, cache.n_kv_heads, cache.head_dim)
    k, v = cache.k_scale.new_empty(shape, dtype=dtype), cache.k_scale.new_empty(shape, dtype=dtype)
    rc = _call_on(cache._dev, lib.ad_cache_read, cache._ref, k.data_ptr(), v.data_ptr(), AD_DTYPE_BF16 if dtype is _BF16 else AD_DTYPE_FP32,
                  off_t.data_ptr(), start_t.data_ptr(), B, tokens, max_tokens, _status_pointer(entry, cache._dev, status_t))
    if rc != AD_OK:
        _raise(lib, rc)
    return k, v


def cache_attention(cache, q_t, off_t, len_t, max_new, max_keys, causal=True, scale=None, out=None, status_t=None):
    """Attention of q_t [M, n_heads, head_dim] over the cache; returns [M, n_heads, head_dim] in q_t's type (`out`, if given).  Causal: query i of
    row b sees len_t[b] + i + 1 positions (its block has been appended), otherwise all see len_t[b].  scale: head_dim ** -0.5 unless given."""
    entry, lib = "ad_cache_attention", _lib or load()
    if (max_new | max_keys) >> 31:
        _refuse(entry, _TOO_LARGE)
    B = cache._batch(entry, off_t, len_t)
    if q_t.dim() != 3:
        _refuse(entry, "queries are [tokens, heads, head_dim]")
    H = q_t.size(1)
    dtype, M, stride = cache._tokens(entry, q_t, H)
    if out is None:
        out = q_t.new_empty((M, H, cache.head_dim))
    elif not _matrix(out, q_t.shape, q_t.dtype, cache._dev):
        _refuse(entry, "the result is a contiguous tensor like the queries")
    sizes = (dtype, H, B, max_new, max_keys)
    nbytes = cache._scratch.get(sizes)
    if nbytes is None:
        nbytes = _call_on(cache._dev, lambda *a: lib.ad_cache_attention_scratch_bytes(*a[:-1]), cache._ref, *sizes)
        if len(cache._scratch) < 4096:
            cache._scratch[sizes] = nbytes
    scratch = off_t.new_empty((nbytes + 3) // 4) if nbytes else None       # (torch's allocations are 512-byte aligned)
    rc = _call_on(cache._dev, lib.ad_cache_attention, cache._ref, q_t.data_ptr(), dtype, stride, H, off_t.data_ptr(), len_t.data_ptr(), B, M, max_new,
                  max_keys, 1 if causal else 0, cache.head_dim ** -0.5 if scale is None else scale, out.data_ptr(),
                  scratch.data_ptr() if nbytes else None, nbytes, _status_pointer(entry, cache._dev, status_t))
    if rc != AD_OK:
        _raise(lib, rc)
    return out


_accept_scratch = {}     # (device, tokens, vocabulary, drafter) -> bytes


def accept_sampled(target_t, draft_t, drafts_t, off_t, u_t, r_t, temperature=1.0, eos=-1, status_t=None):
    """Sampled verification of drafts_t [B, kmax] against scores target_t [M, vocab] (and the drafter's, draft_t, or None for drafts that were not
    sampled) with uniform numbers u_t [B, kmax] and r_t [B].  Returns (tokens [B, kmax], n_accepted [B])."""
    entry, lib = "ad_accept_sampled", _lib or load()
    if _INT32 is None:
        _names()
    dev = target_t.get_device()
    dtype = AD_DTYPE_BF16 if target_t.dtype is _BF16 else AD_DTYPE_FP32
    if dev < 0 or target_t.dim() != 2 or drafts_t.dim() != 2 or (dtype == AD_DTYPE_FP32 and target_t.dtype is not _FP32):
        _refuse(entry, "scores are [tokens, vocab] on a CUDA device, in float32 or bfloat16, and drafts [rows, kmax]")
    shape = drafts_t.shape
    B, kmax = shape
    if not (_matrix(drafts_t, shape, _INT32, dev) and _vector(off_t, B + 1, _INT32, dev)):
        _refuse(entry, f"drafts and offsets are contiguous int32 tensors [B, kmax] and [B + 1] on device {dev}")
    if not (_matrix(u_t, shape, _FP32, dev) and _vector(r_t, B, _FP32, dev)):
        _refuse(entry, f"random numbers are contiguous float32 tensors [B, kmax] and [B] on device {dev}")
    M, V = target_t.shape
    if (M | V | B | kmax) >> 31:
        _refuse(entry, _TOO_LARGE)
    stride, one = target_t.stride()
    draft_stride, draft = V, None
    if draft_t is not None:
        if draft_t.dtype is not target_t.dtype or draft_t.shape != target_t.shape or draft_t.get_device() != dev:
            _refuse(entry, "the drafter's scores are like the verifier's in type, shape and place")
        draft_stride, draft_one = draft_t.stride()
        draft = draft_t.data_ptr()
        if draft_one != 1:
            one = draft_one
    if one != 1 and V > 1:
        _refuse(entry, "a row's scores must lie next to each other")
    if M < 2:
        stride = draft_stride = V
    sizes = (dev, M, V, draft_t is not None)
    nbytes = _accept_scratch.get(sizes)
    if nbytes is None:
        nbytes = _call_on(dev, lambda m, v, z, _: lib.ad_accept_sampled_scratch_bytes(m, v, 1 if z else 0), *sizes[1:])
        if len(_accept_scratch) < 4096:
            _accept_scratch[sizes] = nbytes
    tokens, count, scratch = drafts_t.new_empty(shape), off_t.new_empty(B), off_t.new_empty(max(1, nbytes // 4))
    rc = _call_on(dev, lib.ad_accept_sampled, target_t.data_ptr(), stride, draft, draft_stride, dtype, temperature, V, off_t.data_ptr(),
                  drafts_t.data_ptr(), kmax, B, M, u_t.data_ptr(), r_t.data_ptr(), eos, tokens.data_ptr(), count.data_ptr(), scratch.data_ptr(), nbytes,
                  _status_pointer(entry, dev, status_t))
    if rc != AD_OK:
        _raise(lib, rc)
    return tokens, count
