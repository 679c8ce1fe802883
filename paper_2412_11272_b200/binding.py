"""ctypes binding of libwf_encoder.so: argument marshalling only.

Every step of the encoding path runs inside the library's CUDA kernels; this module turns
torch tensors into pointers, keeps them alive, and raises on error codes.  PyTorch is used
for device memory and streams, nothing else.  There is no CPU fallback: if the shared
library is missing or cannot be loaded, importing the handle raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libwf_encoder.so")

WF_F32, WF_BF16 = 0, 1
STATUS = {0: "WF_OK", 1: "WF_ERR_INVALID_ARG", 2: "WF_ERR_TOO_SHORT", 3: "WF_ERR_TOO_LONG",
          4: "WF_ERR_CAPACITY", 5: "WF_ERR_CUDA", 6: "WF_ERR_DEVICE_TIMEOUT",
          7: "WF_ERR_UNSUPPORTED_ARCH", 8: "WF_ERR_UNIMPLEMENTED"}
N_KERNEL_CLASSES = 6
KERNEL_CLASSES = ("front_end", "layout", "conv_gemm", "layernorm", "block_gemm", "attention")


class WfError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"{STATUS.get(code, code)}: {message}")
        self.code = code
        self.status = STATUS.get(code, str(code))


class wf_config(C.Structure):
    _fields_ = [("n_mel", C.c_int), ("d_model", C.c_int), ("n_layer", C.c_int), ("n_head", C.c_int),
                ("d_mlp", C.c_int), ("n_ctx", C.c_int), ("hush_frames", C.c_int), ("dtype", C.c_int),
                ("max_batch", C.c_int), ("max_tokens", C.c_long), ("max_samples", C.c_long)]


_PP = C.POINTER(C.c_void_p)


class wf_weights(C.Structure):
    _fields_ = [("mel_fb", C.c_void_p), ("conv1_w", C.c_void_p), ("conv1_b", C.c_void_p),
                ("conv2_w", C.c_void_p), ("conv2_b", C.c_void_p),
                ("ln1_g", _PP), ("ln1_b", _PP), ("wq", _PP), ("bq", _PP), ("wk", _PP), ("wv", _PP),
                ("bv", _PP), ("wo", _PP), ("bo", _PP), ("ln2_g", _PP), ("ln2_b", _PP),
                ("w1", _PP), ("b1", _PP), ("w2", _PP), ("b2", _PP),
                ("lnp_g", C.c_void_p), ("lnp_b", C.c_void_p)]


class wf_decoder_config(C.Structure):
    _fields_ = [("n_head", C.c_int), ("n_kv_head", C.c_int), ("d_head", C.c_int), ("dtype", C.c_int), ("cache_format", C.c_int),
                ("page_size", C.c_int)]


class wf_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("n_pages", C.c_int)]


class wf_rows(C.Structure):
    _fields_ = [("n_seq", C.c_int), ("n_rows", C.c_int), ("cu_rows", C.c_void_p), ("start", C.c_void_p), ("page_table", C.c_void_p),
                ("table_stride", C.c_int)]


class wf_beam_state(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("row_bytes", C.c_long), ("stride_bytes", C.c_long)]


class wf_page_pool(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("state", C.c_void_p), ("n_pages", C.c_int)]


class wf_e4m3(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("ld", C.c_long), ("scale_ld", C.c_long)]


_PER_LAYER = ("ln1_g", "ln1_b", "wq", "bq", "wk", "wv", "bv", "wo", "bo", "ln2_g", "ln2_b",
              "w1", "b1", "w2", "b2")

EXPORTS = ("wf_encoder_create", "wf_logmel", "wf_encode", "wf_encode_raw_hush", "wf_encode_mel", "wf_encode_host", "wf_encode_host_async", "wf_encode_host_wait", "wf_check",
           "wf_encoder_destroy", "wf_last_error", "wf_profile_enable", "wf_profile_read",
           "wf_plan", "wf_gemm_bf16", "wf_gemm_resid_bf16", "wf_ln_fold", "wf_gemm_ln_bf16", "wf_selftest_wait_timeout", "wf_attention", "wf_cross_kv", "wf_dtw",
           "wf_streams_create", "wf_streams_destroy", "wf_streams_length", "wf_streams_push", "wf_encode_streams", "wf_attention_f32_static",
           "wf_beam_pruner_create", "wf_beam_pruner_step", "wf_beam_pruner_state", "wf_beam_pruner_destroy",
           "wf_decoder_create", "wf_decoder_destroy", "wf_decoder_last_error", "wf_cache_write", "wf_cache_read",
           "wf_tree_attention_workspace", "wf_tree_attention", "wf_selftest_attention_timeout", "wf_beam_select", "wf_beam_reorder",
           "wf_page_plan", "wf_draft_verify", "wf_draft_commit", "wf_quantise_e4m3", "wf_gemm_e4m3")

_lib = None


def load_library() -> C.CDLL:
    """Loads the shared library (building it is the job of ``paper_2412_11272_b200.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -m paper_2412_11272_b200.build`")
    lib = C.CDLL(LIB_PATH)
    vp, ip, lp = C.c_void_p, C.POINTER(C.c_int), C.POINTER(C.c_long)
    lib.wf_encoder_create.argtypes = [C.POINTER(wf_config), C.POINTER(wf_weights), vp, C.POINTER(vp)]
    lib.wf_logmel.argtypes = [vp, vp, lp, C.c_int, vp, lp, vp]
    lib.wf_encode.argtypes = [vp, vp, lp, C.c_int, vp, vp, ip, vp]
    lib.wf_encode_mel.argtypes = [vp, vp, lp, C.c_int, vp, vp, ip, vp]
    lib.wf_encode_raw_hush.argtypes = [vp, vp, lp, C.c_int, vp, C.c_int, vp, ip, vp]
    lib.wf_encode_host.argtypes = [vp, vp, lp, C.c_int, vp, vp, ip, vp]
    lib.wf_encode_host_async.argtypes = [vp, vp, lp, C.c_int, vp, vp, ip, vp, lp]
    lib.wf_encode_host_wait.argtypes = [vp, C.c_long]
    lib.wf_check.argtypes = [vp, vp]
    lib.wf_encoder_destroy.argtypes = [vp]
    lib.wf_last_error.argtypes = [vp]
    lib.wf_last_error.restype = C.c_char_p
    lib.wf_plan.argtypes = [C.POINTER(wf_config), lp, C.c_int, C.c_int, C.c_long, C.c_int, ip, lp, ip, C.c_int]
    lib.wf_selftest_wait_timeout.argtypes = [vp, C.c_uint, vp]
    lib.wf_profile_enable.argtypes = [vp, C.c_int]
    lib.wf_profile_read.argtypes = [vp, lp, C.POINTER(C.c_double)]
    lib.wf_gemm_bf16.argtypes = [vp, vp, vp, vp, vp, C.c_long, C.c_int, C.c_int, C.c_int, vp]
    lib.wf_gemm_resid_bf16.argtypes = [vp, vp, vp, vp, vp, vp, vp, C.c_long, C.c_int, C.c_int, vp]
    lib.wf_ln_fold.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, C.c_int, C.c_int, vp]
    lib.wf_gemm_ln_bf16.argtypes = [vp, vp, vp, vp, vp, vp, vp, C.c_long, C.c_int, C.c_int, C.c_int, vp]
    lib.wf_attention.argtypes = [vp, vp, ip, C.c_int, vp, vp]
    lib.wf_cross_kv.argtypes = [vp, vp, vp, vp, C.c_long, C.c_int, vp, vp]
    lib.wf_streams_create.argtypes = [vp, C.c_int, C.c_long, C.POINTER(vp)]
    lib.wf_streams_destroy.argtypes = [vp]
    lib.wf_streams_length.argtypes = [vp, C.c_int, lp]
    lib.wf_streams_push.argtypes = [vp, ip, C.c_int, vp, lp, lp, vp]
    lib.wf_encode_streams.argtypes = [vp, ip, C.c_int, vp, vp, ip, vp]
    lib.wf_dtw.argtypes = [vp, vp, ip, ip, C.c_int, vp, vp, vp, vp]
    lib.wf_attention_f32_static.argtypes = [vp, ip, C.c_int, C.c_int, vp, vp]
    lib.wf_beam_pruner_create.argtypes = [ip, C.c_int, C.POINTER(C.c_ubyte), C.c_int, C.c_int, C.POINTER(vp)]
    lib.wf_beam_pruner_step.argtypes = [vp, C.c_int]
    lib.wf_beam_pruner_state.argtypes = [vp, lp, ip, lp, lp]
    lib.wf_beam_pruner_destroy.argtypes = [vp]
    lib.wf_decoder_create.argtypes = [C.POINTER(wf_decoder_config), C.POINTER(vp)]
    lib.wf_decoder_destroy.argtypes = [vp]
    lib.wf_decoder_last_error.argtypes = [vp]
    lib.wf_decoder_last_error.restype = C.c_char_p
    cp, rp = C.POINTER(wf_cache), C.POINTER(wf_rows)
    lib.wf_cache_write.argtypes = [vp, cp, rp, vp, C.c_long, vp, C.c_long, vp, vp]
    lib.wf_cache_read.argtypes = [vp, cp, rp, vp, C.c_long, vp, C.c_long, vp, vp]
    lib.wf_tree_attention_workspace.argtypes = [vp, C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_size_t)]
    lib.wf_tree_attention.argtypes = [vp, cp, rp, vp, C.c_long, C.c_float, C.c_int, vp, C.c_int, C.c_int, C.c_int, vp, C.c_long, vp, vp,
                                      C.c_size_t, vp, vp]
    lib.wf_selftest_attention_timeout.argtypes = [vp, C.c_int]
    lib.wf_beam_select.argtypes = [vp, vp, C.c_int, C.c_long, C.c_int, C.c_int, C.c_int, vp, vp, vp, C.c_int, vp, C.c_int, vp, vp, vp, vp, vp, vp]
    lib.wf_beam_reorder.argtypes = [vp, vp, C.c_int, C.c_int, C.POINTER(wf_beam_state), C.c_int, cp, C.c_int, vp, C.c_int, vp, vp, vp]
    ci, cl = C.c_int, C.c_long
    lib.wf_page_plan.argtypes = [vp, C.POINTER(wf_page_pool), ci, vp, vp, vp, vp, vp, ci, ci, vp, vp, vp, vp, vp, vp]
    lib.wf_draft_verify.argtypes = [vp, vp, ci, cl, ci, ci, ci, ci, vp, vp, vp, vp, cl, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.wf_draft_commit.argtypes = [vp, ci, vp, vp, vp, ci, vp, cp, ci, vp, ci, vp, vp]
    lib.wf_quantise_e4m3.argtypes = [vp, vp, ci, cl, cl, ci, C.POINTER(wf_e4m3), vp]
    lib.wf_gemm_e4m3.argtypes = [vp, C.POINTER(wf_e4m3), C.POINTER(wf_e4m3), vp, vp, ci, cl, cl, ci, ci, ci, vp, vp]
    for name in EXPORTS:
        if name not in ("wf_last_error", "wf_decoder_last_error"):
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _stream_ptr(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def _longs(values):
    arr = np.ascontiguousarray(np.asarray(values, dtype=np.int64))
    return arr, arr.ctypes.data_as(C.POINTER(C.c_long))


class Encoder:
    """Owns one ``wf_encoder`` handle.  ``weights`` maps the names of
    ``inputs.encoder_weights`` to float32 arrays (numpy or torch); they are moved to the
    current CUDA device and may be released by the caller afterwards."""

    def __init__(self, shape, weights: dict, mel_fb, max_batch: int, max_tokens: int, max_samples: int,
                 hush_frames: int | None = None, n_ctx: int | None = None, dtype: str | None = None,
                 device="cuda:0"):
        self.lib = load_library()
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.shape = shape
        self.dtype = dtype or shape.dtype
        self.hush_frames = shape.hush_frames if hush_frames is None else hush_frames
        self.n_ctx = shape.n_ctx if n_ctx is None else n_ctx
        self.d_model = shape.d_model
        self.n_mel = shape.n_mel
        self.out_dtype = torch.bfloat16 if self.dtype == "bf16" else torch.float32
        cfg = wf_config(shape.n_mel, shape.d_model, shape.n_layer, shape.n_head, shape.d_mlp, self.n_ctx,
                        self.hush_frames, WF_BF16 if self.dtype == "bf16" else WF_F32,
                        int(max_batch), int(max_tokens), int(max_samples))
        dev = {}

        def put(a):
            t = torch.as_tensor(np.ascontiguousarray(a) if isinstance(a, np.ndarray) else a)
            return t.to(device=self.device, dtype=torch.float32).contiguous()

        w = wf_weights()
        for name in ("conv1_w", "conv1_b", "conv2_w", "conv2_b", "lnp_g", "lnp_b"):
            dev[name] = put(weights[name])
            setattr(w, name, dev[name].data_ptr())
        dev["mel_fb"] = put(mel_fb)
        w.mel_fb = dev["mel_fb"].data_ptr()
        arrays = {}
        for name in _PER_LAYER:
            arr = (C.c_void_p * max(shape.n_layer, 1))()
            for l in range(shape.n_layer):
                dev[f"{name}.{l}"] = put(weights[f"{name}.{l}"])
                arr[l] = dev[f"{name}.{l}"].data_ptr()
            arrays[name] = arr
            setattr(w, name, C.cast(arr, _PP))
        handle = C.c_void_p()
        st = self.lib.wf_encoder_create(C.byref(cfg), C.byref(w), _stream_ptr(), C.byref(handle))
        self.handle = handle
        if st != 0:
            msg = self.lib.wf_last_error(handle).decode() if handle else "create failed"
            if handle:
                self.lib.wf_encoder_destroy(handle)
            self.handle = None
            raise WfError(st, msg)
        torch.cuda.synchronize()
        del dev, arrays  # the library holds its own converted copies

    # -- helpers
    def _check(self, st: int):
        if st != 0:
            raise WfError(st, self.lib.wf_last_error(self.handle).decode())

    def close(self):
        if getattr(self, "handle", None):
            self.lib.wf_encoder_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- entry points (same names as the C ABI)
    def wf_logmel(self, audio: torch.Tensor, lengths, stream=None):
        """audio: float32 CUDA tensor of packed samples.  Returns (mel [sum T, n_mel] f32, frames)."""
        arr, ptr = _longs(lengths)
        B = len(arr)
        total_frames = int((arr // 160).sum())
        mel = torch.empty((total_frames, self.n_mel), dtype=torch.float32, device=self.device)
        frames = np.zeros(max(B, 1), dtype=np.int64)
        self._check(self.lib.wf_logmel(self.handle, audio.data_ptr() if B else None, ptr, B, mel.data_ptr(),
                                       frames.ctypes.data_as(C.POINTER(C.c_long)), _stream_ptr(stream)))
        return mel, frames[:B]

    def _tokens(self, frames):
        return (np.asarray(frames, dtype=np.int64) + self.hush_frames + 1) // 2

    def wf_encode(self, audio: torch.Tensor, lengths, hush_mel: torch.Tensor | None, out=None, stream=None):
        """Returns (hidden [sum n_i, d_model], cu_seqlens int32 numpy [B+1]).  No host sync."""
        arr, ptr = _longs(lengths)
        B = len(arr)
        M = int(self._tokens(arr // 160).sum())
        if out is None:
            out = torch.empty((M, self.d_model), dtype=self.out_dtype, device=self.device)
        cu = np.zeros(B + 1, dtype=np.int32)
        self._check(self.lib.wf_encode(self.handle, audio.data_ptr() if B else None, ptr, B,
                                       hush_mel.data_ptr() if hush_mel is not None else None,
                                       out.data_ptr(), cu.ctypes.data_as(C.POINTER(C.c_int)),
                                       _stream_ptr(stream)))
        return out, cu

    def wf_encode_raw_hush(self, audio: torch.Tensor, lengths, hush_audio: torch.Tensor, out=None, stream=None):
        """Hush word at raw-audio level: float32 CUDA samples appended (virtually) to every buffer."""
        arr, ptr = _longs(lengths)
        B = len(arr)
        hs = int(hush_audio.numel())
        M = int(self._tokens((arr + hs) // 160).sum())
        if out is None:
            out = torch.empty((M, self.d_model), dtype=self.out_dtype, device=self.device)
        cu = np.zeros(B + 1, dtype=np.int32)
        self._check(self.lib.wf_encode_raw_hush(self.handle, audio.data_ptr() if B else None, ptr, B,
                                                hush_audio.data_ptr(), hs, out.data_ptr(),
                                                cu.ctypes.data_as(C.POINTER(C.c_int)), _stream_ptr(stream)))
        return out, cu

    def wf_encode_mel(self, mel: torch.Tensor, frames, hush_mel, out=None, stream=None):
        arr, ptr = _longs(frames)
        B = len(arr)
        M = int(self._tokens(arr).sum())
        if out is None:
            out = torch.empty((M, self.d_model), dtype=self.out_dtype, device=self.device)
        cu = np.zeros(B + 1, dtype=np.int32)
        self._check(self.lib.wf_encode_mel(self.handle, mel.data_ptr() if B else None, ptr, B,
                                           hush_mel.data_ptr() if hush_mel is not None else None,
                                           out.data_ptr(), cu.ctypes.data_as(C.POINTER(C.c_int)),
                                           _stream_ptr(stream)))
        return out, cu

    def wf_encode_host(self, audio_host: torch.Tensor, lengths, hush_mel, out_host: torch.Tensor, stream=None):
        """audio_host / out_host: (pinned) CPU tensors.  Copies in, encodes, copies out, synchronises."""
        arr, ptr = _longs(lengths)
        B = len(arr)
        cu = np.zeros(B + 1, dtype=np.int32)
        self._check(self.lib.wf_encode_host(self.handle, audio_host.data_ptr(), ptr, B,
                                            hush_mel.data_ptr() if hush_mel is not None else None,
                                            out_host.data_ptr(), cu.ctypes.data_as(C.POINTER(C.c_int)),
                                            _stream_ptr(stream)))
        return out_host, cu

    def wf_encode_host_async(self, audio_host: torch.Tensor, lengths, hush_mel, out_host: torch.Tensor, stream=None):
        """As wf_encode_host without the wait: returns (ticket, cu_seqlens); out_host is valid after
        wf_encode_host_wait(ticket)."""
        arr, ptr = _longs(lengths)
        B = len(arr)
        cu = np.zeros(B + 1, dtype=np.int32)
        ticket = C.c_long(0)
        self._check(self.lib.wf_encode_host_async(self.handle, audio_host.data_ptr(), ptr, B,
                                                  hush_mel.data_ptr() if hush_mel is not None else None,
                                                  out_host.data_ptr(), cu.ctypes.data_as(C.POINTER(C.c_int)),
                                                  _stream_ptr(stream), C.byref(ticket)))
        return int(ticket.value), cu

    def wf_encode_host_wait(self, ticket: int):
        self._check(self.lib.wf_encode_host_wait(self.handle, ticket))

    def wf_check(self, stream=None):
        self._check(self.lib.wf_check(self.handle, _stream_ptr(stream)))

    def wf_selftest_wait_timeout(self, poll_limit: int = 4096, stream=None):
        self._check(self.lib.wf_selftest_wait_timeout(self.handle, poll_limit, _stream_ptr(stream)))

    def wf_profile_enable(self, on: bool):
        self._check(self.lib.wf_profile_enable(self.handle, 1 if on else 0))

    def wf_profile_read(self) -> dict:
        n = (C.c_long * N_KERNEL_CLASSES)()
        ms = (C.c_double * N_KERNEL_CLASSES)()
        self._check(self.lib.wf_profile_read(self.handle, n, ms))
        return {KERNEL_CLASSES[i]: {"launches": int(n[i]), "ms": float(ms[i])} for i in range(N_KERNEL_CLASSES)}

    def wf_gemm_bf16(self, A: torch.Tensor, W: torch.Tensor, bias: torch.Tensor, mode: int, C_out=None,
                     stream=None):
        M, K = A.shape
        N = W.shape[0]
        if C_out is None:
            C_out = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
        self._check(self.lib.wf_gemm_bf16(self.handle, A.data_ptr(), W.data_ptr(), bias.data_ptr(),
                                          C_out.data_ptr(), M, N, K, mode, _stream_ptr(stream)))
        return C_out

    def wf_gemm_resid_bf16(self, A: torch.Tensor, W: torch.Tensor, bias: torch.Tensor, x_hi: torch.Tensor,
                           x_lo: torch.Tensor, stream=None):
        """(x_hi, x_lo) <- split(x_hi + x_lo + A W^T + bias) in place; returns the row statistics
        [N / 128, M, 2] (sum and sum of squares of every 128 columns of the new x)."""
        M, K = A.shape
        N = W.shape[0]
        stats = torch.empty((max(N // 128, 1), M, 2), dtype=torch.float32, device=A.device)
        self._check(self.lib.wf_gemm_resid_bf16(self.handle, A.data_ptr(), W.data_ptr(), bias.data_ptr(), x_hi.data_ptr(),
                                                x_lo.data_ptr(), stats.data_ptr(), M, N, K, _stream_ptr(stream)))
        return stats

    def wf_ln_fold(self, W: torch.Tensor, ln_g: torch.Tensor, ln_b: torch.Tensor, bias: torch.Tensor | None, stream=None):
        """W float32 [N, K] -> (Wg bf16 [N, K], colsum float32 [N], cbias float32 [N])."""
        N, K = W.shape
        Wg = torch.empty((N, K), dtype=torch.bfloat16, device=W.device)
        colsum = torch.empty(N, dtype=torch.float32, device=W.device)
        cbias = torch.empty(N, dtype=torch.float32, device=W.device)
        self._check(self.lib.wf_ln_fold(self.handle, W.data_ptr(), ln_g.data_ptr(), ln_b.data_ptr(),
                                        bias.data_ptr() if bias is not None else None, Wg.data_ptr(), colsum.data_ptr(),
                                        cbias.data_ptr(), N, K, _stream_ptr(stream)))
        return Wg, colsum, cbias

    def wf_gemm_ln_bf16(self, x_hi: torch.Tensor, stats: torch.Tensor, Wg: torch.Tensor, colsum: torch.Tensor,
                        cbias: torch.Tensor, gelu: bool, stream=None):
        """C bf16 [M, N] = (gelu of) LayerNorm(x) W^T + bias from x_hi, the row statistics of x and folded weights."""
        M, K = x_hi.shape
        N = Wg.shape[0]
        out = torch.empty((M, N), dtype=torch.bfloat16, device=x_hi.device)
        self._check(self.lib.wf_gemm_ln_bf16(self.handle, x_hi.data_ptr(), stats.data_ptr(), Wg.data_ptr(), colsum.data_ptr(),
                                             cbias.data_ptr(), out.data_ptr(), M, N, K, 1 if gelu else 0, _stream_ptr(stream)))
        return out

    def wf_cross_kv(self, hidden: torch.Tensor, W_kv: torch.Tensor, b_kv: torch.Tensor, kv_out=None, stream=None):
        """hidden [M, d], W_kv [n_dec * 2 d, d] (path dtype), b_kv float32 [n_dec * 2 d] -> kv [M, n_dec * 2 d]."""
        M, d = hidden.shape
        n_dec = W_kv.shape[0] // (2 * d)
        if kv_out is None:
            kv_out = torch.empty((M, W_kv.shape[0]), dtype=hidden.dtype, device=hidden.device)
        self._check(self.lib.wf_cross_kv(self.handle, hidden.data_ptr(), W_kv.data_ptr(), b_kv.data_ptr(), M, n_dec,
                                         kv_out.data_ptr(), _stream_ptr(stream)))
        return kv_out

    def wf_dtw(self, cost: torch.Tensor, n_tokens, n_frames, stream=None):
        """cost: float32 CUDA tensor holding the B matrices back to back.  Returns
        (token_start int32 [sum n_tokens], total_cost float32 [B]) as CUDA tensors."""
        nt = np.ascontiguousarray(np.asarray(n_tokens, dtype=np.int32))
        nf = np.ascontiguousarray(np.asarray(n_frames, dtype=np.int32))
        B = len(nt)
        cells = int((nt.astype(np.int64) * nf).sum())
        trace = torch.empty(max(cells, 1), dtype=torch.uint8, device=cost.device)
        start = torch.empty(max(int(nt.sum()), 1), dtype=torch.int32, device=cost.device)
        total = torch.empty(max(B, 1), dtype=torch.float32, device=cost.device)
        ip = C.POINTER(C.c_int)
        self._check(self.lib.wf_dtw(self.handle, cost.data_ptr(), nt.ctypes.data_as(ip), nf.ctypes.data_as(ip), B,
                                    trace.data_ptr(), start.data_ptr(), total.data_ptr(), _stream_ptr(stream)))
        return start[:int(nt.sum())], total[:B]

    def wf_attention(self, qkv: torch.Tensor, cu_seqlens, stream=None):
        cu = np.ascontiguousarray(np.asarray(cu_seqlens, dtype=np.int32))
        out = torch.empty((qkv.shape[0], self.d_model), dtype=qkv.dtype, device=qkv.device)
        self._check(self.lib.wf_attention(self.handle, qkv.data_ptr(), cu.ctypes.data_as(C.POINTER(C.c_int)),
                                          len(cu) - 1, out.data_ptr(), _stream_ptr(stream)))
        return out


def wf_plan(shape, lengths, hush_frames: int, max_batch: int, max_tokens: int, max_samples: int, frames_given=False,
            tail_samples: int = 0, num_sms: int = 148, n_ctx=None):
    """The host-side planner alone (no GPU): returns (cu_seqlens, totals dict, attention work list)."""
    lib = load_library()
    cfg = wf_config(shape.n_mel, shape.d_model, shape.n_layer, shape.n_head, shape.d_mlp, n_ctx or shape.n_ctx, hush_frames,
                    1 if shape.dtype == "bf16" else 0, max_batch, max_tokens, max_samples)
    B = len(lengths)
    arr, ptr = _longs(lengths)
    cu = (C.c_int * (B + 1))()
    totals = (C.c_long * 6)()
    cap = 8 * (max_tokens // 16 + B + 4) + 4 * (max_tokens // 128 + 2 * B + 2) * max(shape.n_head, 1)
    work = (C.c_int * cap)()
    st = lib.wf_plan(C.byref(cfg), ptr, B, 1 if frames_given else 0, tail_samples, num_sms, cu, totals, work, cap)
    if st != 0:
        raise WfError(st, "wf_plan rejected the batch")
    names = ("frames", "padded_rows", "tokens", "front_end_tiles", "attention_entries", "attention_items")
    t = dict(zip(names, [int(v) for v in totals]))
    n = (2 * t["attention_entries"]) if shape.dtype != "bf16" else (3 * t["attention_entries"] + t["attention_items"])
    return np.array(cu[:B + 1]), t, np.array(work[:n])


def wf_attention_f32_static(qkv: torch.Tensor, cu_seqlens, d_model: int, out: torch.Tensor, stream=None):
    """Handle-free float32 attention that makes no allocation of its own: the caller passes the
    output tensor too.  For code that may not call cudaMalloc (see the header).  Raises WfError."""
    lib = load_library()
    cu = np.ascontiguousarray(np.asarray(cu_seqlens, dtype=np.int32))
    st = lib.wf_attention_f32_static(qkv.data_ptr(), cu.ctypes.data_as(C.POINTER(C.c_int)), len(cu) - 1,
                                     int(d_model), out.data_ptr(), _stream_ptr(stream))
    if st != 0:
        raise WfError(st, "wf_attention_f32_static rejected its arguments or a CUDA call failed")
    return out


class Streams:
    """Resident windows of ``n_streams`` audio streams on an encoder's device (``wf_streams_*``)."""

    def __init__(self, enc: Encoder, n_streams: int, max_window_samples: int):
        self.enc = enc
        self.handle = C.c_void_p()
        enc._check(enc.lib.wf_streams_create(enc.handle, n_streams, max_window_samples, C.byref(self.handle)))

    def close(self):
        if self.handle:
            self.enc.lib.wf_streams_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def wf_streams_length(self, stream_id: int) -> int:
        n = C.c_long()
        self.enc._check(self.enc.lib.wf_streams_length(self.handle, stream_id, C.byref(n)))
        return n.value

    def wf_streams_push(self, ids, new_audio: torch.Tensor | None, n_new, trim=None, stream=None):
        """Drops ``trim[i]`` samples at the front of stream ``ids[i]`` and appends ``n_new[i]`` samples
        taken back to back from ``new_audio`` (float32 CUDA)."""
        idv = np.ascontiguousarray(np.asarray(ids, dtype=np.int32))
        nn, nn_ptr = _longs(n_new)
        tr_ptr = None
        if trim is not None:
            tr, tr_ptr = _longs(trim)
        self.enc._check(self.enc.lib.wf_streams_push(
            self.handle, idv.ctypes.data_as(C.POINTER(C.c_int)), len(idv),
            new_audio.data_ptr() if new_audio is not None and new_audio.numel() else None, nn_ptr, tr_ptr,
            _stream_ptr(stream)))

    def wf_encode_streams(self, ids, hush_mel: torch.Tensor | None, out=None, stream=None):
        """Encodes the current windows of the listed streams; returns (hidden, cu_seqlens)."""
        enc = self.enc
        idv = np.ascontiguousarray(np.asarray(ids, dtype=np.int32))
        B = len(idv)
        frames = np.array([self.wf_streams_length(int(i)) // 160 for i in idv], dtype=np.int64)
        M = int(enc._tokens(frames).sum()) if B else 0
        if out is None:
            out = torch.empty((M, enc.d_model), dtype=enc.out_dtype, device=enc.device)
        cu = np.zeros(B + 1, dtype=np.int32)
        enc._check(enc.lib.wf_encode_streams(self.handle, idv.ctypes.data_as(C.POINTER(C.c_int)), B,
                                             hush_mel.data_ptr() if hush_mel is not None else None, out.data_ptr(),
                                             cu.ctypes.data_as(C.POINTER(C.c_int)), _stream_ptr(stream)))
        return out, cu


class BeamPruner:
    """Marshals the host-side beam-pruning state machine (wf_beam_pruner_*)."""

    def __init__(self, reference, is_special, full_beam: int = 5):
        self.lib = load_library()
        ref = np.ascontiguousarray(np.asarray(reference, dtype=np.int32))
        flags = np.ascontiguousarray(np.asarray(is_special, dtype=np.uint8))
        h = C.c_void_p()
        st = self.lib.wf_beam_pruner_create(ref.ctypes.data_as(C.POINTER(C.c_int)), len(ref),
                                            flags.ctypes.data_as(C.POINTER(C.c_ubyte)), len(flags), int(full_beam),
                                            C.byref(h))
        if st != 0:
            raise WfError(st, "wf_beam_pruner_create rejected its arguments")
        self.handle = h

    def step(self, top1: int) -> int:
        r = self.lib.wf_beam_pruner_step(self.handle, int(top1))
        if r < 0:
            raise WfError(1, "wf_beam_pruner_step: token id outside the vocabulary")
        return r

    def state(self):
        idx, rounds, ones, fb = C.c_long(), C.c_long(), C.c_long(), C.c_int()
        self.lib.wf_beam_pruner_state(self.handle, C.byref(idx), C.byref(fb), C.byref(rounds), C.byref(ones))
        return {"reference_index": idx.value, "fallen_back": bool(fb.value), "rounds": rounds.value,
                "rounds_at_one": ones.value}

    def close(self):
        if getattr(self, "handle", None):
            self.lib.wf_beam_pruner_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- operators of the decoding stage

TAILS = {"none": 0, "causal": 1, "mask": 2, "tree": 2}
CACHE_FORMATS = {"path": 0, "e4m3": 1, "int8": 2}
STATUS_BAD_PAGE, STATUS_BAD_ROWS, STATUS_BAD_PARENT, STATUS_GAVE_UP, STATUS_PUT_OFF, STATUS_BAD_VALUE = 1, 2, 4, 8, 16, 32
_INT, _U8, _F32, _BF16, _E4M3 = torch.int32, torch.uint8, torch.float32, torch.bfloat16, torch.float8_e4m3fn


def _refuse(message: str):
    raise WfError(1, message)


def _vector(t, name: str, device, dtype=_INT, n: int | None = None):
    """Checks a contiguous device array of one type (and at least ``n`` elements); returns its address."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or not t.is_contiguous() or t.device != device:
        _refuse(f"{name} must be a contiguous {dtype} tensor on {device}")
    if n is not None and t.numel() < n:
        _refuse(f"{name} has {t.numel()} elements, {n} are needed")
    return t.data_ptr()


class KvCache:
    """One decoder layer's paged keys and values: tensors the caller owns (see ``Decoder.cache``).
    k, v: [n_pages, n_kv_head, page_size, d_head]; k_scale, v_scale: bfloat16 [n_pages, n_kv_head, page_size], None for a
    cache of the path's own type.  It stands for the tensors' memory as it is when it is made: their contents may change, but they are
    not exchanged, and one that is resized or set to another storage needs another KvCache."""

    __slots__ = ("k", "v", "k_scale", "v_scale", "device", "shape", "c", "raw", "kind")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None, v_scale: torch.Tensor | None = None):
        if k.shape != v.shape or k.dim() != 4 or k.dtype != v.dtype or k.device != v.device:
            _refuse("k and v must be alike: [n_pages, n_kv_head, page_size, d_head]")
        if not (k.is_contiguous() and v.is_contiguous()):
            _refuse("cache pages must be contiguous")
        if (k_scale is None) != (v_scale is None):
            _refuse("k_scale and v_scale go together")
        for s in (k_scale, v_scale):
            if s is not None and (s.shape != k.shape[:3] or s.dtype != _BF16 or s.device != k.device or not s.is_contiguous()):
                _refuse("scales must be contiguous bfloat16 [n_pages, n_kv_head, page_size] beside their pages")
        c = wf_cache(k.data_ptr(), v.data_ptr(), None if k_scale is None else k_scale.data_ptr(),
                     None if v_scale is None else v_scale.data_ptr(), k.shape[0])
        kind = (*k.shape[1:], k.dtype, k_scale is not None, k.device.type)  # what a decoder compares with its own
        for name, value in zip(self.__slots__, (k, v, k_scale, v_scale, k.device, tuple(k.shape), c, bytes(c), kind)):
            object.__setattr__(self, name, value)

    def __setattr__(self, name, value):  # the descriptor holds the tensors' addresses
        raise AttributeError(f"{name} of a KvCache is fixed: make another KvCache for other tensors")

    def __delattr__(self, name):
        self.__setattr__(name, None)


class PagePool:
    """Free pages of a cache (see ``Decoder.page_pool``): a ring of page numbers, int32 [n_pages], and its state, int32 (head,
    count).  Both are updated in place by ``wf_page_plan``; the tensors stay the caller's."""

    __slots__ = ("pages", "state", "device")

    def __init__(self, pages: torch.Tensor, state: torch.Tensor):
        _vector(pages, "pages", pages.device)
        _vector(state, "state", pages.device, n=2)
        if pages.dim() != 1 or pages.numel() < 1:
            _refuse("pages must be a vector of at least one page number")
        self.pages, self.state, self.device = pages, state, pages.device


class ScaledCodes:
    """A matrix [rows, k] in 8 bits: e4m3 ``codes`` (rows 16-byte aligned) and ``scales``, uint8 [ceil(k / 512), rows, 4]: byte b at
    [j, r, i] stands for 2^(b - 127), the scale of row r's channels 128 (4 j + i) and the 127 behind them.  Made by
    ``Decoder.wf_quantise_e4m3``, or from codes of other origin by ``pack``.
    It stands for the tensors' memory as it is when it is made, as a KvCache does."""

    __slots__ = ("_codes", "_scales", "_memory", "shape", "device", "c")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        if codes.dim() != 2 or codes.dtype is not _E4M3 or codes.shape[1] < 1 or (codes.stride(1) != 1 and codes.shape[1] > 1):
            _refuse("codes must be float8_e4m3fn [rows, k], a row's elements contiguous")
        rows, k = codes.shape
        if scales.dtype is not _U8 or scales.device != codes.device or scales.shape != ((k + 511) // 512, rows, 4) or \
                (rows > 0 and (scales.stride(2) != 1 or (rows > 1 and scales.stride(1) != 4) or (k > 512 and scales.stride(0) % 4))):
            _refuse("scales must be uint8 [ceil(k / 512), rows, 4] beside their codes, the words of consecutive rows side by side")
        self._codes, self._scales, self._memory, self.shape, self.device = codes, scales, None, (rows, k), codes.device
        self.c = wf_e4m3(codes.data_ptr(), scales.data_ptr(), codes.stride(0) if rows > 1 else (k + 15) // 16 * 16,
                         scales.stride(0) // 4 if k > 512 else max(rows, 1)) if self.device.type == "cuda" else None

    @classmethod
    def _within(cls, memory: torch.Tensor, rows: int, k: int, device):
        """Codes (rows padded to 16 bytes) and, behind them, scales in bytes of one tensor; the views of it are made when they are asked for."""
        self, ld = cls.__new__(cls), (k + 15) // 16 * 16
        self._codes = self._scales = None
        self._memory, self.shape, self.device = memory, (rows, k), device
        at = memory.data_ptr()
        self.c = wf_e4m3(at, at + rows * ld, ld, rows) if device.type == "cuda" else None
        return self

    @staticmethod
    def _bytes(rows: int, k: int) -> int:
        return rows * ((k + 15) // 16 * 16 + (k + 511) // 512 * 4)

    @property
    def codes(self) -> torch.Tensor:
        if self._codes is None:
            (rows, k), ld = self.shape, self.c.ld if self.c else (self.shape[1] + 15) // 16 * 16
            self._codes = self._memory[:rows * ld].view(_E4M3).view(rows, ld)[:, :k]
        return self._codes

    @property
    def scales(self) -> torch.Tensor:
        if self._scales is None:
            rows, k = self.shape
            self._scales = self._memory[rows * ((k + 15) // 16 * 16):].view((k + 511) // 512, rows, 4)
        return self._scales

    def __getitem__(self, rows: slice):
        """Some of the rows."""
        if not isinstance(rows, slice) or rows.step not in (None, 1):
            _refuse("rows are taken by a slice without a step")
        return ScaledCodes(self.codes[rows], self.scales[:, rows])

    @classmethod
    def empty(cls, rows: int, k: int, device="cuda"):
        """Room for a matrix, rows padded to 16 bytes."""
        memory = torch.empty(cls._bytes(rows, k), dtype=_U8, device=device)
        return cls._within(memory, rows, k, memory.device)

    @classmethod
    def pack(cls, codes: torch.Tensor, scales: torch.Tensor):
        """Codes [rows, k] with scales as numbers: powers of two (or NaN), [rows, ceil(k / 128)], or one for each 128 x 128 block,
        [ceil(rows / 128), ceil(k / 128)].  For weights, once: it waits for the device (the scales' values are checked) and cannot be captured."""
        rows, k = codes.shape
        blocks = (k + 127) // 128
        if scales.dim() != 2 or scales.shape[1] != blocks or scales.shape[0] not in (rows, (rows + 127) // 128):
            _refuse(f"scales must be [{rows} or {(rows + 127) // 128}, {blocks}] for these codes")
        mantissa, exponent = torch.frexp(scales.float())
        if not bool(((mantissa == 0.5) | scales.isnan()).all()) or not bool((((exponent >= -125) & (exponent <= 128)) | scales.isnan()).all()):
            _refuse("scales must be powers of two from 2^-126 to 2^127")
        byte = torch.where(scales.isnan(), 255, exponent + 126).to(_U8)
        if scales.shape[0] != rows:
            byte = byte.repeat_interleave(128, dim=0)[:rows]
        out = cls.empty(rows, k, codes.device)
        out.codes.view(_U8).copy_(codes.view(_U8))
        words = torch.full((rows, out.scales.shape[0] * 4), 127, dtype=_U8, device=codes.device)
        words[:, :blocks] = byte
        out.scales.copy_(words.view(rows, -1, 4).transpose(0, 1))
        return out

    def values(self) -> torch.Tensor:
        """What the matrix stands for, in float32."""
        rows, k = self.shape
        b = self.scales.transpose(0, 1).reshape(rows, -1)
        s = torch.exp2(b.double() - 127).float().masked_fill(b == 255, float("nan"))
        return self.codes.float() * s.repeat_interleave(128, dim=1)[:, :k]


class Decoder:
    """Owns one ``wf_decoder`` handle: the heads, element types and page size of a decoder's attention.  The handle
    holds no device memory; creating one needs no GPU.  Device arrays are int32 unless stated; every method enqueues
    on ``stream`` (default: the current stream of the tensors' device) and returns without synchronising.  ``status``
    (an int32 device tensor of one element, zeroed by the caller) collects what kernels find wrong in device arrays."""

    def __init__(self, n_head: int, n_kv_head: int | None = None, d_head: int = 64, dtype: str = "bf16", cache_format: str = "path",
                 page_size: int = 64):
        self.handle = None
        self._workspace_bytes = {}
        self.lib = load_library()
        if dtype not in ("bf16", "f32") or cache_format not in CACHE_FORMATS:
            _refuse(f"dtype is bf16 or f32, cache_format one of {', '.join(CACHE_FORMATS)}")
        self.n_head, self.n_kv_head, self.d_head, self.page_size = int(n_head), int(n_kv_head or n_head), int(d_head), int(page_size)
        self.dtype, self.cache_format = dtype, cache_format
        self.torch_dtype = _BF16 if dtype == "bf16" else _F32
        self.code_dtype = {"path": self.torch_dtype, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}[cache_format]
        self._kind = (self.n_kv_head, self.page_size, self.d_head, self.code_dtype, cache_format != "path", "cuda")
        cfg = wf_decoder_config(self.n_head, self.n_kv_head, self.d_head, WF_BF16 if dtype == "bf16" else WF_F32,
                                CACHE_FORMATS[cache_format], self.page_size)
        handle = C.c_void_p()
        st = self.lib.wf_decoder_create(C.byref(cfg), C.byref(handle))
        self.handle = handle
        if st != 0:
            msg = self.lib.wf_decoder_last_error(handle).decode() if handle else "create failed"
            self.close()
            raise WfError(st, msg)

    def _check(self, st: int):
        if st != 0:
            raise WfError(st, self.lib.wf_decoder_last_error(self.handle).decode())

    def close(self):
        if getattr(self, "handle", None):
            self.lib.wf_decoder_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- helpers
    def cache(self, n_pages: int, device="cuda") -> KvCache:
        """A zeroed cache of ``n_pages`` pages for one layer."""
        shape = (n_pages, self.n_kv_head, self.page_size, self.d_head)
        k, v = (torch.zeros(shape, dtype=torch.uint8 if self.code_dtype.itemsize == 1 else self.code_dtype, device=device).view(self.code_dtype)
                for _ in range(2))
        if self.cache_format == "path":
            return KvCache(k, v)
        return KvCache(k, v, *(torch.ones(shape[:3], dtype=_BF16, device=device) for _ in range(2)))

    def _cache(self, cache: KvCache):
        if cache.kind == self._kind:
            return cache.c
        if cache.shape[1:] != (self.n_kv_head, self.page_size, self.d_head) or cache.k.dtype != self.code_dtype:
            _refuse(f"the cache is {cache.k.dtype} {cache.shape}, this decoder's pages are {self.code_dtype} "
                    f"[n, {self.n_kv_head}, {self.page_size}, {self.d_head}]")
        if (cache.k_scale is None) != (self.cache_format == "path"):
            _refuse("scales belong to quantised caches, and only to them")
        if cache.device.type != "cuda":
            _refuse("the cache must be in device memory")
        return cache.c

    def _caches(self, caches, device):
        """The descriptors of several layers' caches, one behind the other."""
        for c in caches:
            if c.kind != self._kind:
                self._cache(c)
            if c.device != device:
                _refuse("a cache is on another device than the call's arrays")
        return (wf_cache * len(caches)).from_buffer_copy(b"".join([c.raw for c in caches])) if caches else (wf_cache * 0)()

    def _rows(self, page_table, cu_rows, start, n_rows, device):
        n_seq, shape = cu_rows.numel() - 1, page_table.shape
        if n_seq < 0 or len(shape) != 2 or shape[0] < n_seq:
            _refuse("cu_rows has n_seq + 1 entries, page_table [n_seq, pages]")
        return wf_rows(n_seq, n_rows, _vector(cu_rows, "cu_rows", device), _vector(start, "start", device, n=n_seq),
                       _vector(page_table, "page_table", device), shape[1])

    def _vectors(self, t, name, device, heads):
        """A [n, heads, d_head] tensor with contiguous rows: (address, row stride)."""
        shape, d = t.shape, self.d_head
        if len(shape) != 3 or t.dtype is not self.torch_dtype or shape[1] != heads or shape[2] != d or t.device != device:
            _refuse(f"{name} must be {self.torch_dtype} [rows, {heads}, {d}] on {device}")
        if t.is_contiguous():
            return t.data_ptr(), heads * d
        s = t.stride()
        if s[2] != 1 or (heads > 1 and s[1] != d):
            _refuse(f"{name}: the heads of a row must lie one after the other")
        return t.data_ptr(), s[0] if shape[0] > 1 else max(s[0], heads * d)

    @staticmethod
    def _empty(like, shape, dtype, stream):
        """Memory beside ``like`` for a call on ``stream``: the allocator then gives it to nobody else before that stream is
        done with it."""
        if stream is None:  # (the shorter way where the type is the same)
            return like.new_empty(shape) if like.dtype is dtype else torch.empty(shape, dtype=dtype, device=like.device)
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=like.device)

    @staticmethod
    def _status(status, device):
        return None if status is None else _vector(status, "status", device, n=1)

    def _call(self, fn, device, stream, *args):
        """Runs one entry point with the tensors' device current, on its stream."""
        index = device.index
        if torch._C._cuda_getDevice() != index:
            with torch.cuda.device(device):
                return self._call(fn, device, stream, *args)
        st = fn(self.handle, *args, stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(index))
        if st != 0:
            self._check(st)

    # -- entry points (same names as the C ABI)
    def wf_cache_write(self, cache: KvCache, page_table, cu_rows, start, k: torch.Tensor, v: torch.Tensor, status=None, stream=None):
        """Stores keys and values [n, n_kv_head, d_head] of new rows (row stride free) at their sequences' positions
        start[s], start[s] + 1, ..."""
        c, device = self._cache(cache), cache.device
        if k.shape[0] != v.shape[0]:
            _refuse("k and v have different numbers of rows")
        (kp, ks), (vp, vs) = self._vectors(k, "k", device, self.n_kv_head), self._vectors(v, "v", device, self.n_kv_head)
        rows = self._rows(page_table, cu_rows, start, k.shape[0], device)
        self._call(self.lib.wf_cache_write, device, stream, c, rows, kp, ks, vp, vs, self._status(status, device))

    def wf_cache_read(self, cache: KvCache, page_table, cu_rows, start, n_rows: int, k=None, v=None, status=None, stream=None):
        """The values of the rows at positions start[s], start[s] + 1, ... of every sequence: (k, v) [n_rows, n_kv_head, d_head]
        in the path's type.  Rows at or behind cu_rows[-1] are left as they are."""
        c, device = self._cache(cache), cache.device
        shape = (n_rows, self.n_kv_head, self.d_head)
        k = self._empty(cache.k, shape, self.torch_dtype, stream) if k is None else k
        v = self._empty(cache.k, shape, self.torch_dtype, stream) if v is None else v
        if k.shape[0] < n_rows or v.shape[0] < n_rows:
            _refuse("k and v must have n_rows rows")
        (kp, ks), (vp, vs) = self._vectors(k, "k", device, self.n_kv_head), self._vectors(v, "v", device, self.n_kv_head)
        rows = self._rows(page_table, cu_rows, start, n_rows, device)
        self._call(self.lib.wf_cache_read, device, stream, c, rows, kp, ks, vp, vs, self._status(status, device))
        return k, v

    def wf_tree_attention(self, cache: KvCache, page_table, cu_rows, start, q: torch.Tensor, max_rows: int, max_len: int | None = None,
                          tail: str = "causal", mask=None, scale: float | None = None, out=None, lse=None, workspace=None, status=None,
                          stream=None):
        """Attention of queries [n_rows, n_head, d_head] over their sequences' cache; returns (out, lse float32 [n_rows, n_head]).
        ``tail``: "none" (the start[s] committed positions alone), "causal" (and the sequence's rows up to the query's own) or "mask"
        (and those rows t whose bit is set in the query's row of ``mask``, int32 or uint32 [n_rows, words]; "tree" is the same).
        ``max_rows`` and ``max_len`` bound the rows and the positions (rows included) of any sequence.  ``scale`` defaults to
        d_head ** -0.5.  ``workspace``: a uint8 tensor of ``tree_attention_workspace`` bytes, allocated per call if not given."""
        c, device = self._cache(cache), cache.device
        n = q.shape[0]
        qp, qs = self._vectors(q, "q", device, self.n_head)
        rows = self._rows(page_table, cu_rows, start, n, device)
        if tail not in TAILS:
            _refuse(f"tail is one of {', '.join(TAILS)}")
        mp, words = None, 0
        if TAILS[tail] == 2:
            if mask is None or mask.dim() != 2 or mask.shape[0] < n or mask.dtype not in (_INT, torch.uint32):
                _refuse("a tree needs mask: int32 or uint32 [n_rows, words]")
            mp, words = _vector(mask, "mask", device, mask.dtype), mask.shape[1]
        if max_len is None:
            max_len = page_table.shape[1] * self.page_size
        if out is None:
            out = torch.empty_like(q) if stream is None and q.is_contiguous() else self._empty(q, q.shape, self.torch_dtype, stream)
        elif out.shape[0] < n:
            _refuse("out must have the rows of q")
        op, os_ = self._vectors(out, "out", device, self.n_head)
        if lse is None:
            lse = self._empty(q, (n, self.n_head), _F32, stream)
        lp = _vector(lse, "lse", device, _F32, n * self.n_head)
        need = self.tree_attention_workspace(rows.n_seq, n, max_rows, max_len, device)
        if workspace is None and need:
            workspace = self._empty(q, need, _U8, stream)
        wp, have = (None, 0) if workspace is None else (_vector(workspace, "workspace", device, _U8), workspace.numel())
        self._call(self.lib.wf_tree_attention, device, stream, c, rows, qp, qs, self.d_head ** -0.5 if scale is None else scale, TAILS[tail],
                   mp, words, max_rows, max_len, op, os_, lp, wp, have, self._status(status, device))
        return out, lse

    def tree_attention_workspace(self, n_seq: int, n_rows: int, max_rows: int, max_len: int, device="cuda") -> int:
        """Bytes of workspace of ``wf_tree_attention`` for these sizes: a function of them and the device alone ("cuda": the current
        one).  It does not grow with every size: fewer sequences are split more, and may need more than a larger batch."""
        index = device.index if isinstance(device, torch.device) else device if isinstance(device, int) else torch.device(device).index
        if index is None:
            index = torch.cuda.current_device()
        key = (n_seq, n_rows, max_rows, max_len, index)
        if key not in self._workspace_bytes:
            n = C.c_size_t()
            with torch.cuda.device(index):
                self._check(self.lib.wf_tree_attention_workspace(self.handle, n_seq, n_rows, max_rows, max_len, C.byref(n)))
            if len(self._workspace_bytes) > 4096:
                self._workspace_bytes.clear()
            self._workspace_bytes[key] = n.value
        return self._workspace_bytes[key]

    def wf_selftest_attention_timeout(self, on: bool | int = True):
        """While on, the bounded waits of ``wf_tree_attention`` on 128-row tiles and of ``wf_gemm_e4m3`` give up at once: rows are NaN, status
        bit 8.  -1 - w: in ``wf_gemm_e4m3`` at first those of warp w alone."""
        self._check(self.lib.wf_selftest_attention_timeout(self.handle, int(on)))

    def wf_beam_select(self, logits: torch.Tensor, scores: torch.Tensor, keep: int, beams=None, finished=None, end_token: int = -1,
                       suppress=None, status=None, stream=None):
        """One round of beam search: the ``keep`` best continuations of every sequence.  logits [B * n_beam, vocab] float32 or
        bfloat16 (row stride free), scores float32 [B, n_beam]; beams [B] live beams, finished uint8 or bool [B, n_beam], suppress int32
        or uint32 bit words of tokens that are never chosen.  Returns (scores float32, parents int32, tokens int32, finished uint8),
        each [B, keep]; places without a continuation hold (-inf, -1, -1, 0)."""
        device = logits.device
        if device.type != "cuda" or logits.dim() != 2 or logits.dtype not in (_F32, _BF16) or logits.stride(1) != 1:
            _refuse("logits must be float32 or bfloat16 [B * n_beam, vocab] in device memory, a row's elements contiguous")
        if scores.dim() != 2 or logits.shape[0] != scores.numel():
            _refuse("scores must be [B, n_beam] for the B * n_beam rows of logits")
        (B, W), V = scores.shape, logits.shape[1]
        sp = _vector(scores, "scores", device, _F32)
        bp = None if beams is None else _vector(beams, "beams", device, n=B)
        fp = None if finished is None else _vector(finished, "finished", device, torch.bool if finished.dtype == torch.bool else _U8, B * W)
        up = None
        if suppress is not None:
            up = _vector(suppress, "suppress", device, suppress.dtype if suppress.dtype in (_INT, torch.uint32) else _INT, -(-V // 32))
        out = self._empty(logits, (B, keep), _F32, stream)
        parents, tokens = self._empty(logits, (B, keep), _INT, stream), self._empty(logits, (B, keep), _INT, stream)
        done = self._empty(logits, (B, keep), _U8, stream)
        ld = logits.stride(0) if logits.shape[0] > 1 else max(logits.stride(0), V)
        self._call(self.lib.wf_beam_select, device, stream, logits.data_ptr(), WF_BF16 if logits.dtype == _BF16 else WF_F32, ld, B, W, V, sp, bp, fp,
                   end_token, up, keep, out.data_ptr(), parents.data_ptr(), tokens.data_ptr(), done.data_ptr(), self._status(status, device))
        return out, parents, tokens, done

    def wf_beam_reorder(self, parents: torch.Tensor, states=(), caches=(), page_table=None, lengths=None, status=None, stream=None):
        """Moves every beam's states to the beams that grew from it, in place.  parents: [B, n_beam] (negative: stays).
        states: tensors [B * n_beam, ...] whose rows are contiguous (row stride free); caches: paged caches that share
        ``page_table`` [B * n_beam, pages], the beams of a sequence holding ``lengths`` [B] positions.  No two of them share
        memory (one given twice is refused)."""
        device = parents.device
        if parents.dim() != 2 or device.type != "cuda":
            _refuse("parents must be a [B, n_beam] tensor in device memory")
        B, W = parents.shape
        pp = _vector(parents, "parents", device)
        state_array = (wf_beam_state * len(states))()
        for i, t in enumerate(states):
            if t.device != device or t.dim() < 1 or t.shape[0] != B * W:
                _refuse(f"state {i} must be a [{B * W}, ...] tensor on {device}")
            row = t[0] if t.shape[0] else t
            if not row.is_contiguous():
                _refuse(f"state {i}: the elements of a row must be contiguous")
            size = row.numel() * t.element_size() if t.shape[0] else 0
            step = t.stride(0) * t.element_size() if t.shape[0] > 1 else size
            if step < size:
                _refuse(f"state {i}: rows overlap")
            state_array[i] = wf_beam_state(t.data_ptr(), size, step)
        cache_array = self._caches(caches, device)
        table = stride = lens = None
        if caches:
            if page_table is None or lengths is None or page_table.dim() != 2 or page_table.shape[0] != B * W:
                _refuse("paged caches need page_table [B * n_beam, pages] and lengths [B]")
            table, stride = _vector(page_table, "page_table", device), page_table.shape[1]
            lens = _vector(lengths, "lengths", device, n=B)
        self._call(self.lib.wf_beam_reorder, device, stream, pp, B, W, state_array, len(states), cache_array, len(caches), table, stride or 0,
                   lens, self._status(status, device))

    # -- rows and pages of a round
    def page_pool(self, n_pages: int, device="cuda") -> PagePool:
        """A pool in which all of ``n_pages`` pages are free, to be handed out in their order."""
        return PagePool(torch.arange(n_pages, dtype=_INT, device=device), torch.tensor([0, n_pages], dtype=_INT, device=device))

    def wf_page_plan(self, pool: PagePool, page_table, held, lengths, new_rows, n_rows: int, ended=None, status=None, stream=None):
        """Plans a round: which sequences get the ``new_rows`` [n_seq] that they ask for, with at most ``n_rows`` rows in all, and the
        pages that these lack.  ``pool``, ``page_table`` [n_seq, pages], ``held`` (pages) and ``lengths`` (positions) [n_seq] are updated in
        place; sequences with an ``ended`` flag (uint8 or bool [n_seq]) first give their pages back and begin at 0.  Returns (cu_rows
        [n_seq + 1], row_seq, row_pos int32 [n_rows], row_slot int64 [n_rows]); rows that nobody has hold -1."""
        device = pool.device
        if device.type != "cuda":
            _refuse("the pool must be in device memory")
        n_seq, shape = new_rows.numel(), page_table.shape
        if len(shape) != 2 or shape[0] < n_seq:
            _refuse("page_table must be [n_seq, pages]")
        args = (_vector(new_rows, "new_rows", device),
                None if ended is None else _vector(ended, "ended", device, torch.bool if ended.dtype == torch.bool else _U8, n_seq),
                _vector(lengths, "lengths", device, n=n_seq), _vector(held, "held", device, n=n_seq), _vector(page_table, "page_table", device))
        c = wf_page_pool(_vector(pool.pages, "pages", device), _vector(pool.state, "state", device, n=2), pool.pages.numel())
        cu = self._empty(new_rows, n_seq + 1, _INT, stream)
        seq, pos = self._empty(new_rows, max(n_rows, 0), _INT, stream), self._empty(new_rows, max(n_rows, 0), _INT, stream)
        slot = self._empty(new_rows, max(n_rows, 0), torch.int64, stream)
        self._call(self.lib.wf_page_plan, device, stream, c, n_seq, *args, shape[1], n_rows, cu.data_ptr(), seq.data_ptr(), pos.data_ptr(),
                   slot.data_ptr(), self._status(status, device))
        return cu, seq, pos, slot

    # -- drafted tokens
    def wf_draft_verify(self, logits: torch.Tensor, cu_rows, tokens, accept_u, sample_u, max_rows: int, parents=None, draft=None,
                        temperature=None, status=None, stream=None):
        """Which drafted tokens the target keeps, and the token behind them.  logits [n_rows, vocab] float32 or bfloat16 (row stride
        free); tokens, parents int32 [n_rows] (parents None: chains); draft float32 [n_rows, vocab]: row w is the distribution that w's
        children were drawn from (None: they were not drawn); temperature float32 [n_seq] (None: 1; 0: the largest logit); accept_u
        float32 [n_rows] and sample_u [n_seq]: random numbers from [0, 1).  Returns int32 (kept [n_seq], tokens [n_seq, max_rows], path
        [n_seq, max_rows]): how many rows stay, the new tokens (as many) and the rows that stay; -1 behind them."""
        device = logits.device
        if device.type != "cuda" or logits.dim() != 2 or logits.dtype not in (_F32, _BF16) or logits.stride(1) != 1:
            _refuse("logits must be float32 or bfloat16 [n_rows, vocab] in device memory, a row's elements contiguous")
        (n, V), n_seq = logits.shape, cu_rows.numel() - 1
        if n_seq < 0 or max_rows < 1:
            _refuse("cu_rows has n_seq + 1 entries, max_rows is at least 1")
        dp, dld = None, 0
        if draft is not None:
            if draft.dim() != 2 or draft.shape[0] < n or draft.shape[1] != V or draft.dtype is not _F32 or draft.device != device or draft.stride(1) != 1:
                _refuse(f"draft must be float32 [n_rows, {V}] beside the logits, a row's elements contiguous")
            dp, dld = draft.data_ptr(), draft.stride(0) if draft.shape[0] > 1 else max(draft.stride(0), V)
        kept = self._empty(logits, n_seq, _INT, stream)
        out, path = self._empty(logits, (n_seq, max_rows), _INT, stream), self._empty(logits, (n_seq, max_rows), _INT, stream)
        self._call(self.lib.wf_draft_verify, device, stream, logits.data_ptr(), WF_BF16 if logits.dtype is _BF16 else WF_F32,
                   logits.stride(0) if n > 1 else max(logits.stride(0), V), V, n_seq, n, max_rows, _vector(cu_rows, "cu_rows", device),
                   _vector(tokens, "tokens", device, n=n), None if parents is None else _vector(parents, "parents", device, n=n), dp, dld,
                   None if temperature is None else _vector(temperature, "temperature", device, _F32, n_seq),
                   _vector(accept_u, "accept_u", device, _F32, n), _vector(sample_u, "sample_u", device, _F32, n_seq), kept.data_ptr(),
                   out.data_ptr(), path.data_ptr(), self._status(status, device))
        return kept, out, path

    def wf_draft_commit(self, start, kept, path=None, caches=(), page_table=None, lengths=None, status=None, stream=None):
        """Moves the rows that stay (``path`` [n_seq, rows], the first ``kept`` [n_seq] of each; None: they lie as they should) behind
        the ``start`` [n_seq] committed positions in every cache, and returns the new lengths start + kept.  ``lengths``: where these go
        (``start`` itself: in place)."""
        device, n_seq = start.device, start.numel()
        if device.type != "cuda":
            _refuse("start must be in device memory")
        pp, stride = None, 0
        if path is not None:
            if path.dim() != 2 or path.shape[0] < n_seq or path.shape[1] < 1:  # (an empty one has no address, as if there were none)
                _refuse("path must be [n_seq, rows], of one row at least")
            pp, stride = _vector(path, "path", device), path.shape[1]
        cache_array = self._caches(caches, device)
        table = tstride = None
        if caches or page_table is not None:
            if page_table is None or page_table.dim() != 2 or page_table.shape[0] < n_seq:
                _refuse("caches need page_table [n_seq, pages]")
            table, tstride = _vector(page_table, "page_table", device), page_table.shape[1]
        if lengths is None:
            lengths = self._empty(start, n_seq, _INT, stream)
        self._call(self.lib.wf_draft_commit, device, stream, n_seq, _vector(start, "start", device), _vector(kept, "kept", device, n=n_seq), pp,
                   stride, _vector(lengths, "lengths", device, n=n_seq), cache_array, len(caches), table, tstride or 0, self._status(status, device))
        return lengths

    # -- products with 8-bit codes
    def wf_quantise_e4m3(self, x: torch.Tensor, out: ScaledCodes | None = None, stream=None) -> ScaledCodes:
        """x [rows, k] (float32 or bfloat16, row stride free) as e4m3 codes with a power-of-two scale for each 128 channels of a row:
        activations before a product, or weights, once."""
        device, shape, dtype, strides = x.device, x.shape, x.dtype, x.stride()
        if device.type != "cuda" or len(shape) != 2 or (dtype is not _F32 and dtype is not _BF16) or shape[1] < 1 or (strides[1] != 1 and shape[1] > 1):
            _refuse("x must be float32 or bfloat16 [rows, k] in device memory, a row's elements contiguous")
        rows, k = shape
        if out is None:
            out = ScaledCodes._within(self._empty(x, ScaledCodes._bytes(rows, k), _U8, stream), rows, k, device)
        elif out.shape != (rows, k) or out.device != device:
            _refuse("out must have the shape and the device of x")
        self._call(self.lib.wf_quantise_e4m3, device, stream, x.data_ptr(), WF_BF16 if dtype is _BF16 else WF_F32,
                   strides[0] if rows > 1 else max(strides[0], k), rows, k, out.c)
        return out

    def wf_gemm_e4m3(self, a: ScaledCodes, w: ScaledCodes, bias=None, gelu: bool = False, out=None, out_dtype: str | None = None, status=None,
                     stream=None) -> torch.Tensor:
        """act(a w^T + bias): a [m, k], w [n, k], bias float32 [n]; ``gelu``: the activation.  Returns [m, n] in ``out_dtype`` ("bf16" or
        "f32", default: the decoder's), or writes to ``out`` (row stride free)."""
        (m, k), (n, kw), device = a.shape, w.shape, a.device
        if k != kw or w.device != device or device.type != "cuda":
            _refuse(f"a has {k} channels and w {kw}, or they are not in one device's memory")
        if out is None:
            if out_dtype not in (None, "bf16", "f32"):
                _refuse("out_dtype is bf16 or f32")
            dtype, ld = self.torch_dtype if out_dtype is None else _BF16 if out_dtype == "bf16" else _F32, n
            out = self._empty(a._codes if a._memory is None else a._memory, (m, n), dtype, stream)
        elif out.shape != (m, n) or out.dtype not in (_F32, _BF16) or out.device != device or (out.stride(1) != 1 and n > 1):
            _refuse(f"out must be float32 or bfloat16 [{m}, {n}] on {device}, a row's elements contiguous")
        elif out_dtype is not None and out.dtype is not (_BF16 if out_dtype == "bf16" else _F32):
            _refuse("out is not of out_dtype")
        else:
            dtype, ld = out.dtype, out.stride(0) if m > 1 else max(out.stride(0), n)
        bp = None if bias is None else _vector(bias, "bias", device, _F32, n)
        self._call(self.lib.wf_gemm_e4m3, device, stream, a.c, w.c, bp, out.data_ptr(), WF_BF16 if dtype is _BF16 else WF_F32, ld, m, n, k,
                   int(gelu), self._status(status, device))
        return out
