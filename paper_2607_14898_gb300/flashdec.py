"""Python binding of libflashdec.so (ctypes): argument marshalling only.

Every step of the decode path runs in the library's CUDA kernels; this module only converts
Python / torch arguments into the C ABI of include/flashdec.h and include/flashdec_ops.h.
There is no fallback: if the library is missing or the device is not an sm_103 GPU, calls
raise.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

from . import build as _build

_LIB = None

FD_OK = 0
STATUS = {0: "FD_OK", 1: "FD_ERR_INVALID_ARG", 2: "FD_ERR_CONFIG", 3: "FD_ERR_OOM",
          4: "FD_ERR_CUDA", 5: "FD_ERR_STATE", 6: "FD_ERR_DEVICE_TIMEOUT",
          7: "FD_ERR_UNSUPPORTED"}
DTYPE_F32, DTYPE_BF16, DTYPE_U8, DTYPE_F16 = 0, 1, 2, 3
# fd_rope_mode, keyed like the oracle's rope_mode argument
ROPE_MODES = {"abs": 0, "window": 1}
EPI_F32, EPI_RESID, EPI_GELU, EPI_TUP, EPI_SWIGLU = 0, 1, 2, 3, 4
# fd_kernel_kind order
KERNEL_KINDS = ["unshuffle", "embed", "rmsnorm", "qkv", "attn_backbone", "attn_refine", "out",
                "mlp1", "mlp2", "tup", "head1", "head2", "pixel", "advance", "rope"]
# kernel kinds of the training step (enum fd_train_kind)
TRAIN_KINDS = ["linear", "dgrad", "wgrad", "attn_gemm", "softmax", "transpose", "norm",
               "pointwise"]


class FdError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {STATUS.get(code, code)}")
        self.code = code


class fd_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "latent_channels", "latent_h", "latent_w", "patch", "hidden", "heads", "kv_groups",
        "mlp_ratio", "n_blocks", "n_refine", "window", "r_t", "vae_spatial", "out_channels",
        "out_dtype", "mlp_gated")] + [("norm_eps", ctypes.c_float), ("rope_base", ctypes.c_float),
                                      ("qk_norm", ctypes.c_int32), ("mlp_fp8", ctypes.c_int32),
                                      ("first_chunk_frames", ctypes.c_int32),
                                      ("rope_mode", ctypes.c_int32)]


class fd_rotary_config(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("axes", ctypes.c_int32),
                ("axis_dims", ctypes.c_int32 * 3), ("scaling", ctypes.c_int32),
                ("base", ctypes.c_float), ("factor", ctypes.c_float),
                ("trained_len", ctypes.c_int32), ("fast_turns", ctypes.c_float),
                ("slow_turns", ctypes.c_float), ("amplitude", ctypes.c_float)]


class fd_cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("streams", "groups", "capacity", "head_dim",
                                              "dtype", "reserved")] + [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + [
        (n, ctypes.c_int64) for n in ("stream_stride", "group_stride", "slot_stride")] + [
        ("pos", ctypes.c_void_p), ("weight", ctypes.c_void_p)]


_P = ctypes.c_void_p
_I = ctypes.c_int
_F = ctypes.c_float
_L = ctypes.c_int64
_SIGS = {
    "fd_status_str": (ctypes.c_char_p, [_I]),
    "fd_weights_blob_elems": (ctypes.c_size_t, [ctypes.POINTER(fd_config)]),
    "fd_weights_blob_bytes": (ctypes.c_size_t, [ctypes.POINTER(fd_config), _I]),
    "fd_latent_bytes": (ctypes.c_size_t, [ctypes.POINTER(fd_config)]),
    "fd_pixels_bytes": (ctypes.c_size_t, [ctypes.POINTER(fd_config)]),
    "fd_handle_device_bytes": (ctypes.c_size_t, [ctypes.POINTER(fd_config)]),
    "fd_weights_create": (_I, [ctypes.POINTER(fd_config), _P, ctypes.c_size_t, _I,
                               ctypes.POINTER(_P)]),
    "fd_weights_destroy": (_I, [_P]),
    "fd_create": (_I, [ctypes.POINTER(fd_config), _P, ctypes.POINTER(_P)]),
    "fd_decode_chunk": (_I, [_P, _P, _P, _P]),
    "fd_decode_chunks": (_I, [ctypes.POINTER(_P), _I, ctypes.POINTER(_P), ctypes.POINTER(_P),
                              _P]),
    "fd_decode_chunk_host": (_I, [_P, _P, _P, _P]),
    "fd_decode_sequence_host": (_I, [_P, _I, _P, _P, _P]),
    "fd_batch_create": (_I, [ctypes.POINTER(fd_config), _P, _I, ctypes.POINTER(_P)]),
    "fd_decode_batch": (_I, [_P, ctypes.POINTER(_P), _I, ctypes.POINTER(_P),
                             ctypes.POINTER(_P), _P]),
    "fd_batch_destroy": (_I, [_P]),
    "fd_reset": (_I, [_P]),
    "fd_profile_enable": (_I, [_P, _I]),
    "fd_profile_collect": (_I, [_P, ctypes.POINTER(ctypes.c_int64),
                                ctypes.POINTER(ctypes.c_double)]),
    "fd_launch_count": (ctypes.c_int64, [_P]),
    "fd_destroy": (_I, [_P]),
    "fd_chunk_index": (ctypes.c_int64, [_P]),
    "fd_sync_status": (_I, [_P]),
    "fd_debug_read_ring": (_I, [_P, _I, _I, _P, ctypes.c_size_t]),
    "fd_debug_wait_timeout": (_I, [_P, ctypes.c_uint, _P]),
    "fd_train_grad_elems": (ctypes.c_size_t, [ctypes.POINTER(fd_config)]),
    "fd_op_linear_pixel": (_I, [_I, _I, _P, _P, _P, _I, _I, _I, _I, _I, _I, _P, _P, _P]),
    "fd_op_rmsnorm_bwd": (_I, [_P, _P, _P, _I, _I, _F, _P, _P, _P, _P]),
    "fd_op_scores_bwd": (_I, [_I, _I, _P, _P, _P, _P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _P]),
    "fd_op_gelu_bwd": (_I, [_P, _P, ctypes.c_int64, _P, _P, _P]),
    "fd_op_l1_pixel_bwd": (_I, [_P, _P, _I, _I, _I, _I, _I, _P, _P, _P, _P]),
    "fd_train_create": (_I, [ctypes.POINTER(fd_config), _P, _I, ctypes.POINTER(_P)]),
    "fd_train_step": (_I, [_P, _P, _P, _P, _P, _P]),
    "fd_train_status": (_I, [_P, _P]),
    "fd_train_profile_enable": (_I, [_P, _I]),
    "fd_train_profile_collect": (_I, [_P, ctypes.POINTER(ctypes.c_int64),
                                      ctypes.POINTER(ctypes.c_double)]),
    "fd_train_destroy": (_I, [_P]),
    "fd_state_bytes": (ctypes.c_size_t, [ctypes.POINTER(fd_config)]),
    "fd_save_state": (_I, [_P, _P, ctypes.c_size_t, _P]),
    "fd_load_state": (_I, [_P, _P, ctypes.c_size_t, _P]),
    "fd_op_linear": (_I, [_I, _I, _I, _I, _P, _P, _P, _P, _I, _I, _P, _P]),
    "fd_op_linear_tiled": (_I, [_I, _I, _I, _I, _P, _P, _P, _P, _I, _I, _I, _P, _P]),
    "fd_op_rope_table": (_I, [_I, _I, _F, _P, _P]),
    "fd_op_qkv": (_I, [_I, _I, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _F, _F,
                       _P, _P, _P, _P, _I, _I, _P, _P]),
    "fd_attention_workspace_bytes": (ctypes.c_size_t, [_I, _I, _I, _I, _I]),
    "fd_op_attention": (_I, [_I, _I, _I, _P, _P, _P, _I, _I, _P, _I, _P, _P, _P]),
    "fd_op_attention_static": (_I, [_I, _I, _I, _P, _P, _P, _I, _I, _P, _I, _P, _P]),
    "fd_op_kv_append": (_I, [_P, _P, _I, _I, _I, _I, _I, _P, _P, _P]),
    "fd_op_rmsnorm": (_I, [_P, _P, _I, _I, _F, _P, _P]),
    "fd_op_rmsnorm_e4m3": (_I, [_P, _P, _I, _I, _F, _F, _P, _P]),
    "fd_op_linear_e4m3": (_I, [_I, _I, _I, _I, _P, _P, _P, _P, _P, _F, _I, _P, _P]),
    "fd_op_unshuffle": (_I, [_P, _I, _I, _I, _I, _P, _P]),
    "fd_op_pixel_head": (_I, [_P, _I, _I, _I, _I, _I, _I, _P, _P]),
    "fd_rotary_create": (_I, [ctypes.POINTER(fd_rotary_config), ctypes.POINTER(_P)]),
    "fd_rotary_destroy": (_I, [_P]),
    "fd_op_rotary": (_I, [_P, _I, _I, _I, _P, _I, _P, _L, _L, _P, _L, _L, _I, _P, _L, _L, _P, _L,
                          _L, _P]),
    "fd_cache_attention_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(fd_cache), _I, _I,
                                                             _I]),
    "fd_op_cache_attention": (_I, [ctypes.POINTER(fd_cache), _I, _I, _I, _P, _L, _L, _L, _P, _F,
                                   _F, _P, _L, _L, _L, _P, _P, _P, _P]),
    "fd_debug_cache_wait_timeout": (_I, [_I, _P, _P]),
    "fd_op_cache_insert": (_I, [ctypes.POINTER(fd_cache), _I, _P, _P, _L, _L, _L, _P, _I, _I, _P,
                                _P, _P, _P]),
    "fd_op_cache_compact": (_I, [ctypes.POINTER(fd_cache), _I, ctypes.POINTER(fd_cache), _P, _I,
                                 _I, _P, _P]),
}


def lib(build_if_missing: bool = True) -> ctypes.CDLL:
    """Load libflashdec.so (building it in-tree first if needed)."""
    global _LIB
    if _LIB is None:
        path = _build.LIB
        if build_if_missing:
            path = _build.build()
        if not os.path.exists(path):
            raise RuntimeError(f"libflashdec.so not built ({path}); run __graft_entry__.build()")
        L = ctypes.CDLL(path)
        for name, (res, args) in _SIGS.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = L
    return _LIB


def _check(code: int, what: str) -> None:
    if code != FD_OK:
        raise FdError(code, what)


def make_config(cfg) -> fd_config:
    """fd_config from any object with the decoder's shape attributes (e.g. synth.FDConfig)."""
    c = fd_config()
    for n in ("latent_channels", "latent_h", "latent_w", "patch", "hidden", "heads",
              "kv_groups", "mlp_ratio", "n_blocks", "n_refine", "window", "r_t", "vae_spatial",
              "out_channels"):
        setattr(c, n, int(getattr(cfg, n)))
    c.out_dtype = DTYPE_U8 if getattr(cfg, "out_u8", False) else DTYPE_F32
    c.mlp_gated = 1 if cfg.mlp_gated else 0
    c.qk_norm = 1 if cfg.qk_norm else 0
    c.mlp_fp8 = 1 if getattr(cfg, "mlp_fp8", False) else 0
    c.first_chunk_frames = int(getattr(cfg, "first_chunk_frames", 0))
    c.rope_mode = ROPE_MODES[getattr(cfg, "rope_mode", "abs")]
    c.norm_eps = float(cfg.norm_eps)
    c.rope_base = float(cfg.rope_base)
    return c


def weight_names(cfg) -> list[str]:
    """Tensor names in weight-blob order (the order documented in include/flashdec.h)."""
    second = "qnorm.g" if getattr(cfg, "qk_norm", False) else "vnorm.g"
    blk = ["norm1.g", "qkv.w", "qkv.b", "knorm.g", second, "out.w", "out.b", "norm2.g",
           "mlp1.w", "mlp1.b", "mlp2.w", "mlp2.b"]
    names = ["embed.w", "embed.b"]
    names += [f"blocks.{b}.{n}" for b in range(cfg.n_blocks) for n in blk]
    names += ["normf.g", "tup.w", "tup.b"]
    names += [f"refine.{b}.{n}" for b in range(cfg.n_refine) for n in blk]
    names += ["normh.g", "head1.w", "head1.b", "head2.w", "head2.b"]
    return names


def pack_blob(cfg, weights: dict) -> np.ndarray:
    """Concatenate a name -> array dict into one fp32 blob in blob order."""
    return np.concatenate([np.asarray(weights[n], dtype=np.float32).ravel()
                           for n in weight_names(cfg)])


def _stream_ptr(stream) -> int:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return int(getattr(stream, "cuda_stream", stream))


def _ptr(x) -> int:
    if x is None:
        return 0
    if isinstance(x, np.ndarray):
        return int(x.ctypes.data)
    return int(x.data_ptr()) if hasattr(x, "data_ptr") else int(x)


def check_buffer(x, what: str, nbytes: int, dtype: str, on_device: bool,
                 device: int | None = None) -> None:
    """Refuse a buffer that the library would overrun or misread. The C ABI receives raw
    pointers and cannot see sizes, so the binding checks, for the stream-level calls, that each
    buffer is where the call expects it (CUDA device / host), contiguous, of the element type
    (dtype "float32" or "uint8") and of exactly nbytes bytes."""
    import torch
    if isinstance(x, np.ndarray):
        if on_device:
            raise TypeError(f"{what}: a CUDA tensor is required, not a numpy array")
        if x.dtype != np.dtype(dtype) or not x.flags.c_contiguous:
            raise TypeError(f"{what}: a C-contiguous {dtype} array is required")
        size = x.nbytes
    elif isinstance(x, torch.Tensor):
        if x.is_cuda != on_device:
            raise TypeError(f"{what}: a {'CUDA' if on_device else 'host'} tensor is required")
        if on_device and device is not None and x.device.index != device:
            raise ValueError(f"{what}: on cuda:{x.device.index}, the decoder is on cuda:{device}")
        if x.dtype != getattr(torch, dtype) or not x.is_contiguous():
            raise TypeError(f"{what}: a contiguous {dtype} tensor is required")
        size = x.numel() * x.element_size()
    else:
        raise TypeError(f"{what}: a torch tensor{'' if on_device else ' or numpy array'} "
                        "is required")
    if size != nbytes:
        raise ValueError(f"{what}: {size} bytes, the call reads or writes {nbytes}")


class Weights:
    """Device copy of the decoder weights (fd_weights_create); shareable by several Decoders."""

    def __init__(self, cfg, blob: np.ndarray):
        L = lib()
        self.cfg = make_config(cfg)
        blob = np.ascontiguousarray(blob)
        dt = DTYPE_F32 if blob.dtype == np.float32 else DTYPE_BF16
        if blob.dtype not in (np.float32, np.uint16):
            raise TypeError("blob must be fp32, or bf16 bits as uint16")
        out = _P()
        _check(L.fd_weights_create(ctypes.byref(self.cfg), blob.ctypes.data, blob.nbytes, dt,
                                   ctypes.byref(out)), "fd_weights_create")
        self.handle = out

    def close(self) -> None:
        if getattr(self, "handle", None):
            _check(lib().fd_weights_destroy(self.handle), "fd_weights_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Decoder:
    """One decoder stream (fd_create): rolling caches + chunk counter."""

    def __init__(self, cfg, weights: Weights):
        L = lib()
        self.cfg = make_config(cfg)
        self.weights = weights
        out = _P()
        _check(L.fd_create(ctypes.byref(self.cfg), weights.handle, ctypes.byref(out)),
               "fd_create")
        self.handle = out
        import torch
        self.device = torch.cuda.current_device()
        self._latent_bytes = L.fd_latent_bytes(ctypes.byref(self.cfg))
        self._pixels_bytes = L.fd_pixels_bytes(ctypes.byref(self.cfg))

    def _check_buffers(self, latent, pixels, on_device: bool) -> None:
        """The latent of one chunk and the pixels of the next chunk this decoder emits (one
        frame instead of r_t for chunk 0 under the causal frame count)."""
        pix = self._pixels_bytes
        if self.cfg.first_chunk_frames == 1 and self.chunk_index == 0:
            pix //= self.cfg.r_t
        dev = self.device if on_device else None
        check_buffer(latent, "latent", self._latent_bytes, "float32", on_device, dev)
        check_buffer(pixels, "pixels", pix,
                     "uint8" if self.cfg.out_dtype == DTYPE_U8 else "float32", on_device, dev)

    @property
    def pixels_bytes(self) -> int:
        return lib().fd_pixels_bytes(ctypes.byref(self.cfg))

    @property
    def latent_bytes(self) -> int:
        return lib().fd_latent_bytes(ctypes.byref(self.cfg))

    def decode_chunk(self, latent, pixels, stream=None) -> None:
        self._check_buffers(latent, pixels, True)
        _check(lib().fd_decode_chunk(self.handle, _ptr(latent), _ptr(pixels),
                                     _stream_ptr(stream)), "fd_decode_chunk")

    def decode_chunk_host(self, latent_host, pixels_host, stream=None) -> None:
        """Decode from / to host buffers (numpy arrays or pinned torch tensors)."""
        self._check_buffers(latent_host, pixels_host, False)
        lp = latent_host.ctypes.data if isinstance(latent_host, np.ndarray) else _ptr(latent_host)
        pp = pixels_host.ctypes.data if isinstance(pixels_host, np.ndarray) else _ptr(pixels_host)
        _check(lib().fd_decode_chunk_host(self.handle, lp, pp, _stream_ptr(stream)),
               "fd_decode_chunk_host")

    def decode_sequence_host(self, latents_host, pixels_host, stream=None) -> None:
        """Decode len(latents_host) consecutive chunks from / to host buffers (pinned torch
        tensors or numpy arrays), the copies overlapped with the decoding
        (fd_decode_sequence_host)."""
        n = len(latents_host)
        if len(pixels_host) != n:
            raise ValueError("one pixel buffer per latent")
        t0 = self.chunk_index
        dt = "uint8" if self.cfg.out_dtype == DTYPE_U8 else "float32"
        lps, pps = [], []
        for i, (z, p) in enumerate(zip(latents_host, pixels_host)):
            pix = self._pixels_bytes
            if self.cfg.first_chunk_frames == 1 and t0 + i == 0:
                pix //= self.cfg.r_t
            check_buffer(z, "latent", self._latent_bytes, "float32", False, None)
            check_buffer(p, "pixels", pix, dt, False, None)
            lps.append(z.ctypes.data if isinstance(z, np.ndarray) else _ptr(z))
            pps.append(p.ctypes.data if isinstance(p, np.ndarray) else _ptr(p))
        ls = (_P * max(n, 1))(*lps)
        ps = (_P * max(n, 1))(*pps)
        _check(lib().fd_decode_sequence_host(self.handle, n, ls, ps, _stream_ptr(stream)),
               "fd_decode_sequence_host")

    def reset(self) -> None:
        _check(lib().fd_reset(self.handle), "fd_reset")

    def profile(self, enable: bool) -> None:
        _check(lib().fd_profile_enable(self.handle, 1 if enable else 0), "fd_profile_enable")

    def profile_collect(self) -> dict:
        """{kind name: (launches, device ms)} since the last collect."""
        n = len(KERNEL_KINDS)
        launches = (ctypes.c_int64 * n)()
        ms = (ctypes.c_double * n)()
        _check(lib().fd_profile_collect(self.handle, launches, ms), "fd_profile_collect")
        return {k: (int(launches[i]), float(ms[i])) for i, k in enumerate(KERNEL_KINDS)}

    @property
    def launch_count(self) -> int:
        return lib().fd_launch_count(self.handle)

    def sync_status(self) -> int:
        return lib().fd_sync_status(self.handle)

    @property
    def chunk_index(self) -> int:
        return lib().fd_chunk_index(self.handle)

    def read_ring(self, which: int, layer: int, groups: int, window: int, rows: int):
        """(K, V) of one layer's ring as bf16 bit arrays [G][W*rows][64]."""
        n = groups * window * rows * 64
        buf = np.zeros(2 * n, dtype=np.uint16)
        _check(lib().fd_debug_read_ring(self.handle, which, layer, buf.ctypes.data, buf.nbytes),
               "fd_debug_read_ring")
        return (buf[:n].reshape(groups, window * rows, 64), buf[n:].reshape(groups, window * rows, 64))

    def debug_wait_timeout(self, limit_us: int, stream=None) -> None:
        """Enqueue the failure-path check: a bounded wait that runs out after limit_us."""
        _check(lib().fd_debug_wait_timeout(self.handle, int(limit_us), _stream_ptr(stream)),
               "fd_debug_wait_timeout")

    def state_bytes(self) -> int:
        return lib().fd_state_bytes(ctypes.byref(self.cfg))

    def save_state(self, buf, stream=None) -> None:
        """Copy the streaming state (chunk index, rolling caches) into buf (host memory of
        state_bytes() bytes: a numpy uint8 array or a pinned torch tensor), ordered on stream."""
        _check(lib().fd_save_state(self.handle, _ptr(buf), self.state_bytes(),
                                   _stream_ptr(stream)), "fd_save_state")

    def load_state(self, buf, stream=None) -> None:
        """Restore a state saved by a decoder of the same configuration."""
        _check(lib().fd_load_state(self.handle, _ptr(buf), self.state_bytes(),
                                   _stream_ptr(stream)), "fd_load_state")

    def close(self) -> None:
        if getattr(self, "handle", None):
            _check(lib().fd_destroy(self.handle), "fd_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Trainer:
    """Streaming training step over clips of `chunks` latent frames (fd_train_create)."""

    def __init__(self, cfg, weights: Weights, chunks: int):
        L = lib()
        self.cfg = make_config(cfg)
        self.weights = weights
        self.chunks = int(chunks)
        out = _P()
        _check(L.fd_train_create(ctypes.byref(self.cfg), weights.handle, self.chunks,
                                 ctypes.byref(out)), "fd_train_create")
        self.handle = out
        import torch
        self.device = torch.cuda.current_device()
        self.grad_elems = L.fd_train_grad_elems(ctypes.byref(self.cfg))
        self._latent_bytes = self.chunks * L.fd_latent_bytes(ctypes.byref(self.cfg))
        self._target_bytes = self.chunks * L.fd_pixels_bytes(ctypes.byref(self.cfg))

    def step(self, latents, targets, loss, grads, stream=None) -> None:
        """latents fp32 [T][C'][H'][W'], targets fp32 [T][C][r_t][H][W], loss fp32 [1], grads
        fp32 [grad_elems], all on the trainer's device."""
        dev = self.device
        check_buffer(latents, "latents", self._latent_bytes, "float32", True, dev)
        check_buffer(targets, "targets", self._target_bytes * (4 if self.cfg.out_dtype ==
                                                                DTYPE_U8 else 1),
                     "float32", True, dev)
        check_buffer(loss, "loss", 4, "float32", True, dev)
        check_buffer(grads, "grads", 4 * self.grad_elems, "float32", True, dev)
        _check(lib().fd_train_step(self.handle, _ptr(latents), _ptr(targets), _ptr(loss),
                                   _ptr(grads), _stream_ptr(stream)), "fd_train_step")

    def status(self, stream=None) -> int:
        return lib().fd_train_status(self.handle, _stream_ptr(stream))

    def profile(self, enable: bool) -> None:
        _check(lib().fd_train_profile_enable(self.handle, 1 if enable else 0),
               "fd_train_profile_enable")

    def profile_collect(self) -> dict:
        """{kind name: (launches, device ms)} of the steps since the last collect."""
        n = len(TRAIN_KINDS)
        launches = (ctypes.c_int64 * n)()
        ms = (ctypes.c_double * n)()
        _check(lib().fd_train_profile_collect(self.handle, launches, ms),
               "fd_train_profile_collect")
        return {k: (int(launches[i]), float(ms[i])) for i, k in enumerate(TRAIN_KINDS)}

    def close(self) -> None:
        if getattr(self, "handle", None):
            _check(lib().fd_train_destroy(self.handle), "fd_train_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def decode_chunks(decoders, latents, pixels, stream=None) -> None:
    n = len(decoders)
    if len(latents) != n or len(pixels) != n:
        raise ValueError("one latent and one pixel buffer per decoder")
    for d, z, p in zip(decoders, latents, pixels):
        d._check_buffers(z, p, True)
    hs = (_P * n)(*[d.handle for d in decoders])
    ls = (_P * n)(*[_ptr(x) for x in latents])
    ps = (_P * n)(*[_ptr(x) for x in pixels])
    _check(lib().fd_decode_chunks(hs, n, ls, ps, _stream_ptr(stream)), "fd_decode_chunks")


class Batch:
    """Stacked decode of up to max_streams decoders of one weights object (fd_batch_create):
    the GEMMs of a chunk run once on all streams' rows."""

    def __init__(self, cfg, weights: Weights, max_streams: int):
        self.cfg = make_config(cfg)
        self.weights = weights
        out = _P()
        _check(lib().fd_batch_create(ctypes.byref(self.cfg), weights.handle, int(max_streams),
                                     ctypes.byref(out)), "fd_batch_create")
        self.handle = out

    def decode(self, decoders, latents, pixels, stream=None) -> None:
        """One chunk for each decoder (fd_decode_batch)."""
        n = len(decoders)
        if len(latents) != n or len(pixels) != n:
            raise ValueError("one latent and one pixel buffer per decoder")
        for d, z, p in zip(decoders, latents, pixels):
            d._check_buffers(z, p, True)
        hs = (_P * n)(*[d.handle for d in decoders])
        ls = (_P * n)(*[_ptr(x) for x in latents])
        ps = (_P * n)(*[_ptr(x) for x in pixels])
        _check(lib().fd_decode_batch(self.handle, hs, n, ls, ps, _stream_ptr(stream)),
               "fd_decode_batch")

    def close(self) -> None:
        if getattr(self, "handle", None):
            _check(lib().fd_batch_destroy(self.handle), "fd_batch_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ------------------------------------------------------------------ kernel-level entry points
def op_linear(epi, A, W, bias, out, tup_hidden=0, bn=0, err=None, stream=None, pair=None
              ) -> None:
    """pair: None (fd_op_linear), or 0 / 1 / 2 (library choice / single CTAs / CTA pairs)."""
    M, K = A.shape
    N = W.shape[0]
    if pair is None:
        _check(lib().fd_op_linear(epi, M, N, K, _ptr(A), _ptr(W), _ptr(bias), _ptr(out),
                                  tup_hidden, bn, _ptr(err), _stream_ptr(stream)), "fd_op_linear")
    else:
        _check(lib().fd_op_linear_tiled(epi, M, N, K, _ptr(A), _ptr(W), _ptr(bias), _ptr(out),
                                        tup_hidden, bn, pair, _ptr(err), _stream_ptr(stream)),
               "fd_op_linear_tiled")


def op_rope_table(t, frames_per_chunk, rope_base, table, stream=None) -> None:
    _check(lib().fd_op_rope_table(t, frames_per_chunk, rope_base, _ptr(table),
                                  _stream_ptr(stream)), "fd_op_rope_table")


def op_qkv(A, Wqkv, bqkv, knorm_g, norm2_g, heads, groups, tokens, grid_w, frames_per_chunk,
           window, t, eps, rope_base, rope_t, q_out, k_ring, vt_ring, ring_pitch, bn=0, err=None,
           stream=None, qk_norm=False) -> None:
    """norm2_g: V's gain (KV-norm) or, with qk_norm, Q's gain."""
    M, K = A.shape
    _check(lib().fd_op_qkv(M, K, _ptr(A), _ptr(Wqkv), _ptr(bqkv), _ptr(knorm_g), _ptr(norm2_g),
                           1 if qk_norm else 0,
                           heads, groups, tokens, grid_w, frames_per_chunk, window, t, eps,
                           rope_base, _ptr(rope_t), _ptr(q_out), _ptr(k_ring), _ptr(vt_ring),
                           ring_pitch, bn, _ptr(err), _stream_ptr(stream)), "fd_op_qkv")


def attention_workspace_bytes(Lq, heads, groups, n_keys, parts=0) -> int:
    return lib().fd_attention_workspace_bytes(Lq, heads, groups, n_keys, parts)


def op_attention(q, k_ring, vt_ring, heads, groups, ring_pitch, n_keys, out, parts=0,
                 workspace=None, err=None, stream=None) -> None:
    """fd_op_attention; parts = CTAs of the persistent launch (0: one per SM)."""
    Lq = q.shape[0]
    _check(lib().fd_op_attention(Lq, heads, groups, _ptr(q), _ptr(k_ring), _ptr(vt_ring),
                                 ring_pitch, n_keys, _ptr(out), parts, _ptr(workspace),
                                 _ptr(err), _stream_ptr(stream)), "fd_op_attention")


def op_attention_static(q, k_ring, vt_ring, heads, groups, ring_pitch, n_keys, out, parts=0,
                        err=None, stream=None) -> None:
    """fd_op_attention with its workspace in the library's static device memory."""
    Lq = q.shape[0]
    _check(lib().fd_op_attention_static(Lq, heads, groups, _ptr(q), _ptr(k_ring), _ptr(vt_ring),
                                        ring_pitch, n_keys, _ptr(out), parts, _ptr(err),
                                        _stream_ptr(stream)), "fd_op_attention_static")


def op_kv_append(k, v, window, t, ring_pitch, k_ring, vt_ring, stream=None) -> None:
    G, rows, _ = k.shape
    _check(lib().fd_op_kv_append(_ptr(k), _ptr(v), G, rows, window, t, ring_pitch, _ptr(k_ring),
                                 _ptr(vt_ring), _stream_ptr(stream)), "fd_op_kv_append")


def op_rmsnorm(h, g, eps, u, stream=None) -> None:
    M, D = h.shape
    _check(lib().fd_op_rmsnorm(_ptr(h), _ptr(g), M, D, eps, _ptr(u), _stream_ptr(stream)),
           "fd_op_rmsnorm")


def op_rmsnorm_e4m3(h, g, eps, out_scale, u, stream=None) -> None:
    """u (uint8 tensor holding e4m3 codes) = e4m3(RMSNorm(h) g out_scale)."""
    M, D = h.shape
    _check(lib().fd_op_rmsnorm_e4m3(_ptr(h), _ptr(g), M, D, eps, out_scale, _ptr(u),
                                    _stream_ptr(stream)), "fd_op_rmsnorm_e4m3")


def op_linear_e4m3(epi, A, W, col_scale, bias, out, out_scale=1.0, bn=0, err=None,
                   stream=None) -> None:
    """FP8 linear: A [M][K], W [N][K] e4m3 codes (uint8 tensors), fp32 col_scale / bias."""
    M, K = A.shape
    N = W.shape[0]
    _check(lib().fd_op_linear_e4m3(epi, M, N, K, _ptr(A), _ptr(W), _ptr(col_scale), _ptr(bias),
                                   _ptr(out), out_scale, bn, _ptr(err), _stream_ptr(stream)),
           "fd_op_linear_e4m3")


def op_unshuffle(z, p, x0, stream=None) -> None:
    C, H, W = z.shape
    _check(lib().fd_op_unshuffle(_ptr(z), C, H, W, p, _ptr(x0), _stream_ptr(stream)),
           "fd_op_unshuffle")


def op_pixel_head(F, frames, grid_h, grid_w, channels, rs, out_dtype, pixels, stream=None) -> None:
    _check(lib().fd_op_pixel_head(_ptr(F), frames, grid_h, grid_w, channels, rs, out_dtype,
                                  _ptr(pixels), _stream_ptr(stream)), "fd_op_pixel_head")


def op_linear_pixel(A, W, bias, frames, grid_h, grid_w, channels, rs, out_dtype, pixels,
                    err=None, stream=None) -> None:
    """Head layer 2 with the pixel shuffle in its epilogue (fd_op_linear_pixel)."""
    M, K = A.shape
    _check(lib().fd_op_linear_pixel(M, K, _ptr(A), _ptr(W), _ptr(bias), frames, grid_h, grid_w,
                                    channels, rs, out_dtype, _ptr(pixels), _ptr(err),
                                    _stream_ptr(stream)), "fd_op_linear_pixel")


def op_scores_bwd(Q, dO, K, V, lse, delta, Pc, Lp, L, dS, dST, PT, err=None,
                  stream=None) -> None:
    """The attention's scores backward in one launch (fd_op_scores_bwd)."""
    M, N = Q.shape[0], K.shape[0]
    _check(lib().fd_op_scores_bwd(M, N, _ptr(Q), _ptr(dO), _ptr(K), _ptr(V), _ptr(lse),
                                  _ptr(delta), Pc, Lp, L, _ptr(dS), _ptr(dST), _ptr(PT), _ptr(err),
                                  _stream_ptr(stream)), "fd_op_scores_bwd")


def op_rmsnorm_bwd(x, g, dy, eps, dx, dg, stream=None) -> None:
    M, D = x.shape
    import torch
    work = torch.empty(M, D, dtype=torch.float32, device=x.device)
    _check(lib().fd_op_rmsnorm_bwd(_ptr(x), _ptr(g), _ptr(dy), M, D, eps, _ptr(dx), _ptr(dg),
                                   _ptr(work), _stream_ptr(stream)), "fd_op_rmsnorm_bwd")


def op_gelu_bwd(z, da, dz, dz_bf16, stream=None) -> None:
    _check(lib().fd_op_gelu_bwd(_ptr(z), _ptr(da), z.numel(), _ptr(dz), _ptr(dz_bf16),
                                _stream_ptr(stream)), "fd_op_gelu_bwd")


def op_l1_pixel_bwd(F, target, frames, grid_h, grid_w, channels, rs, dF, loss,
                    stream=None) -> None:
    import torch
    work = torch.empty((F.numel() + 255) // 256, dtype=torch.float32, device=F.device)
    _check(lib().fd_op_l1_pixel_bwd(_ptr(F), _ptr(target), frames, grid_h, grid_w, channels, rs,
                                    _ptr(dF), _ptr(loss), _ptr(work), _stream_ptr(stream)),
           "fd_op_l1_pixel_bwd")


# ------------------------------------------- rotary positions and the cache of bounded size
ROTARY_LAYOUTS = {"interleaved": 0, "half": 1}
ROTARY_SCALINGS = {"none": 0, "linear": 1, "base": 2, "blend": 3}


_DTYPE_CODES: dict = {}


def _dtype_code(dtype) -> int:
    if not _DTYPE_CODES:
        import torch
        _DTYPE_CODES.update({torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16,
                             torch.float16: DTYPE_F16})
    code = _DTYPE_CODES.get(dtype)
    if code is None:
        raise TypeError(f"dtype {dtype}: float32, bfloat16 or float16 is required")
    return code


_raw_stream = _get_device = None


def _stream_on(device: int, stream) -> int:
    """The stream's handle; of the device's current stream where none is given. (The handle alone:
    a torch.cuda.Stream object takes 3 us to make, half of what a small call takes in all.) The
    library launches on the current device: tensors of another one are refused."""
    global _raw_stream, _get_device
    if _get_device is None:
        import torch
        _get_device = torch._C._cuda_getDevice  # torch.cuda.current_device once CUDA is up
    current = _get_device()
    if device != current:
        raise ValueError(f"tensors on cuda:{device}: the library works on the current device, "
                         f"which is cuda:{current}")
    if stream is None:
        if _raw_stream is None:
            import torch
            _raw_stream = torch._C._cuda_getCurrentRawStream
        return _raw_stream(device)
    return int(getattr(stream, "cuda_stream", stream))


def _refuse(t, what: str, shape, dtype, device: int, contiguous: bool) -> None:
    """Says what is wrong with a tensor that a check has turned down."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what}: a CUDA tensor is required")
    if t.dtype != dtype:
        raise TypeError(f"{what}: {t.dtype}, the call takes {dtype}")
    if t.get_device() != device:
        raise ValueError(f"{what}: on {t.device}, the call works on cuda:{device}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, the call takes {tuple(shape)}")
    if contiguous:
        raise ValueError(f"{what}: a contiguous tensor is required")
    raise ValueError(f"{what}: the last dimension must be contiguous")


def _dense(t, what: str, shape, dtype, device: int) -> int:
    """Address of a contiguous tensor of this shape, type and device. The library receives raw
    pointers: anything else would be misread or overrun."""
    try:
        if (t.dtype is dtype and t.shape == shape and t.get_device() == device
                and t.is_contiguous()):
            return t.data_ptr()
    except AttributeError:
        pass
    _refuse(t, what, shape, dtype, device, True)


def _rows(t, what: str, shape, dtype, device: int):
    """(address, strides) of a tensor whose last dimension is contiguous."""
    try:
        st = t.stride()
        if (t.dtype is dtype and t.shape == shape and t.get_device() == device
                and (st[-1] == 1 or shape[-1] < 2)):
            return t.data_ptr(), st
    except AttributeError:
        pass
    _refuse(t, what, shape, dtype, device, False)


def _same_steps(a, b, shape) -> bool:
    """Whether strides a and b lead to the same elements: a dimension of one entry never steps."""
    return all(x == y or n < 2 for x, y, n in zip(a, b, shape))


def _status_word(err, dtype, device: int) -> int:
    """Address of the int32 that a call's kernels report a wait in that gave up (0 for None, which the
    library refuses where it needs one)."""
    if err is None:
        return 0
    try:
        if (err.dtype is dtype and err.get_device() == device and err.numel()
                and err.is_contiguous()):
            return err.data_ptr()
    except AttributeError:
        pass
    raise TypeError(f"err: a contiguous int32 tensor on cuda:{device} is required")


class Rotary:
    """Frequencies of a rotary embedding (fd_rotary_create): the leading rot_dim elements of a
    head (all by default) in pairs of the given layout, split over the position axes by axis_dims."""

    def __init__(self, head_dim, rot_dim=None, layout="interleaved", axis_dims=None,
                 base=10000.0, scaling="none", factor=1.0, trained_len=1, fast_turns=32.0,
                 slow_turns=1.0, amplitude=1.0):
        rot_dim = int(head_dim if rot_dim is None else rot_dim)
        dims = [rot_dim] if axis_dims is None else [int(d) for d in axis_dims]
        if not 1 <= len(dims) <= 3:
            raise ValueError("1 to 3 position axes")
        c = fd_rotary_config(int(head_dim), rot_dim, ROTARY_LAYOUTS[layout], len(dims),
                             (ctypes.c_int32 * 3)(*dims), ROTARY_SCALINGS[scaling], float(base),
                             float(factor), int(trained_len), float(fast_turns),
                             float(slow_turns), float(amplitude))
        import torch
        self.head_dim, self.axes, self.int32 = int(head_dim), len(dims), torch.int32
        out = _P()
        _check(lib().fd_rotary_create(ctypes.byref(c), ctypes.byref(out)), "fd_rotary_create")
        self.handle = out

    def close(self) -> None:
        if getattr(self, "handle", None):
            _check(lib().fd_rotary_destroy(self.handle), "fd_rotary_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def op_rotary(plan: Rotary, positions, q, q_out, k=None, k_out=None, backward=False,
              stream=None) -> None:
    """Turns q [T][heads][head_dim] (and k) by positions int32 [T][axes] ([T] for one axis) into
    q_out (k_out), which may be q (k) itself; with backward=True the gradient (fd_op_rotary)."""
    shape, dtype, dev = q.shape, q.dtype, q.get_device()
    if dev < 0:  # (the other tensors are compared with q)
        raise TypeError("q: a CUDA tensor is required")
    if len(shape) != 3 or shape[2] != plan.head_dim:
        raise ValueError(f"q: shape {tuple(shape)}, [tokens][heads][{plan.head_dim}] is required")
    T = shape[0]
    pos = _dense(positions, "positions",
                 (T,) if plan.axes == 1 and positions.dim() == 1 else (T, plan.axes),
                 plan.int32, dev)
    qp, qs = _rows(q, "q", shape, dtype, dev)
    op, os_ = _rows(q_out, "q_out", shape, dtype, dev)
    if k is None:
        args = (0, 0, 0, 0, 0, 0, 0)
    else:
        ks = k.shape
        if len(ks) != 3 or ks[0] != T or ks[2] != plan.head_dim:
            raise ValueError(f"k: shape {tuple(ks)}, [{T}][heads][{plan.head_dim}] is required")
        kp, kst = _rows(k, "k", ks, dtype, dev)
        ko, kot = _rows(k_out, "k_out", ks, dtype, dev)
        args = (ks[1], kp, kst[0], kst[1], ko, kot[0], kot[1])
    code = lib().fd_op_rotary(plan.handle, 1 if backward else 0, _dtype_code(dtype), T, pos,
                              shape[1], qp, qs[0], qs[1], op, os_[0], os_[1], *args,
                              _stream_on(dev, stream))
    if code:
        raise FdError(code, "fd_op_rotary")


class Cache:
    """A cache of bounded size (fd_cache) over the caller's tensors: k, v bf16 or fp16
    [streams][groups][capacity][head_dim] (any strides that fd_cache allows, the same for both),
    pos int32 and weight fp32 [streams][groups][capacity]; empty slots have pos < 0."""

    def __init__(self, k, v, pos, weight):
        import torch
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            raise ValueError("k: [streams][groups][capacity][head_dim] is required")
        if k.dtype not in (torch.bfloat16, torch.float16):
            raise TypeError(f"k: {k.dtype}, a cache holds bfloat16 or float16")
        S, G, C, D = k.shape
        dev = k.get_device()
        kp, st = _rows(k, "k", k.shape, k.dtype, dev)
        vp, vst = _rows(v, "v", k.shape, k.dtype, dev)
        if dev < 0:
            raise TypeError("k: a CUDA tensor is required")
        if vst != st and not _same_steps(st, vst, k.shape):
            raise ValueError("v: the strides of k are required")
        self.k, self.v, self.pos, self.weight = k, v, pos, weight
        self.streams, self.groups, self.capacity, self.head_dim = S, G, C, D
        self.device, self.dtype, self.int32, self.float32 = dev, k.dtype, torch.int32, torch.float32
        self.view = fd_cache(S, G, C, D, _dtype_code(k.dtype), 0, kp, vp, st[0], st[1], st[2],
                             _dense(pos, "pos", (S, G, C), torch.int32, dev),
                             _dense(weight, "weight", (S, G, C), torch.float32, dev))
        self.ref = ctypes.byref(self.view)
        self._workspace: dict = {}  # bytes by (used, heads, n_q)

    def workspace_bytes(self, used: int, heads: int, n_q: int) -> int:
        key = (used, heads, n_q)
        need = self._workspace.get(key)
        if need is None:
            if len(self._workspace) > 1000:
                self._workspace.clear()
            need = self._workspace[key] = lib().fd_cache_attention_workspace_bytes(
                self.ref, used, heads, n_q)
        return need


def cache_attention_workspace_bytes(cache: Cache, heads, n_q, used=None) -> int:
    return cache.workspace_bytes(cache.capacity if used is None else int(used), heads, n_q)


def op_cache_attention(cache: Cache, q, q_pos, out, weight_out=None, used=None, scale=None,
                       decay=1.0, workspace=None, err=None, stream=None) -> None:
    """Attention of q [streams][n_q][heads][head_dim] at positions q_pos int32 [streams][n_q] over
    the cache's first `used` slots (all by default) into out; weight_out fp32
    [streams][groups][capacity] (may be cache.weight) receives decay times the slots' weights plus
    what this call gives them. scale: 1 / sqrt(head_dim) by default (fd_op_cache_attention)."""
    shape, dev, D = q.shape, cache.device, cache.head_dim
    if len(shape) != 4 or shape[0] != cache.streams or shape[3] != D:
        raise ValueError(f"q: shape {tuple(shape)}, [{cache.streams}][n_q][heads][{D}] is required")
    n, H = shape[1], shape[2]
    qp, qs = _rows(q, "q", shape, cache.dtype, dev)
    op, os_ = _rows(out, "out", shape, cache.dtype, dev)
    pos = _dense(q_pos, "q_pos", (cache.streams, n), cache.int32, dev)
    used = cache.capacity if used is None else int(used)
    wp = 0 if weight_out is None else _dense(
        weight_out, "weight_out", (cache.streams, cache.groups, cache.capacity), cache.float32, dev)
    need = cache.workspace_bytes(used, H, n)
    if need and (workspace is None or workspace.get_device() != dev
                 or not workspace.is_contiguous() or workspace.nbytes < need):
        raise ValueError(f"workspace: {need} bytes of contiguous memory on cuda:{dev} are required")
    code = lib().fd_op_cache_attention(
        cache.ref, used, H, n, qp, qs[0], qs[1], qs[2], pos, D ** -0.5 if scale is None else scale,
        decay, op, os_[0], os_[1], os_[2], wp, _ptr(workspace), _status_word(err, cache.int32, dev),
        _stream_on(dev, stream))
    if code:
        raise FdError(code, "fd_op_cache_attention")


def debug_cache_wait_timeout(which: int, err, stream=None) -> None:
    """One of the attention's bounded waits on a barrier that nothing arrives at, with a limit of 1 ms:
    sets bit 32 of err (fd_debug_cache_wait_timeout)."""
    import torch
    dev = err.get_device()
    code = lib().fd_debug_cache_wait_timeout(which, _status_word(err, torch.int32, dev),
                                             _stream_on(dev, stream))
    if code:
        raise FdError(code, "fd_debug_cache_wait_timeout")


def op_cache_insert(cache: Cache, k_new, v_new, new_pos, slots, pos_out=None, weight_out=None,
                    sinks=0, recent=0, stream=None) -> None:
    """New tokens k_new, v_new [streams][n][groups][head_dim] at new_pos int32 [streams][n] take
    the n slots of each (stream, group) that rank first by (class, weight, slot), written to
    slots int32 [streams][groups][n]; positions and weights go to pos_out and weight_out (the
    cache's own by default) (fd_op_cache_insert)."""
    shape, dev = k_new.shape, cache.device
    S, G, C = cache.streams, cache.groups, cache.capacity
    if len(shape) != 4 or shape[0] != S or shape[2] != G or shape[3] != cache.head_dim:
        raise ValueError(f"k_new: shape {tuple(shape)}, [{S}][n][{G}][{cache.head_dim}] is required")
    n = shape[1]
    kp, st = _rows(k_new, "k_new", shape, cache.dtype, dev)
    vp, vst = _rows(v_new, "v_new", shape, cache.dtype, dev)
    if vst != st and not _same_steps(st, vst, shape):
        raise ValueError("v_new: the strides of k_new are required")
    code = lib().fd_op_cache_insert(
        cache.ref, n, kp, vp, st[0], st[1], st[2],
        _dense(new_pos, "new_pos", (S, n), cache.int32, dev), sinks, recent,
        _dense(cache.pos if pos_out is None else pos_out, "pos_out", (S, G, C), cache.int32, dev),
        _dense(cache.weight if weight_out is None else weight_out, "weight_out", (S, G, C),
               cache.float32, dev),
        _dense(slots, "slots", (S, G, n), cache.int32, dev), _stream_on(dev, stream))
    if code:
        raise FdError(code, "fd_op_cache_insert")


def op_cache_compact(src: Cache, dst: Cache, now, src_slots, used=None, sinks=0, recent=0,
                     stream=None) -> None:
    """The dst.capacity entries of src's first `used` slots (all by default) that rank last by
    (class, weight, slot), recency counted from now int32 [streams], into dst in slot order;
    src_slots int32 [streams][groups][dst.capacity]: where each came from (fd_op_cache_compact)."""
    dev = src.device
    if dst.device != dev:
        raise ValueError(f"dst: on cuda:{dst.device}, src is on cuda:{dev}")
    code = lib().fd_op_cache_compact(
        src.ref, src.capacity if used is None else int(used), dst.ref,
        _dense(now, "now", (src.streams,), src.int32, dev), sinks, recent,
        _dense(src_slots, "src_slots", (src.streams, src.groups, dst.capacity), src.int32, dev),
        _stream_on(dev, stream))
    if code:
        raise FdError(code, "fd_op_cache_compact")
