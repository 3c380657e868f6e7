"""Python binding of libflashdecoder.so (include/flashdecoder.h).

Argument marshalling only: every step of the decoder forward runs in the HIP
library. PyTorch supplies device memory and streams. The functions keep the C
names; ``Decoder`` and ``KvCache`` are thin owners of the C handles.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libflashdecoder.so")

FD_OK, FD_ERR_INVALID_ARGUMENT, FD_ERR_UNSUPPORTED, FD_ERR_OUT_OF_MEMORY, FD_ERR_DEVICE, \
    FD_ERR_STATE = range(6)
FD_DTYPE_F32, FD_DTYPE_BF16, FD_DTYPE_F16 = 0, 1, 2
FD_KC_GEMM, FD_KC_ATTENTION, FD_KC_NORM, FD_KC_QKV_POST, FD_KC_EMBED_IN, FD_KC_ATTENTION_REFINE = range(6)

_DTYPES = {"f32": FD_DTYPE_F32, "bf16": FD_DTYPE_BF16, "f16": FD_DTYPE_F16}


class fd_config(ctypes.Structure):
    _fields_ = [(n, t) for n, t in [
        ("struct_size", ctypes.c_uint32), ("compute_dtype", ctypes.c_int32),
        ("latent_channels", ctypes.c_int32), ("latent_h", ctypes.c_int32),
        ("latent_w", ctypes.c_int32), ("patch", ctypes.c_int32), ("dim", ctypes.c_int32),
        ("n_heads", ctypes.c_int32), ("n_kv_groups", ctypes.c_int32),
        ("n_backbone_blocks", ctypes.c_int32), ("n_refine_blocks", ctypes.c_int32),
        ("mlp_hidden", ctypes.c_int32), ("head_hidden", ctypes.c_int32),
        ("mlp_kind", ctypes.c_int32), ("norm_kind", ctypes.c_int32),
        ("head_kind", ctypes.c_int32), ("kv_norm", ctypes.c_int32), ("rope", ctypes.c_int32),
        ("rope_theta", ctypes.c_float), ("norm_eps", ctypes.c_float), ("r_t", ctypes.c_int32),
        ("s_out", ctypes.c_int32), ("out_channels", ctypes.c_int32), ("window", ctypes.c_int32),
        ("unit_frames", ctypes.c_int32), ("max_batch", ctypes.c_int32),
        ("max_frames_per_call", ctypes.c_int32), ("clamp_output", ctypes.c_int32),
        ("mlp_precision", ctypes.c_int32)]]


class fd_tensor_desc(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("ndim", ctypes.c_int32),
                ("shape", ctypes.c_int64 * 2), ("offset", ctypes.c_uint64)]


class fd_rope(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("n_axes", ctypes.c_int32), ("freq", ctypes.c_void_p), ("axis", ctypes.c_void_p),
                ("magnitude", ctypes.c_float), ("inverse", ctypes.c_int32)]


class fd_token_cache(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("batch", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("capacity", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("pos", ctypes.c_void_p), ("weight", ctypes.c_void_p)]


class FlashDecoderError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"[{status}] {msg}")
        self.status = status


_lib = None


def load_library() -> ctypes.CDLL:
    """Load the HIP library (after torch, so both share one HIP runtime)."""
    global _lib
    if _lib is not None:
        return _lib
    import torch  # noqa: F401  (loads the process's HIP runtime first)
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built: run __graft_entry__.build() "
                           "(python -m paper_2607_14898_amd.build)")
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.c_void_p
    I32, I64, SZ = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    sigs = {
        "fd_config_validate": (I32, [ctypes.POINTER(fd_config)]),
        "fd_weights_layout": (I32, [ctypes.POINTER(fd_config), ctypes.POINTER(fd_tensor_desc),
                                    SZ, ctypes.POINTER(SZ), ctypes.POINTER(SZ)]),
        "fd_decoder_create": (I32, [ctypes.POINTER(fd_config), P, I32, SZ, ctypes.POINTER(P)]),
        "fd_decoder_destroy": (None, [P]),
        "fd_decoder_config": (ctypes.POINTER(fd_config), [P]),
        "fd_kv_cache_create": (I32, [P, I32, ctypes.POINTER(P)]),
        "fd_kv_cache_reset": (I32, [P]),
        "fd_kv_cache_position": (I64, [P]),
        "fd_kv_cache_fp16_saturations": (I32, [P, ctypes.POINTER(ctypes.c_uint64)]),
        "fd_kv_cache_destroy": (None, [P]),
        "fd_output_shape": (I32, [P, I32, I32, ctypes.POINTER(I64)]),
        "fd_decode_chunk": (I32, [P, P, I32, I32, P, P, P]),
        "fd_decode_chunk_trace": (I32, [P, P, I32, I32, P, P, P, P, SZ]),
        "fd_decode_chunk_noalloc": (I32, [P, P, I32, I32, P, P, P]),
        "fd_decode_chunk_as": (I32, [P, P, I32, I32, P, P, I32, P]),
        "fd_decode_chunks": (I32, [P, I32, ctypes.POINTER(P), I32, I32, ctypes.POINTER(P),
                                   ctypes.POINTER(P), I32, P]),
        "fd_trace_elems": (SZ, [P, I32, I32]),
        "fd_probe_enable": (I32, [P, I32]),
        "fd_probe_read": (I32, [P, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(I64),
                                ctypes.POINTER(ctypes.c_double)]),
        "fd_measure_mfma_peak": (I32, [I32, I32, P, ctypes.POINTER(ctypes.c_double),
                                       ctypes.POINTER(ctypes.c_double)]),
        "fd_measure_lds_bandwidth": (I32, [I32, P, ctypes.POINTER(ctypes.c_double),
                                           ctypes.POINTER(ctypes.c_double)]),
        "fd_measure_issue_overlap": (I32, [I32, I32, P, ctypes.POINTER(ctypes.c_double)]),
        "fd_quantize_e4m3_rows": (I32, [P, I64, I64, P, P]),
        "fd_quantize_e4m3_rows_device": (I32, [P, I64, I64, P, P, P]),
        "fd_pack_e4m3_weight": (I32, [P, I64, I64, P]),
        "fd_fp8_act_count": (SZ, [P]),
        "fd_set_fp8_act_amax": (I32, [P, P, SZ]),
        "fd_calibrate_chunk": (I32, [P, P, I32, I32, P, P, P, SZ, P]),
        "fd_gemm_e4m3_device": (I32, [P, I64, P, P, P, P, I32, I32, I32, I32, P, I64, P]),
        "fd_rope_frequencies": (I32, [I32, ctypes.c_double, I32] + [ctypes.c_double] * 4 +
                                [P, ctypes.POINTER(ctypes.c_float)]),
        "fd_rope_device": (I32, [P, P, I32, I64, I32, I32, I64, I64, P, P, I64, I64, P]),
        "fd_token_slots_workspace": (I32, [I32, I32, I32, I32, ctypes.POINTER(SZ)]),
        "fd_token_slots_device": (I32, [P, P, I32, I32, I32, P, I32, I32, I32, P, P, SZ, P]),
        "fd_token_append_device": (I32, [P, P, P, P, P, P, I32, P, P, P, P]),
        "fd_token_attend_workspace": (I32, [P, I32, I32, I32, ctypes.POINTER(SZ)]),
        "fd_token_attend_device": (I32, [P, P, P, I32, I32, P, ctypes.c_float, I32, P, P, P, ctypes.c_float, P, P, SZ, P]),
        "fd_status_string": (ctypes.c_char_p, [I32]),
        "fd_last_error": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sigs.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


def _check(st: int) -> None:
    if st != FD_OK:
        lib = load_library()
        raise FlashDecoderError(st, lib.fd_last_error().decode())


def make_config(model, max_batch: int = 1, max_frames_per_call: int = 4) -> fd_config:
    """fd_config from a workloads.ModelConfig-like object (attribute names match)."""
    c = fd_config()
    c.struct_size = ctypes.sizeof(fd_config)
    c.compute_dtype = _DTYPES[model.compute_dtype]
    for f in ("latent_channels", "latent_h", "latent_w", "patch", "dim", "n_heads",
              "n_kv_groups", "n_backbone_blocks", "n_refine_blocks", "mlp_hidden",
              "head_hidden", "r_t", "s_out", "out_channels", "window", "unit_frames"):
        setattr(c, f, int(getattr(model, f)))
    c.mlp_kind = {"swiglu": 0, "gelu": 1}[model.mlp_kind]
    c.norm_kind = {"rms": 0, "ln": 1}[model.norm_kind]
    c.head_kind = {"temporal_first": 0, "linear": 1}[model.head_kind]
    c.kv_norm = int(model.kv_norm)
    c.rope = int(model.rope)
    c.rope_theta = float(model.rope_theta)
    c.norm_eps = float(model.norm_eps)
    c.clamp_output = int(model.clamp_output)
    c.mlp_precision = {"f16": 0, "fp8": 1, "fp8s": 2}[getattr(model, "mlp_precision", "f16")]
    c.max_batch = max_batch
    c.max_frames_per_call = max_frames_per_call
    return c


def fd_config_validate(cfg: fd_config) -> int:
    return load_library().fd_config_validate(ctypes.byref(cfg))


def fd_weights_layout(cfg: fd_config):
    """[(name, shape, offset)] in canonical order and the total element count."""
    lib = load_library()
    n_t, n_e = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib.fd_weights_layout(ctypes.byref(cfg), None, 0, ctypes.byref(n_t), ctypes.byref(n_e)))
    descs = (fd_tensor_desc * n_t.value)()
    _check(lib.fd_weights_layout(ctypes.byref(cfg), descs, n_t.value, None, None))
    out = []
    for d in descs:
        shape = tuple(int(d.shape[i]) for i in range(d.ndim))
        out.append((d.name.decode(), shape, int(d.offset)))
    return out, n_e.value


def pack_weights(cfg: fd_config, weights: Dict[str, np.ndarray]) -> np.ndarray:
    """Concatenate named arrays into the library's canonical fp32 blob."""
    layout, total = fd_weights_layout(cfg)
    blob = np.empty(total, dtype=np.float32)
    for name, shape, off in layout:
        a = np.asarray(weights[name], dtype=np.float32)
        if a.shape != shape:
            raise ValueError(f"{name}: shape {a.shape} != layout {shape}")
        blob[off:off + a.size] = a.ravel()
    return blob


def fd_decoder_create(cfg: fd_config, blob: np.ndarray) -> int:
    lib = load_library()
    blob = np.ascontiguousarray(blob, dtype=np.float32)
    h = ctypes.c_void_p()
    _check(lib.fd_decoder_create(ctypes.byref(cfg), blob.ctypes.data, FD_DTYPE_F32, blob.size,
                                 ctypes.byref(h)))
    return h.value


def fd_decoder_destroy(dec: int) -> None:
    load_library().fd_decoder_destroy(dec)


def fd_kv_cache_create(dec: int, batch: int = 1) -> int:
    h = ctypes.c_void_p()
    _check(load_library().fd_kv_cache_create(dec, batch, ctypes.byref(h)))
    return h.value


def fd_kv_cache_reset(cache: int) -> None:
    _check(load_library().fd_kv_cache_reset(cache))


def fd_kv_cache_position(cache: int) -> int:
    return load_library().fd_kv_cache_position(cache)


def fd_kv_cache_destroy(cache: int) -> None:
    load_library().fd_kv_cache_destroy(cache)


def fd_output_shape(dec: int, batch: int, n_frames: int):
    arr = (ctypes.c_int64 * 5)()
    _check(load_library().fd_output_shape(dec, batch, n_frames, arr))
    return tuple(arr)


def _latent_dtype(t) -> int:
    import torch
    return {torch.float32: FD_DTYPE_F32, torch.bfloat16: FD_DTYPE_BF16,
            torch.float16: FD_DTYPE_F16}[t.dtype]


def _stream_handle(stream) -> int:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def fd_decode_chunk(dec: int, latent, n_frames: int, cache: int, out, stream=None) -> None:
    """latent, out: contiguous torch tensors on the decoder's GPU."""
    _check(load_library().fd_decode_chunk(dec, latent.data_ptr(), _latent_dtype(latent), n_frames,
                                          cache, out.data_ptr(), _stream_handle(stream)))


def fd_decode_chunk_noalloc(dec: int, latent, n_frames: int, cache: int, out, stream=None) -> None:
    """fd_decode_chunk with the activation workspace in the library's fixed
    per-GPU array (no device allocation); latent, out as for fd_decode_chunk."""
    _check(load_library().fd_decode_chunk_noalloc(dec, latent.data_ptr(), _latent_dtype(latent), n_frames,
                                                  cache, out.data_ptr(), _stream_handle(stream)))


FD_PIXELS_F32, FD_PIXELS_BF16, FD_PIXELS_U8 = 0, 1, 2


def pixel_torch_dtype(out_format: int):
    import torch
    return {FD_PIXELS_F32: torch.float32, FD_PIXELS_BF16: torch.bfloat16,
            FD_PIXELS_U8: torch.uint8}[out_format]


def _check_out(out, out_format: int) -> None:
    if out.dtype != pixel_torch_dtype(out_format) or not out.is_contiguous():
        raise ValueError(f"out must be a contiguous {pixel_torch_dtype(out_format)} tensor")


def fd_decode_chunk_as(dec: int, latent, n_frames: int, cache: int, out, out_format: int,
                       stream=None) -> None:
    """fd_decode_chunk with pixels in out_format (FD_PIXELS_*); out's dtype must match."""
    _check_out(out, out_format)
    _check(load_library().fd_decode_chunk_as(dec, latent.data_ptr(), _latent_dtype(latent), n_frames,
                                             cache, out.data_ptr(), out_format, _stream_handle(stream)))


def fd_decode_chunks(dec: int, latents, n_frames: int, caches, outs, out_format: int,
                     stream=None) -> None:
    """One chunk for each of len(caches) independent caches, run concurrently."""
    n = len(caches)
    if not (len(latents) == len(outs) == n):
        raise ValueError("latents, caches and outs must have the same length")
    dts = {_latent_dtype(z) for z in latents}
    if len(dts) != 1:
        raise ValueError("all latents must have the same dtype")
    for o in outs:
        _check_out(o, out_format)
    arr = ctypes.c_void_p * n
    _check(load_library().fd_decode_chunks(
        dec, n, arr(*[z.data_ptr() for z in latents]), dts.pop(), n_frames, arr(*caches),
        arr(*[o.data_ptr() for o in outs]), out_format, _stream_handle(stream)))


def fd_decode_chunk_trace(dec: int, latent, n_frames: int, cache: int, out, trace,
                          stream=None) -> None:
    _check(load_library().fd_decode_chunk_trace(
        dec, latent.data_ptr(), _latent_dtype(latent), n_frames, cache, out.data_ptr(),
        _stream_handle(stream), trace.data_ptr(), trace.numel()))


def fd_trace_elems(dec: int, batch: int, n_frames: int) -> int:
    return load_library().fd_trace_elems(dec, batch, n_frames)


def fd_probe_enable(cache: int, kernel_class: int) -> None:
    _check(load_library().fd_probe_enable(cache, kernel_class))


def fd_probe_read(cache: int):
    ms, n, w = ctypes.c_double(), ctypes.c_int64(), ctypes.c_double()
    _check(load_library().fd_probe_read(cache, ctypes.byref(ms), ctypes.byref(n), ctypes.byref(w)))
    return ms.value, n.value, w.value


def fd_measure_lds_bandwidth(iters: int = 20000, stream=None):
    """(bytes per shader clock per compute unit, shader clock GHz) of conflict-free
    ds_read_b128 loads on this GPU."""
    b, g = ctypes.c_double(), ctypes.c_double()
    _check(load_library().fd_measure_lds_bandwidth(iters, _stream_handle(stream),
                                                   ctypes.byref(b), ctypes.byref(g)))
    return b.value, g.value


ISSUE_OVERLAP_MODES = ("mfma", "exp4", "mfma+exp4", "fma8", "mfma+fma8", "mfma+exp4+fma4")


def fd_measure_issue_overlap(waves_per_simd: int = 1, iters: int = 20000, stream=None):
    """Shader cycles per slot and wave of the issue-overlap probe, keyed by
    ISSUE_OVERLAP_MODES (a slot: one 32x32x16 MFMA and / or vector work)."""
    c = (ctypes.c_double * 6)()
    _check(load_library().fd_measure_issue_overlap(waves_per_simd, iters, _stream_handle(stream), c))
    return dict(zip(ISSUE_OVERLAP_MODES, list(c)))


def fd_measure_mfma_peak(dtype: str = "f16", iters: int = 100000, stream=None):
    """(TFLOP/s, shader clock GHz) that a dense MFMA load sustains on this GPU."""
    tf, ghz = ctypes.c_double(), ctypes.c_double()
    _check(load_library().fd_measure_mfma_peak(_DTYPES[dtype], iters, _stream_handle(stream),
                                                ctypes.byref(tf), ctypes.byref(ghz)))
    return tf.value, ghz.value


def fd_quantize_e4m3_rows(x: np.ndarray):
    """Host E4M3 row quantisation (the FP8 MLP's weight rule): (codes uint8, scales fp32)."""
    x = np.ascontiguousarray(x, dtype=np.float32)
    rows, cols = x.shape
    codes = np.empty((rows, cols), np.uint8)
    scales = np.empty(rows, np.float32)
    _check(load_library().fd_quantize_e4m3_rows(x.ctypes.data, rows, cols, codes.ctypes.data,
                                                 scales.ctypes.data))
    return codes, scales


def fd_quantize_e4m3_rows_device(x, codes, scales, stream=None) -> None:
    """Device E4M3 row quantisation of the fp32 torch tensor x [rows, cols] into
    codes (uint8) and scales (fp32) torch tensors on the same GPU."""
    rows, cols = x.shape
    _check(load_library().fd_quantize_e4m3_rows_device(x.data_ptr(), rows, cols, codes.data_ptr(),
                                                        scales.data_ptr(), _stream_handle(stream)))


def fd_fp8_act_count(dec: int) -> int:
    return load_library().fd_fp8_act_count(dec)


def fd_set_fp8_act_amax(dec: int, amax) -> None:
    """Static FP8 amplitudes (2 per block: MLP input, SwiGLU output)."""
    a = np.ascontiguousarray(amax, dtype=np.float32)
    _check(load_library().fd_set_fp8_act_amax(dec, a.ctypes.data, a.size))


def fd_calibrate_chunk(dec: int, latent, n_frames: int, cache: int, out, amax: np.ndarray,
                       stream=None) -> None:
    """Decode one chunk with per-token FP8 scales and raise amax (float32 numpy,
    fd_fp8_act_count entries, updated in place) to the maxima seen."""
    if amax.dtype != np.float32 or not amax.flags.c_contiguous:
        raise ValueError("amax must be a contiguous float32 array")
    _check_out(out, FD_PIXELS_F32)
    _check(load_library().fd_calibrate_chunk(dec, latent.data_ptr(), _latent_dtype(latent), n_frames,
                                             cache, out.data_ptr(), amax.ctypes.data, amax.size,
                                             _stream_handle(stream)))


FD_GEMM_E4M3_RESID_ADD, FD_GEMM_E4M3_SWIGLU_F16 = 0, 1


def fd_pack_e4m3_weight(w: np.ndarray) -> np.ndarray:
    """Packed layout of an [N, K] uint8 E4M3 weight for fd_gemm_e4m3_device
    (ceil(N / 16) * 16 * K bytes)."""
    w = np.ascontiguousarray(w, dtype=np.uint8)
    n, k = w.shape
    out = np.empty(((n + 15) // 16 * 16) * k, np.uint8)
    _check(load_library().fd_pack_e4m3_weight(w.ctypes.data, n, k, out.ctypes.data))
    return out


def fd_gemm_e4m3_device(a, a_scale, w_packed, w_scale, bias, n: int, k: int, epilogue: int,
                        out, stream=None) -> None:
    """E4M3 GEMM on torch device tensors: a [M, lda] uint8 codes, a_scale [M],
    w_packed (fd_pack_e4m3_weight's bytes on the device), w_scale [N], bias
    [N] fp32, out [M, ld_out] (fp32 residual, or fp16 for the SwiGLU epilogue)."""
    m, lda = a.shape
    _check(load_library().fd_gemm_e4m3_device(
        a.data_ptr(), lda, a_scale.data_ptr(), w_packed.data_ptr(), w_scale.data_ptr(),
        bias.data_ptr(), m, n, k, epilogue, out.data_ptr(), out.stride(0), _stream_handle(stream)))


class Decoder:
    """Owns an fd_decoder built from a ModelConfig and a dict of named weights."""

    def __init__(self, model, weights: Dict[str, np.ndarray], max_batch: int = 1,
                 max_frames_per_call: int = 4):
        self.model = model
        self.cfg = make_config(model, max_batch, max_frames_per_call)
        self.handle = fd_decoder_create(self.cfg, pack_weights(self.cfg, weights))

    def output_shape(self, batch: int, n_frames: int):
        return fd_output_shape(self.handle, batch, n_frames)

    def close(self) -> None:
        if self.handle:
            fd_decoder_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KvCache:
    """Owns an fd_kv_cache (rolling KV rings + workspace) of a Decoder."""

    def __init__(self, decoder: Decoder, batch: int = 1):
        self.decoder = decoder
        self.batch = batch
        self.handle = fd_kv_cache_create(decoder.handle, batch)

    def reset(self) -> None:
        fd_kv_cache_reset(self.handle)

    def fp16_saturations(self) -> int:
        """fp16 hidden values clamped to +-65504 since the last read (then cleared)."""
        n = ctypes.c_uint64()
        _check(load_library().fd_kv_cache_fp16_saturations(self.handle, ctypes.byref(n)))
        return n.value

    @property
    def position(self) -> int:
        return fd_kv_cache_position(self.handle)

    def decode_chunk(self, latent, out=None, stream=None, out_format: int = FD_PIXELS_F32):
        """Decode latent [B, C', F, H', W'] (torch, on GPU); returns the pixels
        (fp32, or bf16 / uint8 for the other FD_PIXELS_* formats)."""
        import torch
        F = latent.shape[2]
        if out is None:
            out = torch.empty(self.decoder.output_shape(self.batch, F),
                              dtype=pixel_torch_dtype(out_format), device=latent.device)
        if out_format == FD_PIXELS_F32:
            fd_decode_chunk(self.decoder.handle, latent.contiguous(), F, self.handle, out, stream)
        else:
            fd_decode_chunk_as(self.decoder.handle, latent.contiguous(), F, self.handle, out,
                               out_format, stream)
        return out

    def close(self) -> None:
        if self.handle:
            fd_kv_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def decode_chunks(caches, latents, outs=None, out_format: int = FD_PIXELS_F32, stream=None):
    """Concurrent decode of one chunk per KvCache (all of one Decoder, distinct);
    returns the list of pixel tensors."""
    import torch
    dec = caches[0].decoder
    if any(c.decoder is not dec for c in caches):
        raise ValueError("all caches must belong to one Decoder")
    F = latents[0].shape[2]
    latents = [z.contiguous() for z in latents]
    if outs is None:
        outs = [torch.empty(dec.output_shape(c.batch, F), dtype=pixel_torch_dtype(out_format),
                            device=z.device) for c, z in zip(caches, latents)]
    fd_decode_chunks(dec.handle, latents, F, [c.handle for c in caches], outs, out_format, stream)
    return outs


# ------------------------------------------------------------------ rotary positions and the token cache

FD_ROPE_INTERLEAVED, FD_ROPE_HALF = 0, 1
_ROPE_LAYOUTS = {"interleaved": FD_ROPE_INTERLEAVED, "half": FD_ROPE_HALF}
_ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "bands": 3}


def _need(t, name: str, dtype, shape, device=None, strided: bool = False) -> None:
    """ValueError unless t is a GPU tensor of this dtype, shape and device, contiguous
    (strided: along its last dimension only)."""
    if (t.is_cuda and t.dtype is dtype and t.shape == shape and (device is None or t.device == device)
            and (t.is_contiguous() or (strided and (t.shape[-1] <= 1 or t.stride(-1) == 1)))):
        return
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must be on {device or 'a GPU'}, got {t.device}")
    raise ValueError(f"{name} must be contiguous" + (" in its last dimension" if strided else ""))


def _no_grad(hint: str) -> None:
    """For a call with a tensor that requires grad: ValueError if autograd would record it,
    which cannot see it."""
    import torch
    if torch.is_grad_enabled():
        raise ValueError(f"an input requires grad, which this call would lose: {hint}")


_INT32_MAX = 2 ** 31 - 1


def _int32(name: str, x: int) -> None:
    """ValueError for a number that the C interface's int32 would silently cut."""
    if not -_INT32_MAX - 1 <= x <= _INT32_MAX:
        raise ValueError(f"{name} {x} is no 32-bit integer")


_codes: Dict = {}  # torch dtype -> FD_DTYPE_*


def _dtype_code(t, name: str) -> int:
    if not _codes:
        import torch
        _codes.update({torch.float32: FD_DTYPE_F32, torch.bfloat16: FD_DTYPE_BF16, torch.float16: FD_DTYPE_F16})
    code = _codes.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


def _call_on(device, stream, fn, *args) -> None:
    """fn(*args, stream) with `device` current; stream defaults to its current one."""
    import torch
    index = device.index
    if stream is None:  # (the handle alone: a Stream object costs 1.5 us, a launch 3)
        handle = torch._C._cuda_getCurrentRawStream(index)
    elif stream.device != device:
        raise ValueError(f"stream of {stream.device} for tensors on {device}")
    else:
        handle = stream.cuda_stream
    if torch._C._cuda_getDevice() == index:
        st = fn(*args, handle)
    else:
        with torch.cuda.device(device):
            st = fn(*args, handle)
    if st != FD_OK:
        _check(st)


def _new(like, shape, dtype, stream, result: bool = True):
    """An uninitialised tensor on like's GPU for work on `stream` (None: the current one),
    out of that stream's memory: what the current one last freed, its work may still use.
    A result also stays until the current stream's work at its release is done."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    import torch
    if stream.device != like.device:
        raise ValueError(f"stream of {stream.device} for tensors on {like.device}")
    with torch.cuda.stream(stream):
        t = like.new_empty(shape, dtype=dtype)
    if result:
        t.record_stream(torch.cuda.current_stream(like.device))
    return t


def fd_rope_frequencies(rot_dim: int, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                        trained_length: float = 0.0, fast_turns: float = 32.0, slow_turns: float = 1.0):
    """(frequencies float64 numpy [rot_dim / 2], magnitude) of a rotary embedding;
    scaling "none", "linear", "base" or "bands"."""
    _int32("rot_dim", rot_dim)
    freq = np.empty(min(max(rot_dim, 0), 512) // 2, np.float64)  # (of more none is written)
    mag = ctypes.c_float()
    if scaling not in _ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(_ROPE_SCALINGS)}")
    _check(load_library().fd_rope_frequencies(rot_dim, theta, _ROPE_SCALINGS[scaling], factor, trained_length,
                                              fast_turns, slow_turns, freq.ctypes.data, ctypes.byref(mag)))
    return freq, mag.value


class Rope:
    """Rotary positions (fd_rope): frequencies of the pairs (float64, numpy or a GPU
    tensor), and the coordinate that turns each pair (axis, int32; None: one axis)."""

    def __init__(self, freq, axis=None, n_axes: int = 1, layout: str = "interleaved", magnitude: float = 1.0,
                 inverse: bool = False, device="cuda"):
        import torch
        if layout not in _ROPE_LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(_ROPE_LAYOUTS)}")
        if not isinstance(freq, torch.Tensor):
            freq = torch.from_numpy(np.ascontiguousarray(freq, np.float64)).to(device)
        _int32("n_axes", n_axes)
        _need(freq, "freq", torch.float64, freq.shape if freq.dim() == 1 else (freq.numel(),))
        if axis is not None:
            if not isinstance(axis, torch.Tensor):
                axis = torch.from_numpy(np.ascontiguousarray(axis, np.int32)).to(freq.device)
            _need(axis, "axis", torch.int32, freq.shape, freq.device)
        self.freq, self.axis, self.n_axes = freq, axis, n_axes
        self._s = fd_rope(ctypes.sizeof(fd_rope), 2 * freq.numel(), _ROPE_LAYOUTS[layout], n_axes, freq.data_ptr(),
                          None if axis is None else axis.data_ptr(), magnitude, int(inverse))
        self._p = ctypes.addressof(self._s)
        self._args = (layout, magnitude, inverse)

    def inverted(self) -> "Rope":
        """The opposite rotation (its result is also the gradient of this one)."""
        layout, magnitude, inverse = self._args
        return Rope(self.freq, self.axis, self.n_axes, layout, magnitude, not inverse)

    def __call__(self, x, coords, out=None, stream=None):
        """Rotate x [tokens, heads, head_dim] (fp32, bf16 or fp16; strided) at coords
        [tokens] or [tokens, n_axes] (int32); out may be x. Autograd does not see it: the
        gradient of x is ``inverted()`` of out's, and an x that requires grad is refused
        while gradients are recorded."""
        import torch
        if x.requires_grad or (out is not None and out.requires_grad):
            _no_grad("rotate under torch.no_grad() and turn its gradient back with inverted()")
        tokens, heads, dim = x.shape
        dt, dev = _dtype_code(x, "x"), self.freq.device
        _need(x, "x", x.dtype, x.shape, dev, strided=True)
        _need(coords, "coords", torch.int32, (tokens, self.n_axes) if coords.dim() == 2 or self.n_axes > 1 else (tokens,),
              dev)
        if out is None:
            out = _new(x, x.shape, x.dtype, stream)
        else:
            _need(out, "out", x.dtype, x.shape, dev, strided=True)
        _call_on(dev, stream, load_library().fd_rope_device, self._p, x.data_ptr(), dt, tokens, heads, dim,
                 x.stride(0), x.stride(1), coords.data_ptr(), out.data_ptr(), out.stride(0), out.stride(1))
        return out


def fd_token_slots_device(slot_pos, weight, pos, slots, keep_first: int = 0, keep_recent: int = 0,
                          stream=None) -> None:
    """Slots (int32 [batch, groups, n]) for n new tokens at pos (int32 [batch, n], < 0:
    padding) of a cache with positions slot_pos and weights [batch, groups, capacity]."""
    import torch
    if abs(keep_first) > _INT32_MAX or abs(keep_recent) > _INT32_MAX:  # (ctypes cuts them in silence)
        raise ValueError(f"keep_first {keep_first} and keep_recent {keep_recent} must be in [0, 2^31)")
    B, G, C = slot_pos.shape
    n, dev = pos.shape[-1], slot_pos.device
    _need(slot_pos, "slot_pos", torch.int32, slot_pos.shape)
    _need(weight, "weight", torch.float32, slot_pos.shape, dev)
    _need(pos, "pos", torch.int32, (B, n), dev)
    _need(slots, "slots", torch.int32, (B, G, n), dev)
    lib, size, ws = load_library(), 0, None
    if C > 16384:  # (smaller choices need no workspace)
        b = ctypes.c_size_t()
        _check(lib.fd_token_slots_workspace(B, G, C, n, ctypes.byref(b)))
        size = b.value
        ws = _new(slots, (size,), torch.uint8, stream, result=False)
    _call_on(dev, stream, lib.fd_token_slots_device, slot_pos.data_ptr(), weight.data_ptr(), B, G, C, pos.data_ptr(), n,
             keep_first, keep_recent, slots.data_ptr(), None if ws is None else ws.data_ptr(), size)


class TokenCache:
    """A key / value cache with a token budget over caller tensors: k, v [batch, groups,
    capacity, head_dim] (strided), pos int32 and weight fp32 [batch, groups, capacity].

    A step of a stream: ``insert`` the new tokens' keys and values (the least attended
    tokens make room), then ``attend`` with their queries, which adds to the weights.

    For serving: no gradient passes, and tensors that require one are refused while
    gradients are recorded."""

    _SERVING = "call it under torch.no_grad() or detach it"

    def __init__(self, k, v, pos, weight):
        import torch
        B, G, C, D = k.shape
        dt, dev = _dtype_code(k, "k"), k.device
        _need(k, "k", k.dtype, k.shape, None, strided=True)
        _need(v, "v", k.dtype, k.shape, dev, strided=True)
        _need(pos, "pos", torch.int32, (B, G, C), dev)
        _need(weight, "weight", torch.float32, (B, G, C), dev)
        self.k, self.v, self.pos, self.weight = k, v, pos, weight
        self.batch, self.groups, self.capacity, self.head_dim = B, G, C, D
        I3 = ctypes.c_int64 * 3
        self._s = fd_token_cache(ctypes.sizeof(fd_token_cache), dt, B, G, C, D, k.data_ptr(), v.data_ptr(),
                                 I3(*k.stride()[:3]), I3(*v.stride()[:3]), pos.data_ptr(), weight.data_ptr())
        self._p = ctypes.addressof(self._s)
        self._ws = {}

    @classmethod
    def empty(cls, batch: int, groups: int, capacity: int, head_dim: int, dtype, device="cuda") -> "TokenCache":
        """A cache with memory of its own and every slot empty."""
        import torch
        shape = (batch, groups, capacity)
        k, v = (torch.zeros(*shape, head_dim, dtype=dtype, device=device) for _ in range(2))
        return cls(k, v, torch.full(shape, -1, dtype=torch.int32, device=device),
                   torch.zeros(shape, dtype=torch.float32, device=device))

    def reset(self) -> None:
        """Forget every token (on the current stream)."""
        self.pos.fill_(-1)

    def choose(self, pos, keep_first: int = 0, keep_recent: int = 0, stream=None):
        """Slots [batch, groups, n] for new tokens at pos [batch, n] (fd_token_slots_device)."""
        import torch
        slots = _new(self.pos, (self.batch, self.groups, pos.shape[-1]), torch.int32, stream)
        fd_token_slots_device(self.pos, self.weight, pos, slots, keep_first, keep_recent, stream)
        return slots

    def append(self, k, v, pos, slots, rope: Optional[Rope] = None, coords=None, stream=None) -> None:
        """Write k (rotated by rope at coords [batch, n, n_axes] or, for one axis, [batch, n];
        default pos) and v
        [batch, n, groups, head_dim] into their slots (fd_token_append_device)."""
        import torch
        if k.requires_grad or v.requires_grad or self.k.requires_grad or self.v.requires_grad:
            _no_grad(self._SERVING)
        dev, n = self.pos.device, pos.shape[-1]
        shape = (self.batch, n, self.groups, self.head_dim)
        _need(k, "k", self.k.dtype, shape, dev, strided=True)
        _need(v, "v", self.k.dtype, shape, dev, strided=True)
        _need(pos, "pos", torch.int32, (self.batch, n), dev)
        _need(slots, "slots", torch.int32, (self.batch, self.groups, n), dev)
        if coords is not None:
            axes = rope.n_axes if rope else 1
            _need(coords, "coords", torch.int32, (self.batch, n, axes) if coords.dim() == 3 or axes > 1 else
                  (self.batch, n), dev)
        if rope is not None and rope.freq.device != dev:
            raise ValueError(f"rope on {rope.freq.device} for a cache on {dev}")
        I3 = ctypes.c_int64 * 3
        _call_on(dev, stream, load_library().fd_token_append_device, self._p, None if rope is None else rope._p,
                 k.data_ptr(), I3(*k.stride()[:3]), v.data_ptr(), I3(*v.stride()[:3]), n, pos.data_ptr(),
                 None if coords is None else coords.data_ptr(), slots.data_ptr())

    def insert(self, k, v, pos, rope: Optional[Rope] = None, coords=None, keep_first: int = 0,
               keep_recent: int = 0, stream=None):
        """choose, then append; returns the slots."""
        slots = self.choose(pos, keep_first, keep_recent, stream)
        self.append(k, v, pos, slots, rope, coords, stream)
        return slots

    def attend(self, q, pos, scale: Optional[float] = None, causal: bool = True, track: bool = True,
               decay: float = 1.0, weight_out=None, out=None, stream=None):
        """Attention of q [batch, n, heads, head_dim] at pos [batch, n] over the cache
        (fd_token_attend_device); scale defaults to head_dim ** -0.5. Returns (out, lse
        [batch, heads, n]). With track the slots' weights become decay x weight + what
        they received, in place or in weight_out."""
        import torch
        if (q.requires_grad or self.k.requires_grad or self.v.requires_grad
                or (out is not None and out.requires_grad)):
            _no_grad(self._SERVING)
        B, n, heads, D = q.shape
        dev = self.pos.device
        _need(q, "q", self.k.dtype, (self.batch, n, heads, self.head_dim), dev, strided=True)
        _need(pos, "pos", torch.int32, (B, n), dev)
        if weight_out is not None:
            _need(weight_out, "weight_out", torch.float32, self.weight.shape, dev)
        elif track:
            weight_out = self.weight
        if out is None:
            out = _new(q, q.shape, q.dtype, stream)
        else:
            _need(out, "out", q.dtype, q.shape, dev, strided=True)
        lse = _new(self.weight, (B, heads, n), torch.float32, stream)
        lib, I3 = load_library(), ctypes.c_int64 * 3
        key = (heads, n, weight_out is not None)
        size = self._ws.get(key)
        if size is None:  # (a number that follows from the sizes; the memory is each call's own)
            b = ctypes.c_size_t()
            _check(lib.fd_token_attend_workspace(self._p, heads, n, int(key[2]), ctypes.byref(b)))
            size = self._ws[key] = b.value
        ws = _new(q, (size,), torch.uint8, stream, result=False)
        _call_on(dev, stream, lib.fd_token_attend_device, self._p, q.data_ptr(), I3(*q.stride()[:3]), heads, n,
                 pos.data_ptr(), D ** -0.5 if scale is None else scale, int(causal), out.data_ptr(),
                 I3(*out.stride()[:3]), lse.data_ptr(), decay,
                 None if weight_out is None else weight_out.data_ptr(), ws.data_ptr(), size)
        return out, lse
