"""Thin ctypes binding of the C-ABI library (``include/phyai.h``): argument marshalling only.

Every step of the denoising loop runs inside the CUDA library; PyTorch is used here for device
memory and streams.  There is no CPU fallback: loading fails loudly when ``libphyai.so`` has not
been built, and every compute call fails without a CUDA device.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libphyai.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_OOM, ERR_CUDA, ERR_TIMEOUT = range(6)
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "OOM", 4: "CUDA", 5: "TIMEOUT"}
DTYPES = {"f32": 0, "bf16": 1, "w8e4m3": 2, "w8a8e4m3": 3, "w4a16": 4}
CONDS = {"pi0": 0, "pi05": 1}
ENGINES = {"auto": 0, "simt": 1}
BIG = ("wq", "wk", "wv", "wo", "wgate", "wup", "wdown")

#: every symbol the header declares
EXPORTS = ("phyai_expert_create", "phyai_expert_destroy", "phyai_prefix_kv_bytes", "phyai_denoise",
           "phyai_denoise_batched", "phyai_denoise_host", "phyai_denoise_batched_host", "phyai_denoise_requests_host", "phyai_requests_staging_bytes", "phyai_poll_status",
           "phyai_set_option", "phyai_launches_per_call", "phyai_last_error", "phyai_version",
           "phyai_suffix_attention", "phyai_suffix_attention_cleared", "phyai_suffix_attention_scratch_bytes", "phyai_op_last_error",
           "phyai_suffix_attention_static", "phyai_suffix_attention_static_capacity", "phyai_read_trace",
           "phyai_pack_prefix_kv", "phyai_pack_prefix_kv_cleared", "phyai_postprocess_actions", "phyai_adapter_last_error", "phyai_batcher_create",
           "phyai_batcher_destroy", "phyai_batcher_submit", "phyai_batcher_next", "phyai_batcher_pending",
           "phyai_batcher_plan", "phyai_w8a8_project", "phyai_w8a8_last_error", "phyai_project_features_kv", "phyai_kv_projector_create",
           "phyai_kv_projector_run", "phyai_kv_projector_destroy", "phyai_norm_rope_heads", "phyai_append_paged_kv", "phyai_paged_attention",
           "phyai_paged_attention_workspace_bytes", "phyai_pack_paged_kv", "phyai_paged_set_option", "phyai_paged_last_error")


class PhyaiError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"phyai status {STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class ConfigStruct(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in
                ("struct_size", "n_layers", "width", "mlp_dim", "n_q_heads", "n_kv_heads", "head_dim", "state_dim",
                 "action_dim", "horizon", "has_state_token", "max_prefix_len", "max_batch", "cond", "dtype")] + \
               [(n, C.c_float) for n in ("rms_eps", "rope_theta", "time_min_period", "time_max_period")] + \
               [(n, C.c_uint32) for n in ("gelu_exact", "suffix_block_causal", "engine")]


_VP = C.c_void_p
_VPP = C.POINTER(C.c_void_p)


class AttentionDesc(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "n_q_heads", "n_kv_heads", "head_dim", "suffix_len",
                                          "n_layers", "layer", "state_token_block_causal", "num_splits")]


class KvPackDesc(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "n_layers", "n_kv_heads", "head_dim", "elem_bytes", "batch",
                                          "p_max")]


_KV_PACK_SIZE = C.sizeof(KvPackDesc)


class PagedCacheDesc(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "n_layers", "n_kv_heads", "head_dim", "page_size", "dtype")] + \
               [("n_pages", C.c_uint64), ("pages", C.c_void_p)]


class HeadsDesc(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "n_q_heads", "n_kv_heads", "head_dim", "in_dtype", "out_dtype")] + [("eps", C.c_float)]


class BatcherConfig(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "max_batch", "n_workers", "local_batch")] + [("window_ms", C.c_double)]


class WeightsStruct(C.Structure):
    _fields_ = [(n, _VP) for n in
                ("state_w", "state_b", "action_in_w", "action_in_b", "time_mlp1_w", "time_mlp1_b", "time_mlp2_w",
                 "time_mlp2_b", "action_out_w", "action_out_b", "final_norm", "final_norm_b")] + \
               [(n, _VPP) for n in ("wq", "wk", "wv", "wo", "wgate", "wup", "wdown",
                                    "norm1", "norm1_b", "norm2", "norm2_b")] + \
               [("scales", _VPP * 7)]


_lib = None


def load_library() -> C.CDLL:
    """Load ``libphyai.so`` (built by ``paper_2608_03682_b200.build``); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2608_03682_b200.build` "
                           "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    lib.phyai_last_error.restype = C.c_char_p
    lib.phyai_version.restype = C.c_char_p
    lib.phyai_prefix_kv_bytes.restype = C.c_size_t
    lib.phyai_prefix_kv_bytes.argtypes = [C.POINTER(ConfigStruct), C.c_uint64]
    lib.phyai_expert_create.argtypes = [C.POINTER(ConfigStruct), C.POINTER(WeightsStruct), _VP, C.POINTER(_VP)]
    lib.phyai_expert_destroy.argtypes = [_VP]
    lib.phyai_expert_destroy.restype = None
    single = [_VP, _VP, C.c_uint64, C.c_uint32, _VP, _VP, C.c_uint32, _VP, _VP]
    batched = [_VP, C.c_uint32, _VP, C.c_uint64, _VP, _VP, _VP, C.c_uint32, _VP, _VP]
    lib.phyai_denoise.argtypes = single
    lib.phyai_denoise_host.argtypes = single
    lib.phyai_denoise_batched.argtypes = batched
    lib.phyai_denoise_batched_host.argtypes = batched
    lib.phyai_denoise_requests_host.argtypes = [_VP, C.c_uint32, _VP, _VP, _VP, _VP, C.c_uint32, _VP, _VP, C.c_uint64, _VP]
    lib.phyai_requests_staging_bytes.argtypes, lib.phyai_requests_staging_bytes.restype = [_VP, C.c_uint32, C.c_uint64], C.c_uint64
    lib.phyai_poll_status.argtypes = [_VP]
    lib.phyai_set_option.argtypes = [_VP, C.c_char_p, C.c_int64]
    lib.phyai_read_trace.argtypes = [_VP, _VP, C.c_size_t, C.POINTER(C.c_uint32), C.POINTER(C.c_uint32)]
    lib.phyai_launches_per_call.argtypes = [_VP, C.c_uint32, C.c_uint32]
    lib.phyai_launches_per_call.restype = C.c_uint64
    lib.phyai_op_last_error.restype = C.c_char_p
    lib.phyai_suffix_attention_scratch_bytes.restype = C.c_size_t
    lib.phyai_suffix_attention_scratch_bytes.argtypes = [C.POINTER(AttentionDesc), C.c_uint32]
    lib.phyai_suffix_attention.argtypes = [C.POINTER(AttentionDesc), C.c_uint32, _VP, _VP, C.c_uint64, _VP, _VP, _VP,
                                           _VP, _VP]
    lib.phyai_suffix_attention_static.argtypes = lib.phyai_suffix_attention.argtypes
    lib.phyai_suffix_attention_cleared.argtypes = lib.phyai_suffix_attention.argtypes
    lib.phyai_suffix_attention_static_capacity.restype = C.c_size_t
    lib.phyai_pack_prefix_kv.argtypes = [C.POINTER(KvPackDesc), _VP, _VP, _VP, _VP, C.c_uint64, _VP, _VP, _VP]
    lib.phyai_pack_prefix_kv_cleared.argtypes = lib.phyai_pack_prefix_kv.argtypes
    lib.phyai_postprocess_actions.argtypes = [_VP, C.c_uint32, C.c_uint32, C.c_uint32, _VP, _VP, C.c_float, C.c_float,
                                              C.c_uint32, C.c_uint32, _VP, _VP]
    lib.phyai_adapter_last_error.restype = C.c_char_p
    lib.phyai_w8a8_project.argtypes = [_VP, _VP, _VP, C.c_uint32, C.c_uint32, C.c_uint32, _VP, _VP, _VP, _VP]
    lib.phyai_w8a8_last_error.restype = C.c_char_p
    lib.phyai_project_features_kv.argtypes = [_VP, _VP, _VP, _VP, C.c_uint64, C.c_uint64, _VP, _VP]
    lib.phyai_kv_projector_create.argtypes = [_VP, _VP, _VP, C.c_uint64, _VP, C.POINTER(_VP)]
    lib.phyai_kv_projector_run.argtypes = [_VP, _VP, C.c_uint64, C.c_uint64, _VP, _VP]
    lib.phyai_kv_projector_destroy.argtypes = [_VP]
    lib.phyai_kv_projector_destroy.restype = None
    lib.phyai_batcher_create.argtypes = [C.POINTER(BatcherConfig), C.POINTER(_VP)]
    lib.phyai_batcher_destroy.argtypes = [_VP]
    lib.phyai_batcher_destroy.restype = None
    lib.phyai_batcher_submit.argtypes = [_VP, C.c_uint64]
    lib.phyai_batcher_next.argtypes = [_VP, C.c_double, C.POINTER(C.c_uint64), C.POINTER(C.c_uint32)]
    lib.phyai_batcher_pending.argtypes = [_VP]
    lib.phyai_batcher_pending.restype = C.c_uint32
    lib.phyai_batcher_plan.argtypes = [C.POINTER(BatcherConfig), C.c_uint32, C.POINTER(C.c_int32), C.POINTER(C.c_uint32)]
    u32, u64 = C.c_uint32, C.c_uint64
    lib.phyai_norm_rope_heads.argtypes = [_VP, u32, _VP, u64, _VP, u64, _VP, _VP, u64, _VP, _VP, _VP, _VP, _VP, _VP]
    lib.phyai_append_paged_kv.argtypes = [_VP, _VP, u32, u32, _VP, u64, _VP, u64, _VP, u64, u32, _VP, _VP, _VP, u32, _VP, _VP, u64, _VP, _VP,
                                          _VP, _VP, _VP]
    lib.phyai_paged_attention.argtypes = [_VP, u32, u32, u32, _VP, u64, u32, _VP, _VP, _VP, u32, u32, _VP, C.c_float, _VP, _VP, C.c_size_t, _VP, _VP]
    lib.phyai_paged_attention_workspace_bytes.argtypes = [_VP, u32, u32, u32, u32]
    lib.phyai_paged_attention_workspace_bytes.restype = C.c_size_t
    lib.phyai_pack_paged_kv.argtypes = [_VP, u32, _VP, _VP, u32, _VP, u64, _VP, _VP, _VP]
    lib.phyai_paged_set_option.argtypes = [C.c_char_p, C.c_int64]
    lib.phyai_paged_last_error.restype = C.c_char_p
    _lib = lib
    return lib


def _check(status: int):
    if status != OK:
        raise PhyaiError(status, load_library().phyai_last_error().decode())


def make_config_struct(cfg, engine: str = "auto") -> ConfigStruct:
    s = ConfigStruct()
    s.struct_size = C.sizeof(ConfigStruct)
    for n in ("n_layers", "width", "mlp_dim", "n_q_heads", "n_kv_heads", "head_dim", "state_dim", "action_dim",
              "horizon", "max_prefix_len", "max_batch"):
        setattr(s, n, int(getattr(cfg, n)))
    s.has_state_token = int(bool(cfg.has_state_token))
    s.cond = CONDS[cfg.cond]
    s.dtype = DTYPES[cfg.dtype]
    s.rms_eps, s.rope_theta = cfg.rms_eps, cfg.rope_theta
    s.time_min_period, s.time_max_period = cfg.time_min_period, cfg.time_max_period
    s.gelu_exact = int(bool(cfg.gelu_exact))
    s.suffix_block_causal = int(bool(cfg.suffix_block_causal))
    s.engine = ENGINES[engine]
    return s


def prefix_kv_bytes(cfg, tokens: int) -> int:
    s = make_config_struct(cfg)
    return int(load_library().phyai_prefix_kv_bytes(C.byref(s), tokens))


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


def _raw_stream(stream, device: torch.device) -> int:
    """cudaStream_t of ``stream`` (the device's current stream when None) as an integer."""
    return torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream.cuda_stream


class Expert:
    """One action expert on the current CUDA device.  ``weights``: name -> CUDA tensor (per-layer
    names suffixed ``.{layer}``); for the e4m3 mode the seven big matrices are ``(codes, scales)``."""

    def __init__(self, cfg, weights: Dict[str, object], engine: str = "auto", stream=None):
        self.lib = load_library()
        self.cfg = cfg
        self._handle = _VP()
        cs = make_config_struct(cfg, engine)
        ws = WeightsStruct()
        keep = []
        L = cfg.n_layers

        def dev(t):
            if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()):
                raise ValueError("weights must be contiguous CUDA tensors")
            keep.append(t)
            return t.data_ptr()

        for n in ("state_w", "state_b", "action_in_w", "action_in_b", "time_mlp1_w", "time_mlp1_b", "time_mlp2_w",
                  "time_mlp2_b", "action_out_w", "action_out_b", "final_norm", "final_norm_b"):
            if n in weights:
                setattr(ws, n, dev(weights[n]))
        scale_arrays = {m: (C.c_void_p * L)() for m in BIG}
        for n in ("wq", "wk", "wv", "wo", "wgate", "wup", "wdown", "norm1", "norm1_b", "norm2", "norm2_b"):
            if f"{n}.0" not in weights:
                continue
            arr = (C.c_void_p * L)()
            for l in range(L):
                w = weights[f"{n}.{l}"]
                if isinstance(w, tuple):
                    arr[l] = dev(w[0])
                    scale_arrays[n][l] = dev(w[1])
                else:
                    arr[l] = dev(w)
            keep.append(arr)
            setattr(ws, n, C.cast(arr, _VPP))
        if cfg.dtype in ("w8e4m3", "w8a8e4m3", "w4a16"):
            for i, m in enumerate(BIG):
                keep.append(scale_arrays[m])
                ws.scales[i] = C.cast(scale_arrays[m], _VPP)
        _check(self.lib.phyai_expert_create(C.byref(cs), C.byref(ws), _stream_ptr(stream), C.byref(self._handle)))
        del keep  # create has repacked everything and synchronised
        self._staged = []  # (event, buffers) of host-request calls in flight

    # ------------------------------------------------------------------------------------------
    def close(self):
        if getattr(self, "_handle", None) is not None and self._handle.value:
            self.lib.phyai_expert_destroy(self._handle)
            self._handle = _VP()
            self._staged = []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    # ------------------------------------------------------------------------------------------
    def denoise(self, prefix_kv: torch.Tensor, prefix_len: int, state: Optional[torch.Tensor], noise: torch.Tensor,
                n_steps: int, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """phyai_denoise: device tensors; ``prefix_kv`` [L,2,T,Hkv,dh]; returns ``out`` [H,A] (enqueued only)."""
        if out is None:
            out = torch.empty_like(noise)
        kv_tokens = 0 if prefix_kv is None else int(prefix_kv.shape[2])
        _check(self.lib.phyai_denoise(self._handle, _ptr(prefix_kv), kv_tokens, int(prefix_len), _ptr(state),
                                      _ptr(noise), int(n_steps), _ptr(out), _stream_ptr(stream)))
        return out

    def denoise_batched(self, prefix_kv: torch.Tensor, cu_prefix_lens: torch.Tensor, states: Optional[torch.Tensor],
                        noise: torch.Tensor, n_steps: int, out: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
        """phyai_denoise_batched: packed ``prefix_kv`` [L,2,T_total,Hkv,dh], device int32 ``cu_prefix_lens`` [B+1]."""
        if out is None:
            out = torch.empty_like(noise)
        batch = int(noise.shape[0])
        _check(self.lib.phyai_denoise_batched(self._handle, batch, _ptr(prefix_kv), int(prefix_kv.shape[2]),
                                              _ptr(cu_prefix_lens), _ptr(states), _ptr(noise), int(n_steps), _ptr(out),
                                              _stream_ptr(stream)))
        return out

    def denoise_host(self, prefix_kv: torch.Tensor, prefix_len: int, state, noise, n_steps: int, out: torch.Tensor,
                     stream=None) -> torch.Tensor:
        """phyai_denoise_host: all tensors are (ideally pinned) host tensors."""
        _check(self.lib.phyai_denoise_host(self._handle, _ptr(prefix_kv), int(prefix_kv.shape[2]), int(prefix_len),
                                           _ptr(state), _ptr(noise), int(n_steps), _ptr(out), _stream_ptr(stream)))
        return out

    def denoise_batched_host(self, prefix_kv, cu_prefix_lens, states, noise, n_steps: int, out, stream=None):
        batch = int(noise.shape[0])
        _check(self.lib.phyai_denoise_batched_host(self._handle, batch, _ptr(prefix_kv), int(prefix_kv.shape[2]),
                                                   _ptr(cu_prefix_lens), _ptr(states), _ptr(noise), int(n_steps),
                                                   _ptr(out), _stream_ptr(stream)))
        return out

    def denoise_requests_host(self, requests, n_steps: int, out: torch.Tensor, stream=None) -> torch.Tensor:
        """phyai_denoise_requests_host: ``requests`` = (prefix_kv or None, state or None, noise or None) per request, contiguous
        host tensors of the expert's storage types; ``out`` [B,H,A] (ideally pinned) is complete once the stream is.  The staging
        comes from torch's pool of page-locked memory (page-locking 60 MB anew for each handle takes 35 ms)."""
        B = len(requests)
        kv, st, nz = (_VP * B)(), (_VP * B)(), (_VP * B)()
        lens = (C.c_uint32 * B)()
        for b, (k, s, z) in enumerate(requests):
            if k is not None and k.shape[2]:
                kv[b], lens[b] = k.data_ptr(), k.shape[2]
            st[b], nz[b] = _ptr(s), _ptr(z)
        # (the pool does not know of the library's copies: buffers stay referenced until they have run)
        self._staged = [s for s in self._staged if not s[0].query()]
        staging = torch.empty(self.lib.phyai_requests_staging_bytes(self._handle, B, sum(lens)), dtype=torch.uint8, pin_memory=True)
        done = torch.cuda.Event()
        _check(self.lib.phyai_denoise_requests_host(self._handle, B, kv, lens, st, nz, int(n_steps), _ptr(out), _ptr(staging),
                                                    staging.numel(), _stream_ptr(stream)))
        done.record(torch.cuda.current_stream() if stream is None else stream)
        self._staged.append((done, staging, out))
        return out

    def poll_status(self) -> int:
        """Read-and-clear the device status word (call after synchronising); returns the status code."""
        return int(self.lib.phyai_poll_status(self._handle))

    def set_option(self, key: str, value: int):
        _check(self.lib.phyai_set_option(self._handle, key.encode(), int(value)))

    def read_trace(self) -> np.ndarray:
        """Timer stamps (ns) of the traced launches of the last call: array [slots, 16] (option "trace" = 1)."""
        buf = np.zeros(4096 * 16, dtype=np.uint64)
        n_slots, n_st = C.c_uint32(), C.c_uint32()
        _check(self.lib.phyai_read_trace(self._handle, buf.ctypes.data_as(_VP), buf.size, C.byref(n_slots),
                                         C.byref(n_st)))
        return buf.reshape(n_slots.value, n_st.value)

    def launches_per_call(self, batch: int, n_steps: int) -> int:
        return int(self.lib.phyai_launches_per_call(self._handle, batch, n_steps))


def weights_to_device(weights: Dict[str, object], device="cuda") -> Dict[str, object]:
    """Copy a generated weight dictionary to the device (tuples element-wise)."""
    out = {}
    for k, v in weights.items():
        if isinstance(v, tuple):   # (codes, scales) or (packed codes, scales, format tag)
            out[k] = tuple(t.to(device).contiguous() if hasattr(t, "to") else t for t in v)
        else:
            out[k] = v.to(device).contiguous()
    return out


def attention_desc(n_q_heads, n_kv_heads, head_dim, suffix_len, n_layers, layer, block_causal=False, num_splits=0):
    d = AttentionDesc()
    d.struct_size = C.sizeof(AttentionDesc)
    d.n_q_heads, d.n_kv_heads, d.head_dim, d.suffix_len = n_q_heads, n_kv_heads, head_dim, suffix_len
    d.n_layers, d.layer, d.state_token_block_causal, d.num_splits = n_layers, layer, int(block_causal), num_splits
    return d


def suffix_attention(desc: AttentionDesc, qkv: torch.Tensor, prefix_kv: torch.Tensor, cu_prefix_lens: torch.Tensor,
                     rope_cos_sin: Optional[torch.Tensor], entry: str = "phyai_suffix_attention", stream=None):
    """Stand-alone attention operator; returns (out bf16 [rows, Hq*dh], status_word int32 tensor)."""
    lib = _lib or load_library()
    device = qkv.device
    sp = _raw_stream(stream, device)
    batch = cu_prefix_lens.numel() - 1
    out = torch.empty(batch * desc.suffix_len, desc.n_q_heads * desc.head_dim, dtype=torch.bfloat16, device=device)
    if entry == "phyai_suffix_attention":        # (the form whose first kernel clears the word: a launch less per call)
        entry, status = "phyai_suffix_attention_cleared", torch.empty(1, dtype=torch.int32, device=device)
    else:
        with torch.cuda.stream(stream):
            status = torch.zeros(1, dtype=torch.int32, device=device)
    st = getattr(lib, entry)(C.byref(desc), batch, qkv.data_ptr(), prefix_kv.data_ptr(), prefix_kv.shape[2],
                             cu_prefix_lens.data_ptr(), _ptr(rope_cos_sin), out.data_ptr(), status.data_ptr(), sp or None)
    if st != OK:
        raise PhyaiError(st, lib.phyai_op_last_error().decode())
    return out, status


def pack_prefix_kv(k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor, kv_tokens: Optional[int] = None, stream=None):
    """Padded backbone K / V ``[L, B, p_max, Hkv, dh]`` + ``lens`` (int32 ``[B]``, device) -> the library's ragged
    layout.  Returns (prefix_kv ``[L, 2, kv_tokens, Hkv, dh]``, cu_prefix_lens int32 ``[B + 1]``, status word)."""
    lib = _lib or load_library()
    L, B, p_max, Hkv, dh = k.shape
    if kv_tokens is None:
        kv_tokens = B * p_max
    device = k.device
    sp = _raw_stream(stream, device)
    desc = KvPackDesc(_KV_PACK_SIZE, L, Hkv, dh, k.element_size(), B, p_max)
    out = torch.empty(L, 2, kv_tokens, Hkv, dh, dtype=k.dtype, device=device)
    cu = torch.empty(B + 1, dtype=torch.int32, device=device)
    status = torch.empty(1, dtype=torch.int32, device=device)
    st = lib.phyai_pack_prefix_kv_cleared(C.byref(desc), k.data_ptr(), v.data_ptr(), lens.data_ptr(), out.data_ptr(), int(kv_tokens),
                                          cu.data_ptr(), status.data_ptr(), sp or None)
    if st != OK:
        raise PhyaiError(st, lib.phyai_adapter_last_error().decode())
    return out, cu, status


def postprocess_actions(x: torch.Tensor, q01: Optional[torch.Tensor], q99: Optional[torch.Tensor], clip=(-1.0, 1.0),
                        out_horizon: Optional[int] = None, out_dim: Optional[int] = None, stream=None) -> torch.Tensor:
    """Raw chunk ``[B, H, A]`` -> clipped, un-normalised actions ``[B, out_horizon, out_dim]``."""
    lib = _lib or load_library()
    B, H, A = x.shape
    out_horizon, out_dim = out_horizon or H, out_dim or A
    out = torch.empty(B, out_horizon, out_dim, dtype=torch.float32, device=x.device)
    lo, hi = (clip if clip is not None else (0.0, 0.0))
    st = lib.phyai_postprocess_actions(_ptr(x), B, H, A, _ptr(q01), _ptr(q99), float(lo), float(hi), out_horizon, out_dim,
                                       _ptr(out), _raw_stream(stream, x.device) or None)
    if st != OK:
        raise PhyaiError(st, lib.phyai_adapter_last_error().decode())
    return out


class KvProjDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_layers", C.c_uint32), ("n_kv_heads", C.c_uint32), ("head_dim", C.c_uint32),
                ("feat_dim", C.c_uint32)]


def project_features_kv(features: torch.Tensor, wk, wv, n_kv_heads: int, head_dim: int, kv_tokens: Optional[int] = None,
                        stream=None) -> torch.Tensor:
    """Request-local K / V projections of a feature-handoff head (``phyai_project_features_kv``): ``features`` bf16
    ``[tokens, Dv]``, ``wk`` / ``wv`` lists of bf16 ``[Dv, Hkv * dh]`` -> prefix KV bf16 ``[L, 2, kv_tokens, Hkv, dh]``."""
    lib = load_library()
    tokens, Dv = features.shape
    L = len(wk)
    kv_tokens = kv_tokens or tokens
    out = torch.zeros(L, 2, kv_tokens, n_kv_heads, head_dim, dtype=torch.bfloat16, device=features.device)
    desc = KvProjDesc(C.sizeof(KvProjDesc), L, n_kv_heads, head_dim, Dv)
    ak, av = (_VP * L)(), (_VP * L)()
    for l in range(L):
        ak[l], av[l] = wk[l].data_ptr(), wv[l].data_ptr()
    st = lib.phyai_project_features_kv(C.byref(desc), _ptr(features), C.cast(ak, _VP), C.cast(av, _VP), tokens, kv_tokens,
                                       _ptr(out), _stream_ptr(stream))
    if st != OK:
        raise PhyaiError(st, lib.phyai_adapter_last_error().decode())
    return out


class KvProjector:
    """Handle form of the feature K / V projection (``phyai_kv_projector_*``): weights packed once, ``run`` only enqueues."""

    def __init__(self, wk, wv, n_kv_heads: int, head_dim: int, max_tokens: int, stream=None):
        self.lib = load_library()
        self.L, self.n_kv_heads, self.head_dim = len(wk), n_kv_heads, head_dim
        desc = KvProjDesc(C.sizeof(KvProjDesc), self.L, n_kv_heads, head_dim, wk[0].shape[0])
        ak, av = (_VP * self.L)(), (_VP * self.L)()
        for l in range(self.L):
            ak[l], av[l] = wk[l].data_ptr(), wv[l].data_ptr()
        self._h = _VP()
        st = self.lib.phyai_kv_projector_create(C.byref(desc), C.cast(ak, _VP), C.cast(av, _VP), max_tokens,
                                                _stream_ptr(stream), C.byref(self._h))
        if st != OK:
            raise PhyaiError(st, self.lib.phyai_adapter_last_error().decode())

    def run(self, features: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        tokens = features.shape[0]
        if out is None:
            out = torch.empty(self.L, 2, tokens, self.n_kv_heads, self.head_dim, dtype=torch.bfloat16, device=features.device)
        st = self.lib.phyai_kv_projector_run(self._h, _ptr(features), tokens, out.shape[2], _ptr(out), _stream_ptr(stream))
        if st != OK:
            raise PhyaiError(st, self.lib.phyai_adapter_last_error().decode())
        return out

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self.lib.phyai_kv_projector_destroy(self._h)
            self._h = _VP()

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def w8a8_project(x: torch.Tensor, w_codes: torch.Tensor, w_scales: torch.Tensor, return_codes: bool = False, stream=None):
    """Stand-alone W8A8 projection (``phyai_w8a8_project``): ``x`` bf16 ``[M, K]``, ``w_codes`` uint8 ``[K, N]``,
    ``w_scales`` float32 ``[N]`` -> float32 ``[M, N]`` (and, on request, the activation codes and scales)."""
    lib = load_library()
    M, K = x.shape
    N = w_codes.shape[1]
    y = torch.empty(M, N, dtype=torch.float32, device=x.device)
    codes = torch.empty(M, K, dtype=torch.uint8, device=x.device) if return_codes else None
    scales = torch.empty(M, dtype=torch.float32, device=x.device) if return_codes else None
    st = lib.phyai_w8a8_project(_ptr(x), _ptr(w_codes), _ptr(w_scales), M, K, N, _ptr(y), _ptr(codes), _ptr(scales),
                                _stream_ptr(stream))
    if st != OK:
        raise PhyaiError(st, lib.phyai_w8a8_last_error().decode())
    return (y, codes, scales) if return_codes else y


_STORE = {torch.float32: DTYPES["f32"], torch.bfloat16: DTYPES["bf16"]}


class _Elsewhere:
    """For a call on a given stream or another device: the device becomes the current one, outputs are allocated on the call's stream."""

    def __init__(self, device: torch.device, stream):
        if stream is not None and stream.device != device:
            raise ValueError(f"the stream is not one of {device}")
        self.device, self.stream = torch.cuda.device(device), torch.cuda.stream(stream)

    def __enter__(self):
        self.device.__enter__()
        self.stream.__enter__()

    def __exit__(self, *exc):
        self.stream.__exit__(*exc)
        self.device.__exit__(*exc)


_I32, _F32 = torch.int32, torch.float32
_current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


# (devices are compared by index, -1: not a CUDA tensor: a call's checks take a good part of the time of its launch)
def _head_rows(name: str, t: torch.Tensor, index: int, dtype: torch.dtype) -> tuple:
    """Checks rows of heads ``[T, heads, dh]`` (heads contiguous in a row); returns (T, heads, dh, row stride in elements)."""
    if t.dtype is not dtype or t.get_device() != index or t.dim() != 3:
        raise ValueError(f"{name} must be a {dtype} tensor [tokens, heads, head_dim] on cuda:{index}")
    T, H, dh = t.shape
    row, head, one = t.stride()
    if one != 1 or (head != dh and H > 1):
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    return T, H, dh, row if T > 1 else H * dh


def _ints(name: str, t: torch.Tensor, index: int, shape: tuple) -> int:
    if t.dtype is not _I32 or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on cuda:{index}")
    return t.data_ptr()


def _floats(name: str, t: Optional[torch.Tensor], index: int, shape: tuple) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not _F32 or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor {list(shape)} on cuda:{index}")
    return t.data_ptr()


def _rope(t: Optional[torch.Tensor], index: int, dh: int) -> tuple:
    """(address, positions) of a table of cosines and sines."""
    if t is None:
        return None, 0
    n = t.shape[0]
    return _floats("rope_cos_sin", t, index, (n, dh // 2, 2)), n


def _empty_rows(T: int, H: int, dh: int, dtype: torch.dtype, device: torch.device) -> torch.Tensor:
    return torch.empty_strided((T, H, dh), (H * dh, dh, 1), dtype=dtype, device=device)


_heads_descs: Dict[tuple, tuple] = {}     # sizes and types of a call's heads -> (descriptor, its address)


def _heads_desc(*key) -> int:
    d = _heads_descs.get(key)
    if d is None:
        if len(_heads_descs) >= 256:
            _heads_descs.clear()
        desc = HeadsDesc(C.sizeof(HeadsDesc), *key)
        d = _heads_descs[key] = (desc, C.addressof(desc))
    return d


def _paged_fail(lib, st: int):
    raise PhyaiError(st, lib.phyai_paged_last_error().decode())


_unread_words: Dict[int, torch.Tensor] = {}     # device index -> the status word of norm_rope_heads calls without one: written, never read


def _unread_word(index: int, device: torch.device) -> torch.Tensor:
    w = _unread_words.get(index)
    if w is None:
        w = torch.empty(1, dtype=_I32, device=device)
        if not torch.cuda.is_current_stream_capturing():     # (not out of a graph's memory)
            _unread_words[index] = w
    return w


def norm_rope_heads(q: Optional[torch.Tensor], k: torch.Tensor, positions: Optional[torch.Tensor], rope_cos_sin: Optional[torch.Tensor],
                    q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None, eps: float = 1e-6,
                    dtype: Optional[torch.dtype] = None, status: Optional[torch.Tensor] = None, stream=None):
    """Norm (gain ``1 + gain``; None: no norm) of every head of ``q`` ``[T, Hq, dh]`` and ``k`` ``[T, Hkv, dh]`` with the rotation by
    ``positions`` (int32 ``[T]``) in the same pass; rows may be columns of a fused matrix.  Returns (q, k) in ``dtype`` (default: as
    given).  The rows of a token whose position is outside the table are NaN; ``status``: int32 word that it raises as well (zeroed by the caller).
    Results carry no gradients."""
    lib = _lib or load_library()
    device, src = k.device, k.dtype
    index = device.index
    if src not in _STORE or index is None:
        raise ValueError("k must be a float32 or bfloat16 CUDA tensor [tokens, heads, head_dim]")
    if stream is not None or index != _current_device():
        with _Elsewhere(device, stream):
            return norm_rope_heads(q, k, positions, rope_cos_sin, q_gain, k_gain, eps, dtype, status)
    T, Hkv, dh, k_row = _head_rows("k", k, index, src)
    Hq, q_row, q_ptr, q_out, q_out_ptr = 0, 0, None, None, None
    if q is not None:
        Tq, Hq, dq, q_row = _head_rows("q", q, index, src)
        if Tq != T or dq != dh:
            raise ValueError("q and k differ in tokens or head_dim")
        q_ptr = q.data_ptr()
    if dtype is None:
        dtype = src
    elif dtype not in _STORE:
        raise ValueError("dtype must be float32 or bfloat16")
    desc = _heads_desc(Hq, Hkv, dh, _STORE[src], _STORE[dtype], eps)
    rope, n_pos = _rope(rope_cos_sin, index, dh)
    gq, gk = _floats("q_gain", q_gain, index, (dh,)), _floats("k_gain", k_gain, index, (dh,))
    pos = None if positions is None else _ints("positions", positions, index, (T,))
    if q is not None:
        q_out = _empty_rows(T, Hq, dh, dtype, device)
        q_out_ptr = q_out.data_ptr()
    k_out = _empty_rows(T, Hkv, dh, dtype, device)
    if status is None:
        status = _unread_word(index, device)
    st = lib.phyai_norm_rope_heads(desc[1], T, q_ptr, q_row, k.data_ptr(), k_row, pos, rope, n_pos, gq, gk, q_out_ptr, k_out.data_ptr(),
                                   _ints("status", status, index, (1,)), _current_stream(index))
    if st != OK:
        _paged_fail(lib, st)
    return q_out, k_out


def set_paged_option(key: str, value: int):
    """Option of the paged cache's calls (``phyai_paged_set_option``; testing)."""
    lib = _lib or load_library()
    st = lib.phyai_paged_set_option(key.encode(), int(value))
    if st != OK:
        _paged_fail(lib, st)


class PagedCache:
    """Pages of keys and values of every layer: ``pages`` ``[L, 2, n_pages * page_size, Hkv, dh]`` (the caller's, float32 or bfloat16).
    A call's requests: ``cu_q_lens`` int32 ``[B + 1]`` (rows of the new tokens), ``kv_lens`` int32 ``[B]`` (cached tokens with the new
    ones), ``page_table`` int32 ``[B, max_pages]``; see ``phyai.h``.  What a call finds wrong on the device raises the cache's status word
    (``poll_status``), and later calls write nothing until it has been read; a table entry that names no page leaves the call's other requests
    as they would be.  Streams: calls on the cache are ordered by the caller.  Serving only: results carry no gradients."""

    def __init__(self, pages: torch.Tensor, page_size: int):
        self.lib = load_library()
        if pages.dim() != 5 or pages.shape[1] != 2 or pages.dtype not in _STORE or not pages.is_cuda or not pages.is_contiguous():
            raise ValueError("pages must be a contiguous float32 or bfloat16 CUDA tensor [L, 2, n_pages * page_size, Hkv, dh]")
        L, _, rows, self.n_kv_heads, self.head_dim = pages.shape
        if page_size <= 0 or rows % page_size:
            raise ValueError("the pool's rows must be a multiple of page_size")
        self.pages, self.page_size, self.n_layers, self.n_pages, self.device = pages, page_size, L, rows // page_size, pages.device
        self.dtype = pages.dtype
        self._desc = PagedCacheDesc(C.sizeof(PagedCacheDesc), L, self.n_kv_heads, self.head_dim, page_size, _STORE[pages.dtype], rows // page_size,
                                    pages.data_ptr())
        self._desc_ptr = C.addressof(self._desc)
        self.status = torch.zeros(1, dtype=torch.int32, device=pages.device)
        self._status_ptr = self.status.data_ptr()
        self._sizes: Dict[tuple, int] = {}     # sizes of a call -> bytes of its workspace

    def poll_status(self, stream=None) -> int:
        """Read-and-clear the status word, once every call on the cache so far has run; returns the status code.  Waits for the device, since calls may
        be on any stream or replayed from graphs, or with ``stream`` for that one alone: the only one with such calls since the last poll."""
        if stream is not None:
            with _Elsewhere(self.device, stream):
                st = int(self.status.item())
                if st:
                    self.status.zero_()
                    stream.synchronize()
            return st
        torch.cuda.synchronize(self.device)
        st = int(self.status.item())
        if st:
            self.status.zero_()
            torch.cuda.current_stream(self.device).synchronize()       # (a next call may be on another stream)
        return st

    def _requests(self, cu_q_lens, kv_lens, page_table):
        index, shape = self.device.index, page_table.shape
        if len(shape) != 2:
            raise ValueError("page_table must be [batch, max_pages]")
        B, most = shape
        return (B, most, None if cu_q_lens is None else _ints("cu_q_lens", cu_q_lens, index, (B + 1,)), _ints("kv_lens", kv_lens, index, (B,)),
                _ints("page_table", page_table, index, shape))

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, cu_q_lens: torch.Tensor, kv_lens: torch.Tensor, page_table: torch.Tensor,
               rope_cos_sin: Optional[torch.Tensor], k_gain: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
               q_gain: Optional[torch.Tensor] = None, eps: float = 1e-6, positions: Optional[torch.Tensor] = None, stream=None):
        """New keys (normed with gain ``1 + k_gain`` unless None, rotated) and values ``[T, Hkv, dh]`` into the pages of ``layer``; with
        ``q`` ``[T, Hq, dh]`` returns its normed, rotated rows in the cache's type (rows of no request are not written), else None."""
        lib, device, index, src = self.lib, self.device, self.device.index, k.dtype
        if src not in _STORE:
            raise ValueError("k must be a float32 or bfloat16 tensor [tokens, heads, head_dim]")
        if stream is not None or index != _current_device():
            with _Elsewhere(device, stream):
                return self.append(layer, k, v, cu_q_lens, kv_lens, page_table, rope_cos_sin, k_gain, q, q_gain, eps, positions)
        T, Hkv, dh, k_row = _head_rows("k", k, index, src)
        Tv, Hv, dv, v_row = _head_rows("v", v, index, src)
        if Tv != T or Hv != Hkv or dv != dh:
            raise ValueError("k and v differ in tokens, heads or head_dim")
        Hq, q_row, q_ptr, q_out, q_out_ptr = 0, 0, None, None, None
        if q is not None:
            Tq, Hq, dq, q_row = _head_rows("q", q, index, src)
            if Tq != T or dq != dh:
                raise ValueError("q and k differ in tokens or head_dim")
            q_ptr = q.data_ptr()
        desc = _heads_desc(Hq, Hkv, dh, _STORE[src], self._desc.dtype, eps)
        B, most, cu, lens, table = self._requests(cu_q_lens, kv_lens, page_table)
        rope, n_pos = _rope(rope_cos_sin, index, dh)
        gq, gk = _floats("q_gain", q_gain, index, (dh,)), _floats("k_gain", k_gain, index, (dh,))
        pos = None if positions is None else _ints("positions", positions, index, (T,))
        if q is not None:
            q_out = _empty_rows(T, Hq, dh, self.dtype, device)
            q_out_ptr = q_out.data_ptr()
        st = lib.phyai_append_paged_kv(self._desc_ptr, desc[1], layer, T, q_ptr, q_row, k.data_ptr(), k_row, v.data_ptr(), v_row, B, cu, lens, table,
                                       most, pos, rope, n_pos, gq, gk, q_out_ptr, self._status_ptr, _current_stream(index))
        if st != OK:
            _paged_fail(lib, st)
        return q_out

    def attend(self, layer: int, q: torch.Tensor, cu_q_lens: torch.Tensor, kv_lens: torch.Tensor, page_table: torch.Tensor, causal: bool = True,
               prefix_lens: Optional[torch.Tensor] = None, scale: Optional[float] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of the new tokens' queries ``[T, Hq, dh]`` (rotated, the cache's type) over the pages of ``layer``, the tokens' own keys
        included.  ``causal``: a token sees what is cached before it and itself, and with ``prefix_lens`` (int32 ``[B]``) the first so many
        tokens.  Returns ``out`` ``[T, Hq, dh]`` (rows of no request are not written)."""
        lib, device, index = self.lib, self.device, self.device.index
        if stream is not None or index != _current_device():
            with _Elsewhere(device, stream):
                return self.attend(layer, q, cu_q_lens, kv_lens, page_table, causal, prefix_lens, scale, out)
        T, Hq, dh, row = _head_rows("q", q, index, self.dtype)
        if dh != self.head_dim:
            raise ValueError("q and the cache differ in head_dim")
        B, most, cu, lens, table = self._requests(cu_q_lens, kv_lens, page_table)
        prefix = None if prefix_lens is None else _ints("prefix_lens", prefix_lens, index, (B,))
        if out is not None and (out.shape != q.shape or out.dtype != q.dtype or out.device != device or not out.is_contiguous()):
            raise ValueError("out must be a contiguous tensor of q's shape and type")
        if scale is not None and not scale > 0.0:
            raise ValueError("scale must be positive")
        need = self._sizes.get((Hq, T, B, most))
        if need is None:
            if len(self._sizes) >= 4096:
                self._sizes.clear()
            need = self._sizes[Hq, T, B, most] = lib.phyai_paged_attention_workspace_bytes(self._desc_ptr, Hq, T, B, most)
        work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        if out is None:
            out = _empty_rows(T, Hq, dh, self.dtype, device)
        st = lib.phyai_paged_attention(self._desc_ptr, layer, Hq, T, q.data_ptr(), row, B, cu, lens, table, most, 1 if causal else 0, prefix,
                                       0.0 if scale is None else scale, out.data_ptr(), work.data_ptr() if need else None, need,
                                       self._status_ptr, _current_stream(index))
        if st != OK:
            _paged_fail(lib, st)
        return out

    def pack(self, page_table: torch.Tensor, kv_lens: torch.Tensor, kv_tokens: int, out: Optional[torch.Tensor] = None, stream=None):
        """The requests' cached tokens as the ragged prefix cache of ``Expert.denoise_batched``: (``prefix_kv`` ``[L, 2, kv_tokens, Hkv,
        dh]``, ``cu_prefix_lens`` int32 ``[B + 1]``).  ``kv_tokens``: rows of it, at least the sum of ``kv_lens`` (rows past that are not
        written)."""
        lib, device = self.lib, self.device
        if stream is not None or device.index != _current_device():
            with _Elsewhere(device, stream):
                return self.pack(page_table, kv_lens, kv_tokens, out)
        B, most, _, lens, table = self._requests(None, kv_lens, page_table)
        shape = (self.n_layers, 2, kv_tokens, self.n_kv_heads, self.head_dim)
        if out is not None and (out.shape != shape or out.dtype != self.dtype or out.device != device or not out.is_contiguous()):
            raise ValueError("out must be a contiguous tensor [L, 2, kv_tokens, Hkv, dh] of the cache's type")
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=device)
        cu = torch.empty(B + 1, dtype=torch.int32, device=device)
        st = lib.phyai_pack_paged_kv(self._desc_ptr, B, lens, table, most, out.data_ptr(), kv_tokens, cu.data_ptr(), self._status_ptr, _current_stream(device.index))
        if st != OK:
            _paged_fail(lib, st)
        return out, cu


class Batcher:
    """Batching window of the data-parallel front-end (``phyai_batcher_*``): thread-safe queue; ``next`` returns the ids
    of the batch that is due (possibly empty after ``timeout_ms``)."""

    def __init__(self, max_batch: int, n_workers: int, local_batch: int, window_ms: float):
        self.lib = load_library()
        self.cfg = BatcherConfig(C.sizeof(BatcherConfig), max_batch, n_workers, local_batch, float(window_ms))
        h = _VP()
        st = self.lib.phyai_batcher_create(C.byref(self.cfg), C.byref(h))
        if st != OK:
            raise PhyaiError(st, "bad batcher configuration")
        self._h = h

    def submit(self, request_id: int):
        self.lib.phyai_batcher_submit(self._h, int(request_id))

    def pending(self) -> int:
        return int(self.lib.phyai_batcher_pending(self._h))

    def next(self, timeout_ms: float):
        ids = (C.c_uint64 * self.cfg.max_batch)()
        n = C.c_uint32()
        st = self.lib.phyai_batcher_next(self._h, float(timeout_ms), ids, C.byref(n))
        if st != OK:
            raise PhyaiError(st, "phyai_batcher_next failed")
        return [int(ids[i]) for i in range(n.value)]

    def plan(self, n: int):
        """(slots as a list of n_workers lists of local_batch indices, -1 = padding; number of workers with a request)"""
        total = self.cfg.n_workers * self.cfg.local_batch
        slots = (C.c_int32 * total)()
        act = C.c_uint32()
        st = self.lib.phyai_batcher_plan(C.byref(self.cfg), int(n), slots, C.byref(act))
        if st != OK:
            raise PhyaiError(st, "phyai_batcher_plan: n exceeds max_batch")
        L = self.cfg.local_batch
        return [[int(slots[w * L + j]) for j in range(L)] for w in range(self.cfg.n_workers)], int(act.value)

    def close(self):
        if self._h:
            self.lib.phyai_batcher_destroy(self._h)
            self._h = None

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()
