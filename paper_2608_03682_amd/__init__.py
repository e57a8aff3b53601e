"""Python binding of the gfx950 action-expert library (``libphyai.so``).

Argument marshalling only: every step of the denoising loop runs in the HIP
kernels behind the C ABI declared in ``include/phyai.h``.  PyTorch supplies
device memory and streams.  Importing this package never falls back to a CPU
path: if the library is missing or fails to load, every call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libphyai.so")

PHYAI_OK, PHYAI_EINVAL, PHYAI_ENOMEM, PHYAI_EHIP, PHYAI_EUNSUPPORTED = 0, -1, -2, -3, -4
_VARIANT = {"pi0": 0, "pi05": 1, "dit": 2, "prefix_lm": 3, "vision": 4}
_DTYPE = {"f32": 0, "bf16": 1, "fp8": 2, "fp4": 3}

# Every symbol include/phyai.h declares.
EXPORTS = ("phyai_load_expert", "phyai_denoise", "phyai_denoise_static", "phyai_prepare", "phyai_debug_hidden",
           "phyai_profile_stage", "phyai_fp8_to_bf16", "phyai_free_expert", "phyai_last_error",
           "phyai_version", "phyai_prefill", "phyai_encode_images", "phyai_qk_norm_rope", "phyai_paged_append",
           "phyai_paged_attention", "phyai_paged_attention_workspace", "phyai_paged_gather", "phyai_prefill_paged")
STAGES = {"norm1": 0, "qkv": 1, "attn": 2, "oproj": 3, "norm2": 4, "mlp_up": 5, "mlp_down": 6}


class PhyaiError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"phyai error {code}: {msg}")
        self.code = code


class Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "variant", "n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_mlp", "horizon",
        "action_dim", "max_steps", "prefix_cap", "max_batch", "state_token", "rope", "weight_dtype",
        "kv_dtype", "d_feat", "time_dim")] + [(n, ctypes.c_float) for n in (
        "rms_eps", "sin_min_period", "sin_max_period", "rope_base")] + [(n, ctypes.c_int32) for n in (
        "n_images", "n_patches", "patch_dim", "d_out")]


class Tensor(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char_p), ("dtype", ctypes.c_int32), ("rows", ctypes.c_int32),
                ("cols", ctypes.c_int32), ("data", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


class _HeadRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("n_heads", ctypes.c_int32)]


class _PagedCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "page_table")] + [
        (n, ctypes.c_int64) for n in ("layer_stride", "page_stride", "token_stride", "head_stride")] + [
        (n, ctypes.c_int32) for n in ("dtype", "n_layers", "n_kv_heads", "head_dim", "page_size", "n_pages", "batch",
                                      "max_pages", "table_stride")]


# bits of a status word (PHYAI_PAGED_*)
PAGED_BAD_PAGE, PAGED_BAD_LENGTH = 1, 2

_lib_handle = None


def lib() -> ctypes.CDLL:
    """Load libphyai.so (raises if it is missing: there is no fallback)."""
    global _lib_handle
    if _lib_handle is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing; build it with `python -m paper_2608_03682_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.phyai_load_expert.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(Tensor), i32, vp,
                                        ctypes.POINTER(vp)]
        L.phyai_denoise.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp, vp, vp]
        L.phyai_denoise_static.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp, vp, vp]
        L.phyai_prepare.argtypes = [vp, i32, i32, vp]
        L.phyai_debug_hidden.argtypes = [vp, vp, i32, vp]
        L.phyai_fp8_to_bf16.argtypes = [vp, vp, i64, vp]
        L.phyai_profile_stage.argtypes = [vp, i32, i32, vp]
        L.phyai_prefill.argtypes = [vp, vp, vp, vp, i32, vp]
        L.phyai_encode_images.argtypes = [vp, vp, vp, i32, i32, vp]
        f32 = ctypes.c_float
        L.phyai_qk_norm_rope.argtypes = [vp] * 6 + [f32, f32, vp, vp, i32, i32, i32, i32, vp, vp]
        L.phyai_paged_append.argtypes = [vp, i32, vp, vp, f32, vp, vp, i32, i32, vp, vp]
        L.phyai_paged_attention.argtypes = [vp, i32, vp, vp, vp, vp, i32, f32, i32, i32, i32, i32, vp, i64, vp, vp]
        L.phyai_paged_attention_workspace.argtypes = [vp, i32, i32, i32]
        L.phyai_paged_gather.argtypes = [vp, vp, vp, i32, vp, vp]
        L.phyai_prefill_paged.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp, i64, vp, vp]
        L.phyai_free_expert.argtypes = [vp]
        L.phyai_free_expert.restype = None
        L.phyai_last_error.restype = ctypes.c_char_p
        for f in ("phyai_load_expert", "phyai_denoise", "phyai_denoise_static", "phyai_prepare", "phyai_debug_hidden",
                  "phyai_profile_stage", "phyai_fp8_to_bf16", "phyai_version", "phyai_prefill",
                  "phyai_encode_images", "phyai_qk_norm_rope", "phyai_paged_append", "phyai_paged_attention",
                  "phyai_paged_gather", "phyai_prefill_paged"):
            getattr(L, f).restype = ctypes.c_int
        L.phyai_paged_attention_workspace.restype = i64
        _lib_handle = L
    return _lib_handle


def _check(rc: int):
    if rc != PHYAI_OK:
        raise PhyaiError(rc, lib().phyai_last_error().decode())


def _stream(stream) -> int:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    return t.data_ptr()


def make_config(cfg, max_batch: Optional[int] = None, max_steps: Optional[int] = None) -> Config:
    """Fill the C config from any object with the workload fields."""
    return Config(
        variant=_VARIANT[cfg.variant], n_layers=cfg.n_layers, d_model=cfg.d_model,
        n_q_heads=cfg.n_q_heads, n_kv_heads=cfg.n_kv_heads, head_dim=cfg.head_dim, d_mlp=cfg.d_mlp,
        horizon=cfg.horizon, action_dim=cfg.action_dim,
        max_steps=max_steps if max_steps is not None else cfg.n_steps,
        prefix_cap=cfg.prefix_cap, max_batch=max_batch if max_batch is not None else cfg.batch,
        state_token=int(cfg.state_token), rope=int(cfg.rope), weight_dtype=_DTYPE[cfg.weight_dtype],
        kv_dtype=_DTYPE[cfg.kv_dtype], d_feat=cfg.d_feat, time_dim=cfg.time_dim,
        rms_eps=cfg.rms_eps, sin_min_period=cfg.sin_min_period, sin_max_period=cfg.sin_max_period,
        rope_base=cfg.rope_base, n_images=getattr(cfg, "n_images", 0), n_patches=getattr(cfg, "n_patches", 0),
        patch_dim=getattr(cfg, "patch_dim", 0), d_out=getattr(cfg, "d_out", 0))


def _tensor_array(weights: Dict[str, object]):
    """The C tensor list of a weight dict (and the host arrays it points into)."""
    keep = []
    arr = (Tensor * len(weights))()
    for i, (name, t) in enumerate(weights.items()):
        data = np.ascontiguousarray(t.data)
        keep.append(data)
        sc = None
        if t.scale is not None:
            sc = np.ascontiguousarray(t.scale, dtype=np.float32)
            keep.append(sc)
        nm = name.encode()
        keep.append(nm)
        # fp4 data holds two codes per byte: the logical width is twice its columns
        cols = data.shape[1] * (2 if t.dtype == "fp4" else 1)
        arr[i] = Tensor(nm, _DTYPE[t.dtype], data.shape[0], cols, data.ctypes.data,
                        None if sc is None else sc.ctypes.data)
    return arr, keep


class Expert:
    """One loaded expert (owns its device weights, buffers and graphs)."""

    def __init__(self, cfg, weights: Dict[str, object], max_batch: Optional[int] = None,
                 max_steps: Optional[int] = None, stream=None):
        self.cfg = cfg
        c = make_config(cfg, max_batch, max_steps)
        arr, keep = _tensor_array(weights)
        h = ctypes.c_void_p()
        _check(lib().phyai_load_expert(ctypes.byref(c), arr, len(weights), _stream(stream), ctypes.byref(h)))
        del keep
        self._h = h

    def prepare(self, batch: int, n_steps: int, stream=None):
        _check(lib().phyai_prepare(self._h, batch, n_steps, _stream(stream)))

    def denoise(self, prefix, prefix_len, noise, timesteps, state=None, out=None, stream=None,
                static: bool = False):
        """prefix, noise, state, out: device tensors; prefix_len, timesteps: host arrays.
        static=True calls phyai_denoise_static (allocates nothing; `out` must then be given)."""
        plen = np.ascontiguousarray(prefix_len, dtype=np.int32)
        ts = np.ascontiguousarray(timesteps, dtype=np.float32)
        B = int(noise.shape[0])
        if plen.shape[0] < B:
            raise ValueError("prefix_len shorter than the batch")
        if out is None:
            if static:
                raise ValueError("the allocation-free entry point needs a caller-provided `out`")
            import torch
            out = torch.empty_like(noise)
        fn = lib().phyai_denoise_static if static else lib().phyai_denoise
        _check(fn(self._h, _ptr(prefix), plen.ctypes.data, _ptr(noise), ts.ctypes.data,
                  len(ts) - 1, B, _ptr(state), _ptr(out), _stream(stream)))
        return out

    def debug_hidden(self, batch: int, stream=None):
        import torch
        c = self.cfg
        M = c.horizon + (1 if c.state_token else 0)
        dst = torch.empty((batch * M, c.d_model), dtype=torch.float32, device="cuda")
        _check(lib().phyai_debug_hidden(self._h, _ptr(dst), batch, _stream(stream)))
        return dst

    def profile_stage(self, stage: str, reps: int, stream=None):
        """Enqueue `reps` passes over all layers of one block stage (for timing)."""
        _check(lib().phyai_profile_stage(self._h, STAGES[stage], reps, _stream(stream)))

    def close(self):
        if getattr(self, "_h", None):
            lib().phyai_free_expert(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PrefixLM:
    """One loaded prefix LM (variant ``prefix_lm``): prefix token embeddings in,
    the prefix K/V cache an expert reads out (``phyai_prefill``)."""

    def __init__(self, cfg, weights: Dict[str, object], max_batch: Optional[int] = None, stream=None):
        if cfg.variant != "prefix_lm":
            raise ValueError("PrefixLM needs a prefix_lm config")
        import torch
        self.cfg = cfg
        c = make_config(cfg, max_batch, 0)
        arr, keep = _tensor_array(weights)
        h = ctypes.c_void_p()
        _check(lib().phyai_load_expert(ctypes.byref(c), arr, len(weights), _stream(stream), ctypes.byref(h)))
        del keep
        self._h = h
        self.device = torch.device("cuda", torch.cuda.current_device())   # where the library allocated

    def prefill(self, embeds, prefix_len, out=None, stream=None):
        """embeds: device float32 [B][prefix_cap][d]; prefix_len: host array.
        Returns (or fills) the device K/V cache [L][2][B][prefix_cap][n_kv*d_h]
        (bf16 bit patterns as int16, or float32 on the fp32 path)."""
        c = self.cfg
        plen = np.ascontiguousarray(prefix_len, dtype=np.int32)
        B = int(embeds.shape[0])
        if plen.shape[0] < B:
            raise ValueError("prefix_len shorter than the batch")
        if out is None:
            import torch
            dt = torch.float32 if c.kv_dtype == "f32" else torch.int16
            out = torch.empty((c.n_layers, 2, B, c.prefix_cap, c.n_kv_heads * c.head_dim), dtype=dt,
                              device=embeds.device)
        _check(lib().phyai_prefill(self._h, _ptr(embeds), plen.ctypes.data, _ptr(out), B, _stream(stream)))
        return out

    def prefill_paged(self, embeds, cache: "PagedCache", past_len, new_len=None, *, causal: bool = False,
                      workspace=None, status=None, stream=None) -> None:
        """Append the next tokens of each request to a paged cache of all layers
        (``phyai_prefill_paged``).  embeds: device float32 [batch][rows][d];
        past_len, new_len (default: rows): host arrays; workspace: as for
        ``paged_attention``, for the longest past_len + new_len."""
        import torch
        B, rows = int(embeds.shape[0]), int(embeds.shape[1])
        if embeds.dim() != 3 or embeds.dtype != torch.float32 or B != cache.batch or embeds.shape[2] != self.cfg.d_model:
            raise ValueError("embeds: expected float32 [batch of the cache][rows][d_model]")
        if embeds.device != cache.k.device or embeds.device != self.device:
            raise ValueError("embeds: the device must be the cache's and the handle's")
        past = _host_lengths(past_len, B, "past_len")
        new = _host_lengths(np.full(B, rows) if new_len is None else new_len, B, "new_len")
        if _elsewhere(embeds, stream):
            with _there(embeds, stream):
                return self.prefill_paged(embeds, cache, past, new, causal=causal, workspace=workspace, status=status)
        longest = max(1, int((past[:B].astype(np.int64) + new[:B]).max()))
        if workspace is None and longest <= cache.capacity and rows > 0:
            need = paged_attention_workspace(cache, self.cfg.n_q_heads, rows, longest)
            if need:
                workspace = torch.empty(need, dtype=torch.uint8, device=embeds.device)
        size = 0 if workspace is None else _bytes_of(workspace, embeds)
        _check(lib().phyai_prefill_paged(
            self._h, _ptr(embeds), cache._ref, past.ctypes.data, new.ctypes.data, rows, int(causal),
            None if workspace is None else workspace.data_ptr(), size,
            _vector(status, torch.int32, 1, embeds, "status"), _here(embeds)))

    def profile_stage(self, stage: str, reps: int, stream=None):
        """Enqueue `reps` passes over the layers of one block stage (timing aid;
        needs a previous prefill)."""
        _check(lib().phyai_profile_stage(self._h, STAGES[stage], reps, _stream(stream)))

    def close(self):
        if getattr(self, "_h", None):
            lib().phyai_free_expert(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class VisionTower:
    """One loaded vision tower (variant ``vision``): image patches in, the
    image tokens that open the prefix out (``phyai_encode_images``)."""

    def __init__(self, cfg, weights: Dict[str, object], max_batch: Optional[int] = None, stream=None):
        if cfg.variant != "vision":
            raise ValueError("VisionTower needs a vision config")
        self.cfg = cfg
        c = make_config(cfg, max_batch, 0)
        arr, keep = _tensor_array(weights)
        h = ctypes.c_void_p()
        _check(lib().phyai_load_expert(ctypes.byref(c), arr, len(weights), _stream(stream), ctypes.byref(h)))
        del keep
        self._h = h

    def encode(self, patches, out=None, out_rows: Optional[int] = None, stream=None):
        """patches: device float32 [B][n_images][n_patches][patch_dim].  Returns
        (or fills rows 0 .. n_images*n_patches-1 of each request's slab of)
        the device float32 tokens [B][out_rows][d_out]; out_rows defaults to
        out's second dimension, or n_images*n_patches for a new buffer."""
        c = self.cfg
        B = int(patches.shape[0])
        n_tok = c.n_images * c.n_patches
        if out is None:
            import torch
            out = torch.empty((B, out_rows or n_tok, c.d_out), dtype=torch.float32, device=patches.device)
        rows = out_rows if out_rows is not None else int(out.shape[1])
        _check(lib().phyai_encode_images(self._h, _ptr(patches), _ptr(out), rows, B, _stream(stream)))
        return out

    def profile_stage(self, stage: str, reps: int, stream=None):
        """Enqueue `reps` passes over the blocks of one stage (timing aid; needs
        a previous encode)."""
        _check(lib().phyai_profile_stage(self._h, STAGES[stage], reps, _stream(stream)))

    def close(self):
        if getattr(self, "_h", None):
            lib().phyai_free_expert(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------------------
# the paged key/value cache
# ---------------------------------------------------------------------------
_KINDS: Dict[object, int] = {}


def _dtype_of(t) -> int:
    """F32, BF16 (or its bit patterns as int16) and FP8E4M3 (or its codes as uint8)."""
    if not _KINDS:
        import torch
        _KINDS.update({torch.float32: 0, torch.bfloat16: 1, torch.int16: 1, torch.float8_e4m3fn: 2, torch.uint8: 2})
    d = _KINDS.get(t.dtype)
    if d is None:
        raise ValueError(f"unsupported dtype {t.dtype}")
    return d


def _in_32_bits(*values):
    """Refuses what a 32-bit argument of the library cannot hold (ctypes drops the upper bits)."""
    for x in values:
        if not -2 ** 31 <= x < 2 ** 31:
            raise ValueError(f"{x} is out of range of 32 bits")


def _head_rows(t, what: str, like=None) -> _HeadRows:
    """[batch][rows][heads][head_dim] with any strides of the first three dimensions."""
    n, s = t.shape, t.stride()
    if len(n) != 4 or not t.is_cuda:
        raise ValueError(f"{what}: expected a device tensor [batch][rows][heads][head_dim]")
    if (n[0] | n[1] | n[2] | n[3]) >> 31:
        _in_32_bits(*n)
    if s[3] != 1:
        raise ValueError(f"{what}: a head's values must be contiguous")
    if like is not None:
        m = like.shape
        if t.dtype != like.dtype or t.device != like.device or n[0] != m[0] or n[1] != m[1] or n[3] != m[3]:
            raise ValueError(f"{what}: batch, rows, head_dim, dtype and device must be those of the other rows")
    # the stride of a dimension of one is nobody's
    return _HeadRows(t.data_ptr(), s[0] if n[0] > 1 else 0, s[1] if n[1] > 1 else 0, s[2] if n[2] > 1 else 0, n[2])


def _vector(t, dtype, least: int, like, what: str) -> Optional[int]:
    """The address of a contiguous vector of at least `least` values on the call's device."""
    if t is None:
        return None
    if t.dtype != dtype or t.dim() != 1 or t.device != like.device or t.shape[0] < least or not t.is_contiguous():
        raise ValueError(f"{what}: expected {least} contiguous values of {dtype} on {like.device}")
    return t.data_ptr()


def _host_lengths(x, batch: int, what: str) -> np.ndarray:
    """Host lengths of at least `batch` requests as int32, none of them changed by that."""
    x = np.asarray(x)
    if x.ndim != 1 or x.shape[0] < batch or x.dtype.kind not in "iuf":
        raise ValueError(f"{what}: expected {batch} whole numbers")
    with np.errstate(invalid="ignore"):
        y = np.ascontiguousarray(x, dtype=np.int32)
    if not (y == x).all():
        raise ValueError(f"{what}: expected whole numbers of 32 bits")
    return y


def _bytes_of(workspace, like) -> int:
    """The bytes that a workspace owns: plain memory of the call's device."""
    if workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous tensor on {like.device}")
    return workspace.numel() * workspace.element_size()


def _elsewhere(t, stream) -> bool:
    """Whether a call has to make its device or stream the current one first."""
    import torch
    return stream is not None or t.get_device() != torch._C._cuda_getDevice()


class _there:
    """Makes the device of a call's tensors and its stream current, so that outputs and
    workspaces belong to them."""

    def __init__(self, t, stream):
        import torch
        if not t.is_cuda:
            raise ValueError("expected a device tensor")
        if stream is not None and stream.device != t.device:
            raise ValueError(f"the stream belongs to {stream.device}, the tensors to {t.device}")
        self._device, self._stream = torch.cuda.device(t.device), torch.cuda.stream(stream)

    def __enter__(self):
        self._device.__enter__()
        self._stream.__enter__()

    def __exit__(self, *exc):
        self._stream.__exit__(*exc)
        self._device.__exit__(*exc)


def _here(t) -> int:
    """The current stream of the tensor's device."""
    import torch
    return torch._C._cuda_getCurrentRawStream(t.get_device())


class PagedCache:
    """Keys and values in pages (``phyai_paged_cache``): pools ``k`` and ``v`` of
    [n_pages][page_size][n_kv_heads][head_dim], or with the layers in front, in any
    order of the strides before the last dimension; ``page_table`` int32
    [batch][max_pages].  float32, bfloat16 (or int16 bit patterns) or
    float8_e4m3fn (or uint8 codes) with float32 ``k_scale`` and ``v_scale`` [n_kv_heads].

    The tensors stay the caller's; the table may be rewritten between calls."""

    def __init__(self, k, v, page_table, k_scale=None, v_scale=None):
        import torch
        if k.dim() not in (4, 5) or not k.is_cuda:
            raise ValueError("expected device pools [layers][n_pages][page_size][n_kv_heads][head_dim]")
        if k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.device != v.device:
            raise ValueError("k and v must have the same shape, strides, dtype and device")
        if k.stride(-1) != 1:
            raise ValueError("a head's values must be contiguous")
        if page_table.dtype != torch.int32 or page_table.dim() != 2 or page_table.device != k.device:
            raise ValueError(f"page_table: expected an int32 tensor [batch][max_pages] on {k.device}")
        if page_table.shape[1] > 1 and page_table.stride(1) != 1:
            raise ValueError("page_table: a request's entries must be contiguous")
        dtype, n, s = _dtype_of(k), k.shape[-4:], k.stride()[-4:]
        if (dtype == 2) != (k_scale is not None) or (dtype == 2) != (v_scale is not None):
            raise ValueError("an 8-bit cache has k_scale and v_scale, another has none")
        _in_32_bits(*k.shape, *page_table.shape, page_table.stride(0))
        self.k, self.v, self.page_table, self.k_scale, self.v_scale = k, v, page_table, k_scale, v_scale
        self.n_layers = k.shape[0] if k.dim() == 5 else 1
        self.batch, self.page_size, self.n_kv_heads, self.head_dim = page_table.shape[0], n[1], n[2], n[3]
        width = page_table.shape[1]
        self._c = _PagedCache(
            k.data_ptr(), v.data_ptr(), _vector(k_scale, torch.float32, n[2], k, "k_scale"),
            _vector(v_scale, torch.float32, n[2], k, "v_scale"),
            page_table.data_ptr(), k.stride(0) if self.n_layers > 1 else 0, s[0] if n[0] > 1 else 0, s[1],
            s[2] if n[2] > 1 else 0, dtype, self.n_layers, n[2], n[3], n[1], n[0], self.batch, width,
            page_table.stride(0) if self.batch > 1 else width)
        self._ref = ctypes.byref(self._c)

    @property
    def capacity(self) -> int:
        """Tokens that a request's table has room for."""
        return self.page_table.shape[1] * self.page_size


def qk_norm_rope(q, k=None, q_gain=None, k_gain=None, *, eps: float = 1e-6, rope_base: float = 10000.0,
                 past_len=None, new_len=None, q_out=None, k_out=None, status=None, stream=None):
    """Norms of queries and keys for each head and their rotation in one pass
    (``phyai_qk_norm_rope``).  q, k: [batch][rows][heads][head_dim]; q_gain, k_gain:
    float32 [head_dim]; past_len, new_len: device int32 [batch].  eps = 0 only
    rotates, rope_base = 0 only normalises.  Returns (q_out, k_out), new tensors
    where none are given (their rows behind new_len are not written)."""
    import torch
    if _elsewhere(q, stream):
        with _there(q, stream):
            return qk_norm_rope(q, k, q_gain, k_gain, eps=eps, rope_base=rope_base, past_len=past_len, new_len=new_len,
                                q_out=q_out, k_out=k_out, status=status)
    qs = _head_rows(q, "q")
    B, M, _, D = q.shape
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    elif q_out.shape != q.shape:
        raise ValueError("q_out: another shape than q")
    qo = _head_rows(q_out, "q_out", q)
    ks = ko = None
    if k is not None:
        k_struct = _head_rows(k, "k", q)
        if k_out is None:
            k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        elif k_out.shape != k.shape:
            raise ValueError("k_out: another shape than k")
        ko_struct = _head_rows(k_out, "k_out", q)
        ks, ko = ctypes.byref(k_struct), ctypes.byref(ko_struct)
    elif k_out is not None:
        raise ValueError("k_out without k")
    for g, what in ((q_gain, "q_gain"), (k_gain, "k_gain")):
        if g is not None and g.shape != (D,):
            raise ValueError(f"{what}: expected [head_dim]")
    if B * M > 0:
        rc = lib().phyai_qk_norm_rope(
            ctypes.byref(qs), ks, ctypes.byref(qo), ko, _vector(q_gain, torch.float32, D, q, "q_gain"),
            _vector(k_gain, torch.float32, D, q, "k_gain"), eps, rope_base,
            _vector(past_len, torch.int32, B, q, "past_len"), _vector(new_len, torch.int32, B, q, "new_len"), B, M, D,
            _dtype_of(q), _vector(status, torch.int32, 1, q, "status"), _here(q))
        if rc:
            _check(rc)
    return q_out, k_out


def paged_append(cache: PagedCache, k, v, past_len, *, new_len=None, rope_base: float = 0.0, layer: int = 0,
                 status=None, stream=None) -> None:
    """Append keys and values [batch][rows][n_kv_heads][head_dim] of new tokens to the
    cache at tokens past_len[b] .. past_len[b] + new_len[b] - 1, the keys rotated to
    those positions where rope_base is not 0 (``phyai_paged_append``)."""
    import torch
    if _elsewhere(k, stream):
        with _there(k, stream):
            return paged_append(cache, k, v, past_len, new_len=new_len, rope_base=rope_base, layer=layer, status=status)
    ks, vs = _head_rows(k, "k"), _head_rows(v, "v", k)
    B, M, _, D = k.shape
    if B != cache.batch or D != cache.head_dim or k.device != cache.k.device:
        raise ValueError("k: batch, head_dim and device must be the cache's")
    if layer >> 31:
        _in_32_bits(layer)
    if B * M == 0:
        return
    rc = lib().phyai_paged_append(cache._ref, layer, ctypes.byref(ks), ctypes.byref(vs), rope_base,
                                  _vector(past_len, torch.int32, B, k, "past_len"),
                                  _vector(new_len, torch.int32, B, k, "new_len"), M, _dtype_of(k),
                                  _vector(status, torch.int32, 1, k, "status"), _here(k))
    if rc:
        _check(rc)


def paged_attention_workspace(cache: PagedCache, n_q_heads: int, rows: int, max_kv_len: Optional[int] = None) -> int:
    """Bytes of workspace that such a ``paged_attention`` call needs."""
    if max_kv_len is None:
        max_kv_len = cache.capacity
    if (n_q_heads | rows | max_kv_len) >> 31:
        _in_32_bits(n_q_heads, rows, max_kv_len)
    n = lib().phyai_paged_attention_workspace(cache._ref, n_q_heads, rows, max_kv_len)
    if n < 0:
        _check(int(n))
    return n


def paged_attention(q, cache: PagedCache, kv_len, *, new_len=None, max_kv_len: Optional[int] = None,
                    scale: Optional[float] = None, causal: bool = True, window: int = 0, layer: int = 0, out=None,
                    workspace=None, status=None, stream=None):
    """Attention of the last new_len[b] of a request's kv_len[b] cached tokens over all
    of them (``phyai_paged_attention``).  q: [batch][rows][heads][head_dim]; kv_len,
    new_len: device int32 [batch]; max_kv_len: the longest kv_len (default: what
    the table has room for); scale: default 1 / sqrt(head_dim).  workspace: a
    device tensor of at least ``paged_attention_workspace`` bytes (default: one is
    allocated for the call).  Returns out (rows behind new_len are not written)."""
    import torch
    if _elsewhere(q, stream):
        with _there(q, stream):
            return paged_attention(q, cache, kv_len, new_len=new_len, max_kv_len=max_kv_len, scale=scale, causal=causal,
                                   window=window, layer=layer, out=out, workspace=workspace, status=status)
    qs = _head_rows(q, "q")
    B, M, H, D = q.shape
    if B != cache.batch or D != cache.head_dim or q.device != cache.k.device:
        raise ValueError("q: batch, head_dim and device must be the cache's")
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    elif out.shape != q.shape:
        raise ValueError("out: another shape than q")
    os_ = _head_rows(out, "out", q)
    if B * M == 0:
        return out
    if max_kv_len is None:
        max_kv_len = cache.capacity
    if (layer | window | max_kv_len) >> 31:
        _in_32_bits(layer, window, max_kv_len)
    if workspace is None:
        size = paged_attention_workspace(cache, H, M, max_kv_len)
        if size:
            workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
    else:
        size = _bytes_of(workspace, q)
    rc = lib().phyai_paged_attention(
        cache._ref, layer, ctypes.byref(qs), ctypes.byref(os_), _vector(kv_len, torch.int32, B, q, "kv_len"),
        _vector(new_len, torch.int32, B, q, "new_len"), max_kv_len, D ** -0.5 if scale is None else scale, causal,
        window, M, _dtype_of(q), None if workspace is None else workspace.data_ptr(), size,
        _vector(status, torch.int32, 1, q, "status"), _here(q))
    if rc:
        _check(rc)
    return out


def paged_gather(cache: PagedCache, kv_len, rows: int, *, out=None, status=None, stream=None):
    """The first kv_len[b] tokens of every request and layer as the contiguous prefix
    [layers][2][batch][rows][n_kv_heads * head_dim] that ``Expert.denoise`` reads
    (``phyai_paged_gather``): float32 or bfloat16, zeros behind kv_len[b]."""
    import torch
    k = cache.k
    if _elsewhere(k, stream):
        with _there(k, stream):
            return paged_gather(cache, kv_len, rows, out=out, status=status)
    _in_32_bits(rows)
    dt = torch.float32 if k.dtype == torch.float32 else torch.bfloat16
    shape = (cache.n_layers, 2, cache.batch, rows, cache.n_kv_heads * cache.head_dim)
    if out is None:
        out = torch.empty(shape, dtype=dt, device=k.device)
    elif out.shape != shape or (out.dtype != dt and (dt == torch.float32 or out.dtype != torch.int16)) or \
            not out.is_contiguous() or out.device != k.device:
        raise ValueError(f"out: expected a contiguous {dt} tensor {shape} on {k.device}")
    if cache.batch * rows > 0:
        rc = lib().phyai_paged_gather(cache._ref, _vector(kv_len, torch.int32, cache.batch, k, "kv_len"),
                                      out.data_ptr(), rows, _vector(status, torch.int32, 1, k, "status"), _here(k))
        if rc:
            _check(rc)
    return out


def fp8_to_bf16(codes, stream=None):
    """Decode device uint8 e4m3fn codes to bf16 bit patterns (device int16)."""
    import torch
    out = torch.empty(codes.shape, dtype=torch.int16, device=codes.device)
    _check(lib().phyai_fp8_to_bf16(_ptr(codes), _ptr(out), codes.numel(), _stream(stream)))
    return out


def version() -> int:
    return lib().phyai_version()
