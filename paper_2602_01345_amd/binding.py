"""ctypes binding of libnova.so: argument marshalling only.

Every step of the hot path runs in the HIP kernels behind the C ABI declared in
``include/nova.h``.  PyTorch is used for device memory (tensors) and the current
stream; nothing here computes.  The method names mirror the C entry points.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass, field
from typing import Dict, Optional, Sequence, Tuple, Union

import torch

NOVA_F32, NOVA_BF16 = 0, 1
NOVA_INTERP_BILINEAR, NOVA_INTERP_NEAREST, NOVA_INTERP_BICUBIC = 0, 1, 2
STAGES = ("entropy", "select", "gather_ln", "qkv", "attention", "oproj", "ln2", "ffn1", "ffn2", "merge")
_HERE = os.path.dirname(os.path.abspath(__file__))


class NovaError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what} failed: {code}")
        self.code = code


class _Shape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("dtype", "B", "N", "C", "heads", "ffn_mult", "kv_len", "kv_capacity", "k")]


class _Weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in
                ("w_qkv", "b_qkv", "w_o", "b_o", "w_fc1", "b_fc1", "w_fc2", "b_fc2")]


class _Variant(C.Structure):
    _fields_ = [("gelu_tanh", C.c_int32), ("qk_norm", C.c_int32), ("qk_scale", C.c_void_p), ("ada", C.c_void_p),
                ("w_cq", C.c_void_p), ("b_cq", C.c_void_p), ("w_co", C.c_void_p), ("b_co", C.c_void_p),
                ("k_text", C.c_void_p), ("v_text", C.c_void_p), ("text_len", C.c_int32), ("text_capacity", C.c_int32)]


class _FourBitCache(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("k_codes", "k_scales", "v_codes", "v_scales")] +
                [(n, C.c_int32) for n in ("B", "kv_heads", "capacity", "dh")])


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p)] + [(n, C.c_int64) for n in ("stride_b", "stride_row", "stride_head", "stride_channel")]


@dataclass(frozen=True, eq=False)
class FourBitCache:
    """nova_fourbit_cache: keys and values of B images in 4 bits, uint8 device tensors: codes [B, kv_heads, capacity, dh / 2]
    and scales [B, kv_heads, capacity, dh / 32] of either."""
    k_codes: torch.Tensor
    k_scales: torch.Tensor
    v_codes: torch.Tensor
    v_scales: torch.Tensor
    _c: Optional["_FourBitCache"] = field(default=None, init=False, repr=False)

    @classmethod
    def empty(cls, B: int, kv_heads: int, capacity: int, dh: int, device: Union[str, int, torch.device] = "cuda") -> "FourBitCache":
        """A cache without rows (every value in it reads as zero)."""
        def half():
            return (torch.zeros((B, kv_heads, capacity, dh // 2), dtype=torch.uint8, device=device),
                    torch.full((B, kv_heads, capacity, dh // 32), 127, dtype=torch.uint8, device=device))
        return cls(*half(), *half())

    @property
    def capacity(self) -> int:
        return self.k_codes.shape[2]

    @property
    def dh(self) -> int:
        return self.k_codes.shape[3] * 2

    def c_struct(self) -> "_FourBitCache":
        """The C structure: made and checked on the first call, and again only if a tensor has got other memory since."""
        ts = (self.k_codes, self.k_scales, self.v_codes, self.v_scales)
        ptrs = (ts[0].data_ptr(), ts[1].data_ptr(), ts[2].data_ptr(), ts[3].data_ptr())
        c = self._c
        if c is not None and c.made_of == ptrs:
            return c
        codes, scales = ts[0].shape, ts[1].shape
        if ts[2].shape != codes or ts[3].shape != scales or codes[:3] != scales[:3] or codes[3] != 16 * scales[3]:
            raise ValueError(f"no cache in 4 bits: codes {tuple(codes)}, {tuple(ts[2].shape)}, scales {tuple(scales)}, "
                             f"{tuple(ts[3].shape)}")
        assert all(t.dtype == torch.uint8 for t in ts), "codes and scales are uint8"
        c = _FourBitCache(*[_ptr(t) for t in ts], *codes[:3], codes[3] * 2)
        c.made_of, c.device = ptrs, ts[0].get_device()
        if any(t.get_device() != c.device for t in ts):
            raise ValueError("the arrays of a cache lie on one device")
        object.__setattr__(self, "_c", c)
        return c


@dataclass
class BlockVariant:
    """nova_block_variant: tanh GELU, unit-length q/k with a per-head multiplier (fp32 [heads], device),
    per-image modulation and gates ([B, 6, C] in the activations' dtype, device)."""
    gelu_tanh: bool = False
    qk_scale: Optional[torch.Tensor] = None
    ada: Optional[torch.Tensor] = None
    # cross-attention sub-layer: "w_cq", "b_cq", "w_co", "b_co" and the condition tokens' projected keys /
    # values "k_text" [B, heads, capacity, dh], "v_text" [B, heads, dh, capacity] (pack_k_cache / pack_v_cache),
    # "text_len" (int)
    cross: Optional[Dict[str, object]] = None

    def c_struct(self) -> "_Variant":
        if self.qk_scale is not None:
            assert self.qk_scale.dtype == torch.float32
        v = _Variant(int(self.gelu_tanh), int(self.qk_scale is not None), _ptr(self.qk_scale), _ptr(self.ada))
        if self.cross is not None:
            c = self.cross
            v.w_cq, v.b_cq, v.w_co, v.b_co = (_ptr(c.get(n)) for n in ("w_cq", "b_cq", "w_co", "b_co"))
            v.k_text, v.v_text = _ptr(c["k_text"]), _ptr(c["v_text"])
            v.text_len, v.text_capacity = int(c["text_len"]), int(c["k_text"].shape[2])
        return v


@dataclass
class BlockShape:
    dtype: int
    B: int
    N: int
    C: int
    heads: int
    kv_len: int
    kv_capacity: int
    k: int
    ffn_mult: int = 4

    def c_struct(self) -> _Shape:
        return _Shape(self.dtype, self.B, self.N, self.C, self.heads, self.ffn_mult, self.kv_len,
                      self.kv_capacity, self.k)


def library_path() -> str:
    return os.path.join(_HERE, "libnova.so")


_LIB = None


def load_library() -> C.CDLL:
    """Loads libnova.so from the package directory; raises if it has not been built."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2602_01345_amd.build` "
                           "(there is no fallback path)")
    lib = C.CDLL(path)
    vp, i32, i64 = C.c_void_p, C.c_int, C.c_int64
    lib.nova_create.argtypes = [C.POINTER(vp), i32]
    lib.nova_destroy.argtypes = [vp]
    lib.nova_strerror.argtypes = [i32]
    lib.nova_strerror.restype = C.c_char_p
    lib.nova_workspace_bytes.argtypes = [C.POINTER(_Shape)]
    lib.nova_workspace_bytes.restype = C.c_size_t
    lib.nova_entropy.argtypes = [vp, vp, vp, i32, i64, i32, i32, i64, vp, vp]
    lib.nova_select.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp]
    lib.nova_entropy_blocks.argtypes = [vp, vp, i32, vp, i32, i64, i32, i32, i64, vp, vp]
    lib.nova_entropy_blocks.restype = i32
    lib.nova_select_blocks.argtypes = [vp, vp, i32, vp, i32, i32, vp, vp, vp]
    lib.nova_select_blocks.restype = i32
    lib.nova_entropy_bits.argtypes = [vp, vp, vp, i32, i64, i32, i32, vp, vp]
    lib.nova_entropy_bits.restype = i32
    lib.nova_head_entropy_workspace_bytes.argtypes = [i64, i32, i32]
    lib.nova_head_entropy_workspace_bytes.restype = C.c_size_t
    lib.nova_head_entropy.argtypes = [vp, vp, vp, vp, vp, i32, i64, i32, i32, i32, vp, vp, vp, C.c_size_t]
    lib.nova_head_entropy.restype = i32
    lib.nova_head_entropy_static.argtypes = [vp, vp, vp, vp, vp, i32, i64, i32, i32, i32, vp, vp]
    lib.nova_head_entropy_static.restype = i32
    lib.nova_pruned_block.argtypes = [vp, vp, C.POINTER(_Shape), C.POINTER(_Weights), vp, vp, vp, vp, vp, vp,
                                      C.c_size_t]
    lib.nova_pruned_block_variant.argtypes = [vp, vp, C.POINTER(_Shape), C.POINTER(_Weights), C.POINTER(_Variant),
                                              vp, vp, vp, vp, vp, vp, C.c_size_t]
    lib.nova_pruned_block_variant.restype = i32
    lib.nova_pruned_block_rows.argtypes = [vp, vp, C.POINTER(_Shape), C.POINTER(_Weights), C.POINTER(_Variant),
                                           vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t]
    lib.nova_pruned_block_rows.restype = i32
    lib.nova_merge_cache_rows.argtypes = [vp, vp, i32, i32] + [i32] * 7 + [vp] * 8
    lib.nova_merge_cache_rows.restype = i32
    lib.nova_merge_cache.argtypes = [vp, vp, i32] + [i32] * 7 + [vp] * 7
    lib.nova_merge_cache_interp.argtypes = [vp, vp, i32, i32] + [i32] * 7 + [vp] * 7
    lib.nova_merge_cache_interp.restype = i32
    lib.nova_profile_stages.argtypes = [vp, C.c_uint32]
    lib.nova_profile_collect.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    lib.nova_activation_scale.argtypes = [C.POINTER(C.c_double), i32, i32, C.c_double, C.POINTER(i32)]
    lib.nova_scale_ratio.argtypes = [i32, i32, C.c_double, C.c_double, C.c_double, C.POINTER(C.c_double)]
    lib.nova_layer_ratio.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp, vp]
    cache, rows, sz = C.POINTER(_FourBitCache), C.POINTER(_Rows), C.c_size_t
    lib.nova_fourbit_append.argtypes = [vp, vp, i32, cache, i32, rows, rows, vp, i32, vp, vp]
    lib.nova_fourbit_unpack.argtypes = [vp, vp, i32, cache, i32, i32, vp, vp, rows, rows]
    lib.nova_fourbit_attention.argtypes = [vp, vp, i32, cache, i32, i32, rows, vp, i32, vp, C.c_float, vp, vp, vp, sz]
    lib.nova_fourbit_mass.argtypes = [vp, vp, i32, cache, i32, i32, rows, vp, i32, vp, C.c_float, vp, vp, vp, vp, sz]
    lib.nova_fourbit_evict.argtypes = [vp, vp, cache, cache, i32, vp, vp, i32, vp, vp, vp, vp]
    lib.nova_fourbit_block_workspace_bytes.argtypes, lib.nova_fourbit_block_workspace_bytes.restype = [C.POINTER(_Shape)], sz
    lib.nova_pruned_block_fourbit.argtypes = [vp, vp, C.POINTER(_Shape), C.POINTER(_Weights), C.POINTER(_Variant), vp, vp, vp, vp,
                                              vp, cache, vp, vp, vp, vp, sz]
    for f in (lib.nova_fourbit_append, lib.nova_fourbit_unpack, lib.nova_fourbit_attention, lib.nova_fourbit_mass,
              lib.nova_fourbit_evict, lib.nova_pruned_block_fourbit):
        f.restype = i32
    for f in (lib.nova_fourbit_attention_workspace_bytes, lib.nova_fourbit_mass_workspace_bytes):
        f.argtypes, f.restype = [cache, i32, i32, i32], sz
    lib.nova_probe.argtypes = [vp, vp, i32, vp, vp, i64, i32, vp, C.POINTER(C.c_double)]
    lib.nova_probe.restype = i32
    lib.nova_profile_stages.restype = i32
    lib.nova_profile_collect.restype = i32
    for f in (lib.nova_create, lib.nova_destroy, lib.nova_entropy, lib.nova_select, lib.nova_pruned_block,
              lib.nova_merge_cache, lib.nova_activation_scale, lib.nova_scale_ratio, lib.nova_layer_ratio):
        f.restype = i32
    _LIB = lib
    return lib


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return NOVA_F32
    if t.dtype == torch.bfloat16:
        return NOVA_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensors only"
    return t.data_ptr()


def _ptrs(ts: Sequence[torch.Tensor]) -> "C.Array":
    return (C.c_void_p * len(ts))(*[_ptr(t) for t in ts])


def _rows(t: torch.Tensor, heads: int, dh: int, name: str) -> "_Rows":
    """nova_rows of a [B, n, heads, dh] tensor of any strides."""
    shape = t.shape
    if len(shape) != 4 or shape[2] != heads or shape[3] != dh:
        raise ValueError(f"{name}: {tuple(shape)}, expected [B, n, {heads}, {dh}]")
    return _Rows(t.data_ptr(), *t.stride())


def _shaped(name: str, t: Optional[torch.Tensor], shape: Tuple[int, ...], dtype: torch.dtype,
            device: Optional[int] = None) -> Optional[int]:
    """Pointer of an optional dense tensor that has to have this shape and type, and lie on this device where one is given."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or (device is not None and t.get_device() != device):
        raise ValueError(f"{name}: {tuple(t.shape)} {t.dtype} {t.stride()} on {t.device}, expected dense {tuple(shape)} {dtype}"
                         + ("" if device is None else f" on device {device}"))
    return t.data_ptr()


def _check_lengths(n: int, **lists):
    """Host arrays the library reads n entries of."""
    for name, ts in lists.items():
        if ts is not None and len(ts) < n:
            raise ValueError(f"{name}: {len(ts)} entries for {n} blocks")


# The current stream's handle without a Stream object around it (0.3 against 2.7 us): with small kernels the calls below
# are what a step waits for.  Not part of torch's public interface, so a torch without it takes the public way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device: Optional[int] = None) -> int:
    """Handle of the current stream, of the current device or of a given one."""
    if _raw_stream is None:
        return (torch.cuda.current_stream() if device is None else torch.cuda.current_stream(device)).cuda_stream
    return _raw_stream(torch.cuda.current_device() if device is None else device)


def activation_scale(hbar: Sequence[float], t_est: int, alpha: float) -> int:
    """nova_activation_scale: t* (1-based) for the scale mean entropies seen so far, 0 if none (host only)."""
    lib = load_library()
    arr = (C.c_double * max(len(hbar), 1))(*[float(h) for h in hbar])
    out = C.c_int(0)
    rc = lib.nova_activation_scale(arr, len(hbar), int(t_est), float(alpha), C.byref(out))
    if rc != 0:
        raise NovaError(rc, "nova_activation_scale")
    return out.value


def scale_ratio(t: int, t_star: int, g_t: float, tau: float, lam: float) -> float:
    """nova_scale_ratio: the scale-linkage reduction ratio (host only)."""
    lib = load_library()
    out = C.c_double(0.0)
    rc = lib.nova_scale_ratio(int(t), int(t_star), float(g_t), float(tau), float(lam), C.byref(out))
    if rc != 0:
        raise NovaError(rc, "nova_scale_ratio")
    return out.value


class Nova:
    """Handle on one GPU's context; methods are the four C entry points."""

    def __init__(self, device: int = 0):
        self.lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the NOVA hot path has no CPU fallback")
        h = C.c_void_p()
        rc = self.lib.nova_create(C.byref(h), device)
        if rc != 0:
            raise NovaError(rc, "nova_create")
        self.ctx = h
        self.device = device

    def __del__(self):
        ctx = getattr(self, "ctx", None)
        if ctx:
            self.lib.nova_destroy(ctx)
            self.ctx = None

    def strerror(self, code: int) -> str:
        return self.lib.nova_strerror(code).decode()

    def _check(self, rc: int, what: str):
        if rc != 0:
            raise NovaError(rc, f"{what} ({self.strerror(rc)})")

    # -- instrumentation ------------------------------------------------------------
    def profile_stages(self, stages):
        mask = 0
        for st in stages:
            mask |= 1 << int(st)
        self._check(self.lib.nova_profile_stages(self.ctx, mask), "nova_profile_stages")

    def profile_collect(self, stage: int):
        ms, n = C.c_double(0.0), C.c_int64(0)
        self._check(self.lib.nova_profile_collect(self.ctx, int(stage), C.byref(ms), C.byref(n)),
                    "nova_profile_collect")
        return ms.value, n.value

    def probe(self, kind: int, src: Optional[torch.Tensor], dst: Optional[torch.Tensor], iters: int,
              sink: torch.Tensor) -> float:
        """nova_probe: launches one achievable-peak kernel; returns the bytes moved / flops done."""
        work = C.c_double(0.0)
        nbytes = 0 if src is None else src.numel() * src.element_size()
        rc = self.lib.nova_probe(self.ctx, _stream(), int(kind), _ptr(src), _ptr(dst), nbytes, int(iters),
                                 _ptr(sink), C.byref(work))
        self._check(rc, "nova_probe")
        return work.value

    # -- nova_layer_ratio -----------------------------------------------------------
    def layer_ratio(self, mean_entropy: torch.Tensor, entropy_sum: torch.Tensor, ratio_t: torch.Tensor, j: int,
                    N: int, ratio_tj: torch.Tensor, k_per_row: torch.Tensor):
        """Per-row layer-linkage ratio and keep counts of layer j (1-based); entropy_sum is updated in place."""
        B = mean_entropy.shape[0]
        assert k_per_row.dtype == torch.int32 and all(t.dtype == torch.float32 for t in
                                                      (mean_entropy, entropy_sum, ratio_t, ratio_tj))
        rc = self.lib.nova_layer_ratio(self.ctx, _stream(), _ptr(mean_entropy), _ptr(entropy_sum), _ptr(ratio_t),
                                       int(j), B, int(N), _ptr(ratio_tj), _ptr(k_per_row))
        self._check(rc, "nova_layer_ratio")

    # -- nova_entropy ---------------------------------------------------------------
    def entropy(self, logits: torch.Tensor, entropy: torch.Tensor, mean: Optional[torch.Tensor] = None):
        """logits [B, N, V] (f32|bf16) -> entropy [B, N] f32 (and mean [B] f32)."""
        B, N, V = logits.shape
        rc = self.lib.nova_entropy(self.ctx, _stream(), _ptr(logits), _dtype_code(logits), N, B, V,
                                   logits.stride(1), _ptr(entropy), _ptr(mean))
        self._check(rc, "nova_entropy")

    # -- nova_entropy_blocks --------------------------------------------------------
    def entropy_blocks(self, logits: Sequence[torch.Tensor], entropy: Sequence[torch.Tensor],
                       mean: Optional[Sequence[torch.Tensor]] = None):
        """entropy() of every tensor of a list; tensors of one shape, stride and dtype share launches (32 neighbours of
        one alignment each), a list that mixes them takes one call per tensor."""
        _check_lengths(len(logits), entropy=entropy, mean=mean)
        if len(logits) == 0:
            return
        a = logits[0]
        if any(t.shape != a.shape or t.stride(1) != a.stride(1) or t.dtype != a.dtype for t in logits):
            for i, t in enumerate(logits):
                self.entropy(t, entropy[i], None if mean is None else mean[i])
            return
        B, N, V = a.shape
        rc = self.lib.nova_entropy_blocks(self.ctx, _stream(), len(logits), _ptrs(logits), _dtype_code(a), N, B, V,
                                          a.stride(1), _ptrs(entropy), None if mean is None else _ptrs(mean))
        self._check(rc, "nova_entropy_blocks")

    # -- nova_entropy_bits ----------------------------------------------------------
    def entropy_bits(self, bit_logits: torch.Tensor, entropy: torch.Tensor, mean: Optional[torch.Tensor] = None):
        """bit_logits [B, N, d, 2] (f32|bf16) -> entropy [B, N] f32 (and mean [B] f32)."""
        B, N, d, two = bit_logits.shape
        assert two == 2
        rc = self.lib.nova_entropy_bits(self.ctx, _stream(), _ptr(bit_logits), _dtype_code(bit_logits), N, B, d,
                                        _ptr(entropy), _ptr(mean))
        self._check(rc, "nova_entropy_bits")

    # -- nova_head_entropy ----------------------------------------------------------
    def head_entropy_workspace_bytes(self, rows_per_batch: int, batch: int, V: int) -> int:
        return int(self.lib.nova_head_entropy_workspace_bytes(rows_per_batch, batch, V))

    def head_entropy(self, hidden: torch.Tensor, w_head: torch.Tensor, b_head: Optional[torch.Tensor],
                     entropy: torch.Tensor, workspace: torch.Tensor, mean: Optional[torch.Tensor] = None):
        """hidden [B, N, C] bf16, w_head [V, C], b_head [V] or None -> entropy [B, N] f32 (and mean [B])."""
        B, N, Cc = hidden.shape
        V = w_head.shape[0]
        rc = self.lib.nova_head_entropy(self.ctx, _stream(), _ptr(hidden), _ptr(w_head), _ptr(b_head),
                                        _dtype_code(hidden), N, B, Cc, V, _ptr(entropy), _ptr(mean),
                                        _ptr(workspace), workspace.numel() * workspace.element_size())
        self._check(rc, "nova_head_entropy")

    def head_entropy_static(self, hidden: torch.Tensor, w_head: torch.Tensor, b_head: Optional[torch.Tensor],
                            entropy: torch.Tensor, mean: Optional[torch.Tensor] = None):
        """nova_head_entropy_static: as head_entropy, the partials in the library's static device scratch."""
        B, N, Cc = hidden.shape
        V = w_head.shape[0]
        rc = self.lib.nova_head_entropy_static(self.ctx, _stream(), _ptr(hidden), _ptr(w_head), _ptr(b_head),
                                               _dtype_code(hidden), N, B, Cc, V, _ptr(entropy), _ptr(mean))
        self._check(rc, "nova_head_entropy_static")

    # -- nova_select ----------------------------------------------------------------
    def select(self, entropy: torch.Tensor, k: int, kept_idx: torch.Tensor, keep_mask: torch.Tensor,
               k_per_row: Optional[torch.Tensor] = None):
        B, N = entropy.shape
        rc = self.lib.nova_select(self.ctx, _stream(), _ptr(entropy), B, N, k, _ptr(k_per_row),
                                  _ptr(kept_idx), _ptr(keep_mask))
        self._check(rc, "nova_select")

    # -- nova_select_blocks ---------------------------------------------------------
    def select_blocks(self, entropy: Sequence[torch.Tensor], k: Sequence[int], kept_idx: Sequence[torch.Tensor],
                      keep_mask: Sequence[torch.Tensor]):
        """select() of every tensor of a list of [B, N] entropies, each with its own k, 32 of them per launch."""
        _check_lengths(len(entropy), k=k, kept_idx=kept_idx, keep_mask=keep_mask)
        if len(entropy) == 0:
            return
        B, N = entropy[0].shape
        assert all(t.shape == (B, N) for t in entropy)
        rc = self.lib.nova_select_blocks(self.ctx, _stream(), len(entropy), _ptrs(entropy), B, N,
                                         (C.c_int32 * len(k))(*[int(v) for v in k]), _ptrs(kept_idx), _ptrs(keep_mask))
        self._check(rc, "nova_select_blocks")

    # -- nova_pruned_block ----------------------------------------------------------
    def workspace_bytes(self, shape: BlockShape) -> int:
        s = shape.c_struct()
        return int(self.lib.nova_workspace_bytes(C.byref(s)))

    def pruned_block(self, shape: BlockShape, weights: Dict[str, Optional[torch.Tensor]], x: torch.Tensor,
                     kept_idx: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     y_kept: torch.Tensor, workspace: torch.Tensor):
        s = shape.c_struct()
        w = _Weights(*[_ptr(weights.get(n)) for n, _ in _Weights._fields_])
        rc = self.lib.nova_pruned_block(self.ctx, _stream(), C.byref(s), C.byref(w), _ptr(x), _ptr(kept_idx),
                                        _ptr(k_cache), _ptr(v_cache), _ptr(y_kept), _ptr(workspace),
                                        workspace.numel() * workspace.element_size())
        self._check(rc, "nova_pruned_block")

    def pruned_block_variant(self, shape: BlockShape, weights: Dict[str, Optional[torch.Tensor]],
                             variant: Optional[BlockVariant], x: torch.Tensor, kept_idx: torch.Tensor,
                             k_cache: torch.Tensor, v_cache: torch.Tensor, y_kept: torch.Tensor,
                             workspace: torch.Tensor):
        s = shape.c_struct()
        w = _Weights(*[_ptr(weights.get(n)) for n, _ in _Weights._fields_])
        v = variant.c_struct() if variant is not None else None
        rc = self.lib.nova_pruned_block_variant(self.ctx, _stream(), C.byref(s), C.byref(w),
                                                C.byref(v) if v is not None else None, _ptr(x), _ptr(kept_idx),
                                                _ptr(k_cache), _ptr(v_cache), _ptr(y_kept), _ptr(workspace),
                                                workspace.numel() * workspace.element_size())
        self._check(rc, "nova_pruned_block_variant")

    def pruned_block_rows(self, shape: BlockShape, weights: Dict[str, Optional[torch.Tensor]],
                          variant: Optional[BlockVariant], k_per_row: Optional[torch.Tensor],
                          kv_len_per_row: Optional[torch.Tensor], kv_len_next: Optional[torch.Tensor],
                          x: torch.Tensor, kept_idx: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                          y_kept: torch.Tensor, workspace: torch.Tensor):
        """nova_pruned_block_rows: per-image keep counts / cache lengths as int32 device tensors [B]."""
        for t in (k_per_row, kv_len_per_row, kv_len_next):
            assert t is None or t.dtype == torch.int32
        s = shape.c_struct()
        w = _Weights(*[_ptr(weights.get(n)) for n, _ in _Weights._fields_])
        v = variant.c_struct() if variant is not None else None
        rc = self.lib.nova_pruned_block_rows(self.ctx, _stream(), C.byref(s), C.byref(w),
                                             C.byref(v) if v is not None else None, _ptr(k_per_row),
                                             _ptr(kv_len_per_row), _ptr(kv_len_next), _ptr(x), _ptr(kept_idx),
                                             _ptr(k_cache), _ptr(v_cache), _ptr(y_kept), _ptr(workspace),
                                             workspace.numel() * workspace.element_size())
        self._check(rc, "nova_pruned_block_rows")

    def merge_cache_rows(self, interp: int, h: int, w: int, hp: int, wp: int, k: int,
                         k_per_row: Optional[torch.Tensor], x: torch.Tensor, y_kept: Optional[torch.Tensor],
                         kept_idx: Optional[torch.Tensor], keep_mask: torch.Tensor,
                         cache_prev: Optional[torch.Tensor], out: torch.Tensor,
                         cache_new: Optional[torch.Tensor] = None):
        """nova_merge_cache_rows: k is the row pitch, k_per_row the per-image counts (int32 device [B])."""
        assert k_per_row is None or k_per_row.dtype == torch.int32
        B, _, Cc = x.shape
        rc = self.lib.nova_merge_cache_rows(self.ctx, _stream(), _dtype_code(x), interp, B, Cc, h, w, hp, wp, k,
                                            _ptr(k_per_row), _ptr(x), _ptr(y_kept), _ptr(kept_idx), _ptr(keep_mask),
                                            _ptr(cache_prev), _ptr(out), _ptr(cache_new))
        self._check(rc, "nova_merge_cache_rows")

    # -- nova_merge_cache -----------------------------------------------------------
    def merge_cache(self, h: int, w: int, hp: int, wp: int, k: int, x: torch.Tensor,
                    y_kept: Optional[torch.Tensor], kept_idx: Optional[torch.Tensor], keep_mask: torch.Tensor,
                    cache_prev: Optional[torch.Tensor], out: torch.Tensor,
                    cache_new: Optional[torch.Tensor] = None):
        B, _, Cc = x.shape
        rc = self.lib.nova_merge_cache(self.ctx, _stream(), _dtype_code(x), B, Cc, h, w, hp, wp, k, _ptr(x),
                                       _ptr(y_kept), _ptr(kept_idx), _ptr(keep_mask), _ptr(cache_prev),
                                       _ptr(out), _ptr(cache_new))
        self._check(rc, "nova_merge_cache")

    def merge_cache_interp(self, interp: int, h: int, w: int, hp: int, wp: int, k: int, x: torch.Tensor,
                           y_kept: Optional[torch.Tensor], kept_idx: Optional[torch.Tensor],
                           keep_mask: torch.Tensor, cache_prev: Optional[torch.Tensor], out: torch.Tensor,
                           cache_new: Optional[torch.Tensor] = None):
        """interp: NOVA_INTERP_BILINEAR (0), NOVA_INTERP_NEAREST (1), NOVA_INTERP_BICUBIC (2)."""
        B, _, Cc = x.shape
        rc = self.lib.nova_merge_cache_interp(self.ctx, _stream(), _dtype_code(x), interp, B, Cc, h, w, hp, wp, k,
                                              _ptr(x), _ptr(y_kept), _ptr(kept_idx), _ptr(keep_mask),
                                              _ptr(cache_prev), _ptr(out), _ptr(cache_new))
        self._check(rc, "nova_merge_cache_interp")

    # -- a cache in 4 bits ----------------------------------------------------------
    # These work on the context's device, on that device's current stream, whichever device is current.
    def _here(self, *ts: Optional[torch.Tensor]):
        for t in ts:
            if t is not None and t.get_device() != self.device:
                raise ValueError(f"tensor on {t.device}, context on device {self.device}")

    def _cache(self, cache: FourBitCache) -> "_FourBitCache":
        c = cache.c_struct()
        if c.device != self.device:
            raise ValueError(f"cache on device {c.device}, context on device {self.device}")
        return c

    def _counts(self, B: int, name: str, t: Optional[torch.Tensor]) -> Optional[int]:
        return None if t is None else _shaped(name, t, (B,), torch.int32, self.device)

    def fourbit_append(self, cache: FourBitCache, k: torch.Tensor, v: torch.Tensor, kv_len: int,
                       n_per_row: Optional[torch.Tensor] = None, kv_len_per_row: Optional[torch.Tensor] = None,
                       kv_len_next: Optional[torch.Tensor] = None):
        """Quantises k, v [B, n, kv_heads, dh] (f32|bf16, any strides) behind the images' rows.  kv_len: rows every image
        has, or the upper bound of kv_len_per_row ([B] int32, like n_per_row and kv_len_next)."""
        c = self._cache(cache)
        if k.shape != v.shape or k.dtype != v.dtype or k.shape[0] != c.B:
            raise ValueError(f"k {tuple(k.shape)} {k.dtype}, v {tuple(v.shape)} {v.dtype}, {c.B} images in the cache")
        self._here(k, v)
        rc = self.lib.nova_fourbit_append(
            self.ctx, _stream(self.device), _dtype_code(k), c, k.shape[1], _rows(k, c.kv_heads, c.dh, "k"),
            _rows(v, c.kv_heads, c.dh, "v"), self._counts(c.B, "n_per_row", n_per_row), kv_len,
            self._counts(c.B, "kv_len_per_row", kv_len_per_row), self._counts(c.B, "kv_len_next", kv_len_next))
        if rc:
            self._check(rc, "nova_fourbit_append")

    def fourbit_unpack(self, cache: FourBitCache, first: int, k: Optional[torch.Tensor], v: Optional[torch.Tensor],
                       first_per_row: Optional[torch.Tensor] = None, n_per_row: Optional[torch.Tensor] = None):
        """Values of cached rows from row `first` on, into k and v [B, n, kv_heads, dh] (f32|bf16, any strides)."""
        c = self._cache(cache)
        a = v if k is None else k
        if a is None:
            return
        if v is not None and (v.shape != a.shape or v.dtype != a.dtype) or a.shape[0] != c.B:
            raise ValueError(f"outputs {[None if t is None else (tuple(t.shape), t.dtype) for t in (k, v)]}, {c.B} images in the "
                             "cache")
        self._here(k, v)
        rc = self.lib.nova_fourbit_unpack(
            self.ctx, _stream(self.device), _dtype_code(a), c, first, a.shape[1],
            self._counts(c.B, "first_per_row", first_per_row), self._counts(c.B, "n_per_row", n_per_row),
            None if k is None else _rows(k, c.kv_heads, c.dh, "k"), None if v is None else _rows(v, c.kv_heads, c.dh, "v"))
        if rc:
            self._check(rc, "nova_fourbit_unpack")

    def fourbit_attention_workspace_bytes(self, cache: FourBitCache, heads: int, n: int, kv_len: int) -> int:
        return self.lib.nova_fourbit_attention_workspace_bytes(cache.c_struct(), heads, n, kv_len)

    def fourbit_attention(self, cache: FourBitCache, q: torch.Tensor, out: torch.Tensor, workspace: Optional[torch.Tensor],
                          kv_len: int, scale: Optional[float] = None, lse: Optional[torch.Tensor] = None,
                          n_per_row: Optional[torch.Tensor] = None, kv_len_per_row: Optional[torch.Tensor] = None):
        """out [B, n, heads, dh] = attention of q [B, n, heads, dh] (f32|bf16, channels dense) over the cached rows; lse
        [B, n, heads] f32 or None.  scale: 1 / sqrt(dh) where None."""
        c = self._cache(cache)
        shape = q.shape
        B, n, heads, dh = shape
        if B != c.B:
            raise ValueError(f"{B} images of queries, {c.B} in the cache")
        dev = self.device
        self._here(q, workspace)
        rc = self.lib.nova_fourbit_attention(
            self.ctx, _stream(dev), _dtype_code(q), c, heads, n, _rows(q, heads, c.dh, "q"),
            self._counts(B, "n_per_row", n_per_row), kv_len, self._counts(B, "kv_len_per_row", kv_len_per_row),
            dh ** -0.5 if scale is None else scale, _shaped("out", out, shape, q.dtype, dev),
            _shaped("lse", lse, (B, n, heads), torch.float32, dev), _ptr(workspace),
            0 if workspace is None else workspace.nbytes)
        if rc:
            self._check(rc, "nova_fourbit_attention")

    def fourbit_mass_workspace_bytes(self, cache: FourBitCache, heads: int, n: int, kv_len: int) -> int:
        return self.lib.nova_fourbit_mass_workspace_bytes(cache.c_struct(), heads, n, kv_len)

    def fourbit_mass(self, cache: FourBitCache, q: torch.Tensor, lse: torch.Tensor, mass: torch.Tensor,
                     workspace: Optional[torch.Tensor], kv_len: int, scale: Optional[float] = None,
                     mass_in: Optional[torch.Tensor] = None, n_per_row: Optional[torch.Tensor] = None,
                     kv_len_per_row: Optional[torch.Tensor] = None):
        """mass [B, capacity] f32: mass_in (may be the same tensor; None: zeros) plus what the cached rows collect from q; lse
        as fourbit_attention wrote it."""
        c = self._cache(cache)
        B, n, heads, dh = q.shape
        if B != c.B:
            raise ValueError(f"{B} images of queries, {c.B} in the cache")
        dev, per_row = self.device, (B, c.capacity)
        self._here(q, workspace)
        rc = self.lib.nova_fourbit_mass(
            self.ctx, _stream(dev), _dtype_code(q), c, heads, n, _rows(q, heads, c.dh, "q"),
            self._counts(B, "n_per_row", n_per_row), kv_len, self._counts(B, "kv_len_per_row", kv_len_per_row),
            dh ** -0.5 if scale is None else scale, _shaped("lse", lse, (B, n, heads), torch.float32, dev),
            _shaped("mass_in", mass_in, per_row, torch.float32, dev), _shaped("mass", mass, per_row, torch.float32, dev),
            _ptr(workspace), 0 if workspace is None else workspace.nbytes)
        if rc:
            self._check(rc, "nova_fourbit_mass")

    def fourbit_evict(self, src: FourBitCache, dst: FourBitCache, kept_idx: torch.Tensor, kv_len: int,
                      k_per_row: Optional[torch.Tensor] = None, kv_len_per_row: Optional[torch.Tensor] = None,
                      kv_len_next: Optional[torch.Tensor] = None, mass_src: Optional[torch.Tensor] = None,
                      mass_dst: Optional[torch.Tensor] = None):
        """Rows kept_idx [B, k] of src to the front of dst, with their masses."""
        s, d = self._cache(src), self._cache(dst)
        B, k, dev = s.B, kept_idx.shape[1], self.device
        rc = self.lib.nova_fourbit_evict(
            self.ctx, _stream(dev), s, d, k, _shaped("kept_idx", kept_idx, (B, k), torch.int32, dev),
            self._counts(B, "k_per_row", k_per_row), kv_len, self._counts(B, "kv_len_per_row", kv_len_per_row),
            self._counts(B, "kv_len_next", kv_len_next), _shaped("mass_src", mass_src, (B, s.capacity), torch.float32, dev),
            _shaped("mass_dst", mass_dst, (B, d.capacity), torch.float32, dev))
        if rc:
            self._check(rc, "nova_fourbit_evict")

    def fourbit_block_workspace_bytes(self, shape: BlockShape) -> int:
        return self.lib.nova_fourbit_block_workspace_bytes(C.byref(shape.c_struct()))

    def pruned_block_fourbit(self, shape: BlockShape, weights: Dict[str, Optional[torch.Tensor]],
                             variant: Optional[BlockVariant], k_per_row: Optional[torch.Tensor],
                             kv_len_per_row: Optional[torch.Tensor], kv_len_next: Optional[torch.Tensor],
                             x: torch.Tensor, kept_idx: torch.Tensor, cache: FourBitCache, y_kept: torch.Tensor,
                             workspace: torch.Tensor, mass: Optional[torch.Tensor] = None,
                             mass_in: Optional[torch.Tensor] = None):
        """nova_pruned_block_fourbit: pruned_block_rows with the block's cache in 4 bits; mass [B, capacity] f32 (and mass_in,
        what the rows had before) where the weight they collect is wanted."""
        c = self._cache(cache)
        B = shape.B
        self._here(x, kept_idx, y_kept, workspace)
        s = shape.c_struct()
        w = _Weights(*[_ptr(weights.get(n)) for n, _ in _Weights._fields_])
        rc = self.lib.nova_pruned_block_fourbit(
            self.ctx, _stream(self.device), C.byref(s), C.byref(w), None if variant is None else C.byref(variant.c_struct()),
            self._counts(B, "k_per_row", k_per_row), self._counts(B, "kv_len_per_row", kv_len_per_row),
            self._counts(B, "kv_len_next", kv_len_next), _ptr(x), _ptr(kept_idx), c,
            _shaped("mass_in", mass_in, (B, c.capacity), torch.float32, self.device),
            _shaped("mass", mass, (B, c.capacity), torch.float32, self.device), _ptr(y_kept), _ptr(workspace), workspace.nbytes)
        if rc:
            self._check(rc, "nova_pruned_block_fourbit")


# ------------------------------------------------------------------------------------
# KV-cache layout helpers (pure permutations, no arithmetic).  The library stores keys
# as [B, heads, capacity, dh] and values key-minor as [B, heads, dh, capacity].
# ------------------------------------------------------------------------------------
def pack_k_cache(k_rows: torch.Tensor, heads: int, capacity: int, fill: float = 0.0) -> torch.Tensor:
    """[B, P, C] logical key rows -> [B, heads, capacity, dh] with rows [0, P) filled."""
    B, P, Cc = k_rows.shape
    dh = Cc // heads
    out = torch.full((B, heads, capacity, dh), fill, dtype=k_rows.dtype, device=k_rows.device)
    out[:, :, :P] = k_rows.reshape(B, P, heads, dh).permute(0, 2, 1, 3)
    return out


def pack_v_cache(v_rows: torch.Tensor, heads: int, capacity: int, fill: float = 0.0) -> torch.Tensor:
    """[B, P, C] logical value rows -> [B, heads, dh, capacity] with columns [0, P) filled."""
    B, P, Cc = v_rows.shape
    dh = Cc // heads
    out = torch.full((B, heads, dh, capacity), fill, dtype=v_rows.dtype, device=v_rows.device)
    out[:, :, :, :P] = v_rows.reshape(B, P, heads, dh).permute(0, 2, 3, 1)
    return out


def unpack_k_rows(k_cache: torch.Tensor, start: int, stop: int) -> torch.Tensor:
    """cache rows [start, stop) back to the logical [B, stop-start, C]."""
    B, H, _, dh = k_cache.shape
    return k_cache[:, :, start:stop].permute(0, 2, 1, 3).reshape(B, stop - start, H * dh)


def unpack_v_rows(v_cache: torch.Tensor, start: int, stop: int) -> torch.Tensor:
    B, H, dh, _ = v_cache.shape
    return v_cache[:, :, :, start:stop].permute(0, 3, 1, 2).reshape(B, stop - start, H * dh)
