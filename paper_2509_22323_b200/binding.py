"""ctypes binding of librapid3.so: argument marshalling only.

Every step of the path runs in the CUDA kernels behind the C ABI (include/rapid3.h); torch is
used for device memory and streams.  There is no CPU fallback: if the shared library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import array
import ctypes
import os
import types
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "librapid3.so")

OK = 0
ACT_SKIP, ACT_REUSE, ACT_ATTEND = 0, 1, 2

EXPORTS = [
    "rapid3_create", "rapid3_destroy", "rapid3_strerror", "rapid3_num_blocks", "rapid3_mask_words",
    "rapid3_block_scores", "rapid3_select_mask", "rapid3_sparse_joint_attn", "rapid3_gated_step",
    "rapid3_gated_step_host", "rapid3_workspace", "rapid3_launch_count", "rapid3_last_status",
    "rapid3_profile", "rapid3_profile_read", "rapid3_block_scores_static", "rapid3_static_scratch_bytes", "rapid3_cache_step", "rapid3_gated_step_device", "rapid3_gated_step_heads", "rapid3_equivalent_steps", "rapid3_select_mask_mass", "rapid3_gated_step_fused", "rapid3_gated_step_mass",
    "rapid3_debug_inject_timeout",
    "rapid3_rotary", "rapid3_norm_rotary", "rapid3_norm_rotary_backward", "rapid3_norm_rotary_workspace_bytes", "rapid3_rotary_freqs",
    "rapid3_window_attn", "rapid3_window_attn_backward", "rapid3_window_workspace_bytes", "rapid3_window_status",
]


class Rapid3Error(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {strerror(code)} ({code})")
        self.code = code


class Shape(ctypes.Structure):
    _fields_ = [("B_max", ctypes.c_int32), ("H", ctypes.c_int32), ("D", ctypes.c_int32),
                ("n_text", ctypes.c_int32), ("n_image", ctypes.c_int32), ("block", ctypes.c_int32),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64)]


class Heads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("type", "B", "N", "D", "H_q", "H_k")]


class Turn(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("channels", ctypes.c_int32), ("axes", ctypes.c_int32), ("axis_pairs", ctypes.c_int32 * 4),
                ("freq", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("pos_stride_b", ctypes.c_int64), ("pos_stride_n", ctypes.c_int64),
                ("pos0", ctypes.c_int32), ("amplitude", ctypes.c_float)]


class Window(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("type", "B", "H", "H_kv", "D", "n_q", "n_kv", "left", "right", "n_sink", "n_full")] + [
        ("softmax_scale", ctypes.c_float), ("q_len", ctypes.c_void_p), ("kv_len", ctypes.c_void_p)]


_lib = None


def load() -> ctypes.CDLL:
    """Loads librapid3.so (built in-tree by paper_2509_22323_b200.build); raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} not found: build the CUDA library first (python -m paper_2509_22323_b200.build); "
            "there is no CPU fallback")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    i32p, f32p, i64p = ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int64)
    lib.rapid3_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Shape)]
    lib.rapid3_destroy.argtypes = [vp]
    lib.rapid3_strerror.argtypes = [ci]
    lib.rapid3_strerror.restype = ctypes.c_char_p
    lib.rapid3_num_blocks.argtypes = [ctypes.POINTER(Shape)]
    lib.rapid3_mask_words.argtypes = [ctypes.POINTER(Shape)]
    lib.rapid3_block_scores.argtypes = [vp, vp, vp, i32p, ci, vp, vp]
    lib.rapid3_select_mask.argtypes = [vp, vp, f32p, ci, vp, vp, vp, vp]
    lib.rapid3_select_mask_mass.argtypes = [vp, vp, f32p, cf, ci, vp, vp, vp, vp, vp]
    lib.rapid3_sparse_joint_attn.argtypes = [vp, vp, vp, vp, vp, i32p, ci, vp, vp, cf, vp]
    lib.rapid3_gated_step.argtypes = [vp, vp, vp, vp, vp, i32p, f32p, ci, cf, vp]
    lib.rapid3_gated_step_fused.argtypes = [vp, vp, vp, vp, vp, vp, vp, cf, vp, vp, vp, i32p, f32p, ci, cf, vp]
    lib.rapid3_gated_step_mass.argtypes = [vp, vp, vp, vp, vp, i32p, f32p, cf, ci, cf, vp]
    lib.rapid3_gated_step_heads.argtypes = [vp, vp, vp, vp, vp, i32p, f32p, ci, cf, vp]
    lib.rapid3_gated_step_device.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, cf, vp]
    lib.rapid3_gated_step_host.argtypes = [vp, vp, vp, vp, vp, i32p, f32p, ci, cf, vp, i64p, i64p]
    lib.rapid3_debug_inject_timeout.argtypes = [vp, vp, vp, vp, vp, ci, cf, vp]
    lib.rapid3_workspace.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp)]
    lib.rapid3_launch_count.argtypes = [vp]
    lib.rapid3_launch_count.restype = ctypes.c_int64
    lib.rapid3_last_status.argtypes = [vp, ctypes.POINTER(ci)]
    lib.rapid3_profile.argtypes = [vp, ci]
    lib.rapid3_profile_read.argtypes = [vp, ctypes.POINTER(ctypes.c_double), i64p]
    lib.rapid3_block_scores_static.argtypes = [ctypes.POINTER(Shape), vp, vp, i32p, ci, vp, vp]
    lib.rapid3_static_scratch_bytes.argtypes = []
    lib.rapid3_equivalent_steps.argtypes = [i32p, f32p, f32p, ci, ctypes.POINTER(ctypes.c_double), i64p]
    lib.rapid3_cache_step.argtypes = [vp, vp, vp, i32p, ci, ctypes.c_int64, vp]
    lib.rapid3_static_scratch_bytes.restype = ctypes.c_int64
    rows, heads, turn = ctypes.POINTER(Rows), ctypes.POINTER(Heads), ctypes.POINTER(Turn)
    lib.rapid3_rotary.argtypes = [heads, rows, rows, turn, ci, rows, rows, vp]
    lib.rapid3_norm_rotary.argtypes = [heads, rows, rows, vp, vp, cf, turn, rows, rows, vp]
    lib.rapid3_norm_rotary_backward.argtypes = [heads, rows, rows, rows, rows, vp, vp, cf, turn, rows, rows, vp, vp, vp, ctypes.c_int64, vp]
    lib.rapid3_norm_rotary_workspace_bytes.argtypes = [heads]
    lib.rapid3_norm_rotary_workspace_bytes.restype = ctypes.c_int64
    win = ctypes.POINTER(Window)
    lib.rapid3_window_attn.argtypes = [win, rows, rows, rows, rows, vp, vp]
    lib.rapid3_window_attn_backward.argtypes = [win, rows, rows, rows, rows, vp, rows, rows, rows, rows, vp, ctypes.c_int64, vp]
    lib.rapid3_window_workspace_bytes.argtypes = [win]
    lib.rapid3_window_workspace_bytes.restype = ctypes.c_int64
    lib.rapid3_window_status.argtypes = [ctypes.POINTER(ci)]
    lib.rapid3_rotary_freqs.argtypes = [ci, ctypes.c_double, ci, ctypes.c_double, ci, ctypes.c_double, ctypes.c_double, ctypes.POINTER(ctypes.c_double), f32p]
    # the same calls with addresses in the place of the Rows: the functions below lay the rows of a call out in one array
    lib.by_address = types.SimpleNamespace()
    for name in ("rapid3_rotary", "rapid3_norm_rotary", "rapid3_norm_rotary_backward", "rapid3_window_attn", "rapid3_window_attn_backward"):
        fn = lib[name]                             # a function object of its own
        fn.argtypes = [vp if t is rows else t for t in getattr(lib, name).argtypes]
        setattr(lib.by_address, name, fn)
    _lib = lib
    return lib


def strerror(code: int) -> str:
    return load().rapid3_strerror(int(code)).decode()


def _check(code: int, what: str):
    if code != OK:
        raise Rapid3Error(code, what)


def _i32(xs: Optional[Sequence[int]]):
    if xs is None:
        return None
    return (ctypes.c_int32 * len(xs))(*[int(x) for x in xs])


def _f32(xs: Sequence[float]):
    # Number by number through ctypes 192 ratios take 22 us of a call, by way of an array 3.8; four or fewer are the faster so
    # (one 0.45 and 0.70 us, four 0.80 and 0.77).  Only of a list or tuple is an array sure to take the elements: of bytes it takes the memory.
    n = len(xs)
    if n > 4 and isinstance(xs, (list, tuple)):
        try:
            return (ctypes.c_float * n).from_buffer(array.array("f", xs))
        except TypeError:                          # elements that only float() takes
            pass
    return (ctypes.c_float * n)(*[float(x) for x in xs])


def _stream() -> int:
    # the handle of torch.cuda.current_stream() without the Stream object around it, which takes 3.2 us of a call to build (0.2 so)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


class Context:
    """Owns a rapid3_ctx for tensors of shape [B<=B_max, H, N, D] with the given element strides."""

    def __init__(self, B_max: int, H: int, D: int, n_text: int, n_image: int,
                 strides: Optional[Sequence[int]] = None):
        self.lib = load()
        N = n_text + n_image
        if strides is None:
            strides = (H * N * D, N * D, D)
        self.shape = Shape(B_max, H, D, n_text, n_image, 64, int(strides[0]), int(strides[1]), int(strides[2]))
        self.B_max, self.H, self.D, self.n_text, self.n_image, self.N = B_max, H, D, n_text, n_image, N
        self.handle = ctypes.c_void_p()
        _check(self.lib.rapid3_create(ctypes.byref(self.handle), ctypes.byref(self.shape)), "rapid3_create")
        self.nb = self.lib.rapid3_num_blocks(ctypes.byref(self.shape))
        self.words = self.lib.rapid3_mask_words(ctypes.byref(self.shape))

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            self.lib.rapid3_destroy(self.handle)
            self.handle = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- the four calls of the path (same names as the C ABI) ----
    def rapid3_block_scores(self, q: torch.Tensor, k: torch.Tensor, img_idx: Optional[Sequence[int]] = None,
                            n_img: Optional[int] = None, scores: Optional[torch.Tensor] = None) -> torch.Tensor:
        n = len(img_idx) if img_idx is not None else (n_img if n_img is not None else q.shape[0])
        if scores is None:
            scores = torch.empty((n, self.H, self.nb, self.nb), dtype=torch.float32, device=q.device)
        _check(self.lib.rapid3_block_scores(self.handle, _ptr(q), _ptr(k), _i32(img_idx), n, _ptr(scores), _stream()),
               "rapid3_block_scores")
        return scores

    def rapid3_select_mask(self, scores: torch.Tensor, keep_ratio: Sequence[float], out=None):
        n = len(keep_ratio)
        dev = scores.device
        if out is None:
            bitmask = torch.empty((n, self.H, self.nb, self.words), dtype=torch.int64, device=dev)
            kept_idx = torch.empty((n, self.H, self.nb, self.nb), dtype=torch.int32, device=dev)
            kept_cnt = torch.empty((n, self.H, self.nb), dtype=torch.int32, device=dev)
        else:
            bitmask, kept_idx, kept_cnt = out
        _check(self.lib.rapid3_select_mask(self.handle, _ptr(scores), _f32(keep_ratio), n, _ptr(bitmask),
                                           _ptr(kept_idx), _ptr(kept_cnt), _stream()), "rapid3_select_mask")
        return bitmask, kept_idx, kept_cnt

    def rapid3_select_mask_mass(self, scores: torch.Tensor, mass_share: Sequence[float], mass_scale: float):
        """Cumulative-mass selection: returns (row_keep, bitmask, kept_idx, kept_cnt)."""
        n = scores.shape[0]
        assert len(mass_share) == n and scores.dtype == torch.float32 and scores.is_contiguous()
        dev = scores.device
        row_keep = torch.empty((n, self.H, self.nb), dtype=torch.int32, device=dev)
        bitmask = torch.empty((n, self.H, self.nb, self.words), dtype=torch.int64, device=dev)
        kept_idx = torch.empty((n, self.H, self.nb, self.nb), dtype=torch.int32, device=dev)
        kept_cnt = torch.empty((n, self.H, self.nb), dtype=torch.int32, device=dev)
        _check(self.lib.rapid3_select_mask_mass(self.handle, _ptr(scores), _f32(mass_share), float(mass_scale), n,
                                                _ptr(row_keep), _ptr(bitmask), _ptr(kept_idx), _ptr(kept_cnt),
                                                _stream()), "rapid3_select_mask_mass")
        return row_keep, bitmask, kept_idx, kept_cnt

    def rapid3_sparse_joint_attn(self, q, k, v, out, img_idx: Optional[Sequence[int]] = None,
                                 n_img: Optional[int] = None, kept_idx=None, kept_cnt=None,
                                 softmax_scale: Optional[float] = None):
        n = len(img_idx) if img_idx is not None else (n_img if n_img is not None else q.shape[0])
        scale = softmax_scale if softmax_scale is not None else self.D ** -0.5
        _check(self.lib.rapid3_sparse_joint_attn(self.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _i32(img_idx), n,
                                                 _ptr(kept_idx), _ptr(kept_cnt), scale, _stream()),
               "rapid3_sparse_joint_attn")
        return out

    def rapid3_gated_step(self, q, k, v, out, actions: Sequence[int], keep_ratio: Sequence[float],
                          softmax_scale: Optional[float] = None):
        scale = softmax_scale if softmax_scale is not None else self.D ** -0.5
        _check(self.lib.rapid3_gated_step(self.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _i32(actions),
                                          _f32(keep_ratio), len(actions), scale, _stream()), "rapid3_gated_step")
        return out

    def rapid3_gated_step_fused(self, q_raw, k_raw, v, q_gain, k_gain, rot, eps: float, q, k, out,
                                actions: Sequence[int], keep_ratio: Sequence[float],
                                softmax_scale: Optional[float] = None):
        """q_raw, k_raw -> (RMS norm, gain, rotary) -> q, k (may alias the raw tensors), then the gated step."""
        scale = softmax_scale if softmax_scale is not None else self.D ** -0.5
        assert q_gain.dtype == torch.float32 and k_gain.dtype == torch.float32
        assert rot is None or (rot.dtype == torch.float32 and rot.is_contiguous())
        _check(self.lib.rapid3_gated_step_fused(self.handle, _ptr(q_raw), _ptr(k_raw), _ptr(v), _ptr(q_gain),
                                                _ptr(k_gain), _ptr(rot), float(eps), _ptr(q), _ptr(k), _ptr(out),
                                                _i32(actions), _f32(keep_ratio), len(actions), scale, _stream()),
               "rapid3_gated_step_fused")
        return out

    def rapid3_gated_step_mass(self, q, k, v, out, actions: Sequence[int], mass_share: Sequence[float],
                               mass_scale: float, softmax_scale: Optional[float] = None):
        """The gated step with the cumulative-mass selection (share per image) instead of top-k."""
        scale = softmax_scale if softmax_scale is not None else self.D ** -0.5
        _check(self.lib.rapid3_gated_step_mass(self.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _i32(actions),
                                               _f32(mass_share), float(mass_scale), len(actions), scale, _stream()),
               "rapid3_gated_step_mass")
        return out

    def rapid3_gated_step_heads(self, q, k, v, out, actions: Sequence[int], keep_ratio: Sequence[Sequence[float]],
                                softmax_scale: Optional[float] = None):
        """keep_ratio: [B][H], one ratio per image and head."""
        scale = softmax_scale if softmax_scale is not None else self.D ** -0.5
        flat = [r for row in keep_ratio for r in row]
        assert len(flat) == len(actions) * self.H
        _check(self.lib.rapid3_gated_step_heads(self.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _i32(actions),
                                                _f32(flat), len(actions), scale, _stream()),
               "rapid3_gated_step_heads")
        return out

    def rapid3_gated_step_device(self, q, k, v, out, actions_dev: torch.Tensor, keep_ratio_dev: torch.Tensor,
                                 softmax_scale: Optional[float] = None):
        """actions_dev: int32 [B], keep_ratio_dev: float32 [B], both on the GPU; no host read-back."""
        assert actions_dev.dtype == torch.int32 and keep_ratio_dev.dtype == torch.float32
        scale = softmax_scale if softmax_scale is not None else self.D ** -0.5
        _check(self.lib.rapid3_gated_step_device(self.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(actions_dev),
                                                 _ptr(keep_ratio_dev), int(actions_dev.numel()), scale, _stream()),
               "rapid3_gated_step_device")
        return out

    def rapid3_gated_step_host(self, q, k, v, out, actions: Sequence[int], keep_ratio: Sequence[float],
                               softmax_scale: Optional[float] = None):
        """q, k, v, out: contiguous HOST bf16 tensors [B, H, N, D] (pinned for asynchronous copies)."""
        scale = softmax_scale if softmax_scale is not None else self.D ** -0.5
        up, down = ctypes.c_int64(0), ctypes.c_int64(0)
        _check(self.lib.rapid3_gated_step_host(self.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _i32(actions),
                                               _f32(keep_ratio), len(actions), scale, _stream(),
                                               ctypes.byref(up), ctypes.byref(down)), "rapid3_gated_step_host")
        return up.value, down.value

    def rapid3_debug_inject_timeout(self, q, k, v, out, stop_group: int, softmax_scale: Optional[float] = None):
        """Test aid: dense attention over image 0 with the failure-injection build of the kernel."""
        scale = softmax_scale if softmax_scale is not None else self.D ** -0.5
        _check(self.lib.rapid3_debug_inject_timeout(self.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out), int(stop_group),
                                                    scale, _stream()), "rapid3_debug_inject_timeout")

    # ---- helpers ----
    def workspace(self, n_sparse: int, device="cuda"):
        """Views (no copy) of the scores / bitmask / kept lists the last gated step wrote."""
        ptrs = [ctypes.c_void_p() for _ in range(4)]
        _check(self.lib.rapid3_workspace(self.handle, *[ctypes.byref(p) for p in ptrs]), "rapid3_workspace")
        shapes = [((n_sparse, self.H, self.nb, self.nb), torch.float32),
                  ((n_sparse, self.H, self.nb, self.words), torch.int64),
                  ((n_sparse, self.H, self.nb, self.nb), torch.int32),
                  ((n_sparse, self.H, self.nb), torch.int32)]
        return [_view(p.value, s, d, device) for p, (s, d) in zip(ptrs, shapes)]

    def launch_count(self) -> int:
        return int(self.lib.rapid3_launch_count(self.handle))

    def profile(self, enable):
        """False / 0: off; True / 1: an event pair around every launch; 2: around the attention kernel only."""
        _check(self.lib.rapid3_profile(self.handle, int(enable)), "rapid3_profile")

    def profile_read(self):
        """Summed device milliseconds and launch counts per kernel kind since the last read."""
        ms = (ctypes.c_double * 4)()
        n = (ctypes.c_int64 * 4)()
        _check(self.lib.rapid3_profile_read(self.handle, ms, n), "rapid3_profile_read")
        kinds = ("block_pool", "block_scores", "select_mask", "attention")
        return {k: (ms[i], n[i]) for i, k in enumerate(kinds)}

    def last_status(self) -> int:
        v = ctypes.c_int(0)
        _check(self.lib.rapid3_last_status(self.handle, ctypes.byref(v)), "rapid3_last_status")
        return v.value


def rapid3_block_scores_static(shape: Shape, q: torch.Tensor, k: torch.Tensor, scores: torch.Tensor,
                               img_idx: Optional[Sequence[int]] = None, n_img: Optional[int] = None) -> torch.Tensor:
    """Context-free scoring pass for hosts that may not allocate device memory: the block means go
    to the fixed array inside the library instead of a workspace.  `scores` ([n, H, nb, nb] fp32,
    device) is supplied by the caller; nothing is allocated here either."""
    n = len(img_idx) if img_idx is not None else (n_img if n_img is not None else q.shape[0])
    _check(load().rapid3_block_scores_static(ctypes.byref(shape), _ptr(q), _ptr(k), _i32(img_idx), n, _ptr(scores),
                                             _stream()), "rapid3_block_scores_static")
    return scores


def rapid3_equivalent_steps(actions: Sequence[int], c_cache: Sequence[float], c_sparse: Sequence[float]):
    """Equivalent steps K of one trajectory: (exact sum, nearest integer)."""
    n = len(actions)
    assert len(c_cache) == n and len(c_sparse) == n
    k, kr = ctypes.c_double(0.0), ctypes.c_int64(0)
    _check(load().rapid3_equivalent_steps(_i32(actions), _f32(c_cache), _f32(c_sparse), n, ctypes.byref(k),
                                          ctypes.byref(kr)), "rapid3_equivalent_steps")
    return k.value, kr.value


def rapid3_cache_step(x: torch.Tensor, o: torch.Tensor, delta: torch.Tensor, actions: Sequence[int]):
    """Cache-Reuse data path over a batch [B, ...] of contiguous bf16 tensors: refreshes `delta` for
    attending images, writes `o` for reusing ones, leaves skipped ones alone."""
    B = len(actions)
    elems = x[0].numel()
    _check(load().rapid3_cache_step(_ptr(x), _ptr(o), _ptr(delta), _i32(actions), B, elems, _stream()),
           "rapid3_cache_step")


_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


# The checks of the calls below cost a third of a small call on the host (13 us when they were written for brevity): tensor by tensor, each
# attribute read once, and what is wrong said only when something is.
def _device(what: str, like: torch.Tensor) -> int:
    dev = like.get_device()
    if dev < 0 or dev != torch._C._cuda_getDevice():
        raise ValueError(f"{what}: tensors must be on the current CUDA device")
    return dev


def _tensors(what: str, dtype: torch.dtype, dev: int, items):
    """One rapid3_rows (data, stride_b, stride_h, stride_n) after the other for (name, tensor, shape)s, checked; the array, and its address: number i
    lies 32 i behind it."""
    words = []
    for name, t, shape in items:
        if t is None or t.dtype is not dtype or t.get_device() != dev or t.shape != shape:
            raise ValueError(f"{what}: {name} must be {tuple(shape)} of {dtype} on CUDA device {dev}")
        sb, sh, sn, sd = t.stride()
        if sd != 1:
            raise ValueError(f"{what}: {name} must have adjacent channels")
        words += (t.data_ptr(), sb, sh, sn)
    rows = array.array("q", words)                 # (a ctypes array takes 0.6 us more)
    return rows, rows.buffer_info()[0]


def _check_vector(what: str, name: str, t: Optional[torch.Tensor], n: int, dev: int, dtype=torch.float32):
    if t is None or t.dtype is not dtype or t.get_device() != dev or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what}: {name} must be {n} contiguous values of {dtype} on CUDA device {dev}")


def rapid3_rotary_freqs(channels: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained: int = 1,
                        fast_turns: float = 32.0, slow_turns: float = 1.0):
    """Radians per position of channels / 2 pairs (fp64, on the host) and the amplitude; scaling: "none", "linear", "base", "parts"."""
    freq, amplitude = torch.empty(max(0, channels) // 2, dtype=torch.float64), ctypes.c_float(0.0)
    kind = {"none": 0, "linear": 1, "base": 2, "parts": 3}.get(scaling, -1)
    _check(load().rapid3_rotary_freqs(int(channels), float(base), kind, float(factor), int(trained), float(fast_turns), float(slow_turns),
                                      ctypes.cast(freq.data_ptr(), ctypes.POINTER(ctypes.c_double)), ctypes.byref(amplitude)), "rapid3_rotary_freqs")
    return freq, amplitude.value


class Rotary:
    """How positions turn the heads of rapid3_rotary and rapid3_norm_rotary: made once, used for any number of calls.

    layout      "pairs": channels (2 i, 2 i + 1) turn together; "halves": (i, i + channels / 2)
    freq        fp64 [channels / 2] on the GPU, radians per position (see rapid3_rotary_freqs)
    pos         int32 [B or 1, N, axes] on the GPU, read when the kernels run; None: pos0 + n
    axis_pairs  how many pairs each coordinate turns, in order; None: the first turns all
    """

    def __init__(self, layout: str, freq: torch.Tensor, pos: Optional[torch.Tensor] = None, pos0: int = 0, amplitude: float = 1.0,
                 axis_pairs: Optional[Sequence[int]] = None):
        if layout not in ("pairs", "halves"):
            raise ValueError("Rotary: layout must be 'pairs' or 'halves'")
        if freq.dtype != torch.float64 or freq.dim() != 1 or not freq.is_contiguous() or not freq.is_cuda:
            raise ValueError("Rotary: freq must be a contiguous fp64 vector on the GPU")
        axes = 1 if pos is None else pos.shape[-1]
        if pos is not None and (pos.dtype != torch.int32 or pos.dim() != 3 or pos.device != freq.device or not 1 <= axes <= 4 or
                                (pos.stride(-1) != 1 and axes > 1)):
            raise ValueError("Rotary: pos must be int32 [B or 1, N, axes], 1 to 4 axes, adjacent, beside freq")
        pairs = [freq.numel()] if axis_pairs is None else [int(x) for x in axis_pairs]
        if len(pairs) > axes or sum(pairs) != freq.numel() or min(pairs) < 0:
            raise ValueError("Rotary: axis_pairs must be one count for each axis, freq's length in all")
        pairs += [0] * (4 - len(pairs))
        self.freq, self.pos, self.device = freq, pos, freq.get_device()
        self.B, self.N = (0, 0) if pos is None else pos.shape[:2]
        self.turn = Turn(0 if layout == "pairs" else 1, 2 * freq.numel(), axes, (ctypes.c_int32 * 4)(*pairs), freq.data_ptr(), _ptr(pos),
                         0 if pos is None or self.B == 1 else pos.stride(0), 0 if pos is None or self.N == 1 else pos.stride(1), int(pos0),
                         float(amplitude))

    def check(self, what: str, dev: int, B: int, N: int):
        if self.device != dev or (self.pos is not None and (self.N != N or (self.B != 1 and self.B != B))):
            raise ValueError(f"{what}: the positions are those of {self.B} x {self.N} tokens on CUDA device {self.device}, not of {B} x {N} on {dev}")


def _heads(what: str, q: torch.Tensor, k: Optional[torch.Tensor], rotary: Rotary, like_q, like_k):
    """The shape of Q and K (k may be None), after checking them and what is like them, (name, tensor)s; the device; and _tensors() of q, like_q, k, like_k."""
    shape, dtype, dev = q.shape, q.dtype, _device(what, q)
    kind = _TYPES.get(dtype)
    if kind is None or len(shape) != 4:
        raise ValueError(f"{what}: q must be [B, H, N, D] of bf16, fp16 or fp32")
    B, H, N, D = shape
    rotary.check(what, dev, B, N)
    items = [("q", q, shape)] + [(name, t, shape) for name, t in like_q]
    Hk = 0
    if k is not None:
        k_shape = k.shape
        if len(k_shape) != 4 or k_shape[0] != B or k_shape[2] != N or k_shape[3] != D:
            raise ValueError(f"{what}: k must be [B, H, N, D] and differ from q in H only")
        Hk = k_shape[1]
        items += [("k", k, k_shape)] + [(name, t, k_shape) for name, t in like_k]
    rows, at = _tensors(what, dtype, dev, items)
    return Heads(kind, B, N, D, H, Hk), dev, rows, at


def rapid3_rotary(q: torch.Tensor, k: Optional[torch.Tensor], rotary: Rotary, q_out: Optional[torch.Tensor] = None,
                  k_out: Optional[torch.Tensor] = None, backward: bool = False):
    """Turns Q and K heads ([B, H, N, D], any heads each; k may be None) by their positions; outputs may be the inputs.
    backward: q and k are gradients of the outputs, and those of the inputs come back."""
    q_out = torch.empty_like(q) if q_out is None else q_out
    k_out = torch.empty_like(k) if k_out is None and k is not None else k_out
    shape, _, rows, at = _heads("rapid3_rotary", q, k, rotary, (("q_out", q_out),), (("k_out", k_out),))
    k_at, kout_at = (None, None) if k is None else (at + 64, at + 96)
    _check(load().by_address.rapid3_rotary(shape, at, k_at, rotary.turn, int(backward), at + 32, kout_at, _stream()), "rapid3_rotary")
    return q_out, k_out


def rapid3_norm_rotary(q: torch.Tensor, k: Optional[torch.Tensor], q_gain: torch.Tensor, k_gain: Optional[torch.Tensor], eps: float,
                       rotary: Rotary, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """RMS normalisation of each head, gain (fp32 [D]) and rotation in one pass; outputs may be the inputs."""
    what = "rapid3_norm_rotary"
    q_out = torch.empty_like(q) if q_out is None else q_out
    k_out = torch.empty_like(k) if k_out is None and k is not None else k_out
    shape, dev, rows, at = _heads(what, q, k, rotary, (("q_out", q_out),), (("k_out", k_out),))
    _check_vector(what, "q_gain", q_gain, shape.D, dev)
    k_at = kout_at = None
    if k is not None:
        _check_vector(what, "k_gain", k_gain, shape.D, dev)
        k_at, kout_at = at + 64, at + 96
    _check(load().by_address.rapid3_norm_rotary(shape, at, k_at, q_gain.data_ptr(), _ptr(k_gain), float(eps), rotary.turn, at + 32, kout_at, _stream()), what)
    return q_out, k_out


def rapid3_norm_rotary_backward(dq_out: torch.Tensor, dk_out: Optional[torch.Tensor], q: torch.Tensor, k: Optional[torch.Tensor],
                                q_gain: torch.Tensor, k_gain: Optional[torch.Tensor], eps: float, rotary: Rotary,
                                dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                                dq_gain: Optional[torch.Tensor] = None, dk_gain: Optional[torch.Tensor] = None):
    """Gradients of rapid3_norm_rotary's inputs and gains from those of its outputs; q and k are its inputs.
    dq and dk may be dq_out and dk_out.  The same call gives the same bits."""
    what = "rapid3_norm_rotary_backward"
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None and k is not None else dk
    dq_gain = torch.empty_like(q_gain) if dq_gain is None and q_gain is not None else dq_gain
    dk_gain = torch.empty_like(k_gain) if dk_gain is None and k is not None and k_gain is not None else dk_gain
    shape, dev, rows, at = _heads(what, q, k, rotary, (("dq_out", dq_out), ("dq", dq)), (("dk_out", dk_out), ("dk", dk)))
    for name, t in (("q_gain", q_gain), ("dq_gain", dq_gain)) + ((("k_gain", k_gain), ("dk_gain", dk_gain)) if k is not None else ()):
        _check_vector(what, name, t, shape.D, dev)
    lib = load()
    size = lib.rapid3_norm_rotary_workspace_bytes(shape)
    workspace = torch.empty(max(16, size), dtype=torch.uint8, device=q.device)
    k_at, dk_out_at, dk_at = (None, None, None) if k is None else (at + 96, at + 128, at + 160)
    _check(lib.by_address.rapid3_norm_rotary_backward(shape, at + 32, dk_out_at, at, k_at, _ptr(q_gain), _ptr(k_gain), float(eps), rotary.turn, at + 64, dk_at,
                                           _ptr(dq_gain), None if k is None else _ptr(dk_gain), _ptr(workspace), size, _stream()), what)
    return dq, dk, dq_gain, dk_gain


def _window(what: str, q: torch.Tensor, k: torch.Tensor, like_q, like_k, left: int, right: int, n_sink: int, n_full: int,
            q_len: Optional[torch.Tensor], kv_len: Optional[torch.Tensor], softmax_scale: Optional[float]):
    """The shape and rule of a windowed attention, after checking Q, K, the lengths and what is like Q and K, (name, tensor)s; the device; and
    _tensors() of q, like_q, k, like_k."""
    shape, k_shape, dtype, dev = q.shape, k.shape, q.dtype, _device(what, q)
    if len(shape) != 4 or len(k_shape) != 4 or (dtype is not torch.bfloat16 and dtype is not torch.float16):
        raise ValueError(f"{what}: q [B, H, n_q, D] and k [B, H_kv, n_kv, D] must be bf16 or fp16")
    B, H, n_q, D = shape
    Bk, Hk, n_kv, Dk = k_shape
    if Bk != B or Dk != D:
        raise ValueError(f"{what}: q and k must agree in B and D")
    rows, at = _tensors(what, dtype, dev, [("q", q, shape)] + [(name, t, shape) for name, t in like_q] + [("k", k, k_shape)] +
                         [(name, t, k_shape) for name, t in like_k])
    if q_len is not None:
        _check_vector(what, "q_len", q_len, B, dev, torch.int32)
    if kv_len is not None:
        _check_vector(what, "kv_len", kv_len, B, dev, torch.int32)
    return Window(_TYPES[dtype], B, H, Hk, D, n_q, n_kv, int(left), int(right), int(n_sink), int(n_full),
                  float(softmax_scale if softmax_scale is not None else D ** -0.5), _ptr(q_len), _ptr(kv_len)), dev, rows, at


def _check_lse(what: str, lse: Optional[torch.Tensor], q: torch.Tensor, dev: int):
    if lse is None or lse.dtype is not torch.float32 or lse.get_device() != dev or lse.shape != q.shape[:3] or not lse.is_contiguous():
        raise ValueError(f"{what}: lse must be contiguous fp32 {tuple(q.shape[:3])} on CUDA device {dev}")


def rapid3_window_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                       left: int = -1, right: int = -1, n_sink: int = 0, n_full: int = 0, q_len: Optional[torch.Tensor] = None,
                       kv_len: Optional[torch.Tensor] = None, softmax_scale: Optional[float] = None):
    """Attention of q [B, H, n_q, D] over k, v [B, H_kv, n_kv, D]: row i, at position p = i + kv_len - q_len, sees key j if j <= p + right and
    (j >= p - left or j < n_sink), or if 0 <= p < n_full; -1: no bound.  q_len, kv_len: int32 [B] on the GPU, read when the kernels run.
    Returns out (allocated, rows from q_len on unset, unless given) and lse (filled if given)."""
    what = "rapid3_window_attn"
    out = torch.empty_like(q) if out is None else out
    shape, dev, rows, at = _window(what, q, k, (("out", out),), (("v", v),), left, right, n_sink, n_full, q_len, kv_len, softmax_scale)
    if lse is not None:
        _check_lse(what, lse, q, dev)
    _check(load().by_address.rapid3_window_attn(shape, at, at + 64, at + 96, at + 32, _ptr(lse), _stream()), what)
    return out, lse


def rapid3_window_attn_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor,
                                dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None, dv: Optional[torch.Tensor] = None,
                                left: int = -1, right: int = -1, n_sink: int = 0, n_full: int = 0, q_len: Optional[torch.Tensor] = None,
                                kv_len: Optional[torch.Tensor] = None, softmax_scale: Optional[float] = None):
    """Gradients of rapid3_window_attn from dout and what that call read and wrote, with the same rule, lengths and scale.
    Rows from q_len and keys from kv_len on are left as they were.  The same call gives the same bits."""
    what = "rapid3_window_attn_backward"
    dq, dk, dv = (torch.empty_like(x) if g is None else g for x, g in ((q, dq), (k, dk), (v, dv)))
    shape, dev, rows, at = _window(what, q, k, (("out", out), ("dout", dout), ("dq", dq)), (("v", v), ("dk", dk), ("dv", dv)), left, right, n_sink,
                                    n_full, q_len, kv_len, softmax_scale)
    _check_lse(what, lse, q, dev)
    lib = load()
    size = lib.rapid3_window_workspace_bytes(shape)
    workspace = torch.empty(max(16, size), dtype=torch.uint8, device=q.device)
    _check(lib.by_address.rapid3_window_attn_backward(shape, at, at + 128, at + 160, at + 32, _ptr(lse), at + 64, at + 96, at + 192, at + 224, _ptr(workspace),
                                           size, _stream()), what)
    return dq, dk, dv


def rapid3_window_status() -> int:
    """The current device's status word of the windowed attention, and clears it; synchronises the device."""
    v = ctypes.c_int(0)
    _check(load().rapid3_window_status(ctypes.byref(v)), "rapid3_window_status")
    return v.value


def static_scratch_bytes() -> int:
    return int(load().rapid3_static_scratch_bytes())


class _Raw:
    """Minimal __cuda_array_interface__ carrier so torch can view library-owned device memory."""

    def __init__(self, ptr, shape, typestr):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr, "data": (ptr, False), "version": 2}


def _view(ptr: int, shape, dtype, device):
    typestr = {torch.float32: "<f4", torch.int64: "<i8", torch.int32: "<i4"}[dtype]
    return torch.as_tensor(_Raw(ptr, shape, typestr), device=device)


def bitmask_to_dense(bitmask: torch.Tensor, nb: int) -> torch.Tensor:
    """[..., nb, words] int64 bitmask -> [..., nb, nb] uint8 (marshalling for tests and reports)."""
    bm = bitmask.cpu()
    j = torch.arange(nb)
    words = bm[..., (j // 64)]
    return ((words >> (j % 64)) & 1).to(torch.uint8)
