"""ctypes binding of librs3.so (argument marshalling only).

Tensors are torch tensors on the GPU (their data_ptr() is passed); host-side
arrays are numpy.  `stream=None` means torch's current stream.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

RS3_OK, RS3_E_INVALID, RS3_E_CAPACITY, RS3_E_DEVICE, RS3_E_OOM = 0, 1, 2, 3, 4
RS3_F32, RS3_BF16 = 0, 1
RS3_MAX_OBJ = 64
RS3_MAX_MN = 32768
RS3_TRACK_WORDS = 6
RS3_BANK_HDR_WORDS = 8
RS3_NOALLOC_SCRATCH_BYTES = 16 << 20
RS3_PAIRS_ADJACENT, RS3_PAIRS_HALVES = 0, 1

lib_path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librs3.so")

c_i32, c_i64, c_sz, c_vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p
P_i32 = ctypes.POINTER(ctypes.c_int32)


class Grid(ctypes.Structure):
    _fields_ = [("m", c_i32), ("n", c_i32), ("s", c_i32)]


class SelectParams(ctypes.Structure):
    _fields_ = [("r_s", c_i32), ("c", c_i32), ("seed_box", c_i32), ("union_objects", c_i32)]


class FrameIO(ctypes.Structure):
    """rs3_frame_io: the arguments of one frame (select, readout, commit)."""
    _fields_ = [("read_masks", c_vp), ("X", c_vp), ("x_obj_stride", c_i64), ("k", c_vp), ("params", SelectParams),
                ("sel_idx", c_vp), ("sel_count", c_vp), ("prior_out", c_vp), ("max_sel", c_i32),
                ("n_splits", c_i32), ("Y", c_vp), ("y_obj_stride", c_i64), ("y_fp32", c_i32), ("Kmem", c_vp),
                ("Vmem", c_vp), ("kv_obj_stride", c_i64), ("commit_masks", c_vp), ("t", c_i32), ("pin", c_i32),
                ("fall_min", c_i32), ("fall_max", c_i32), ("kept_count", c_vp)]


class StackWeights(ctypes.Structure):
    """rs3_stack_weights: one layer's host arrays (see rs3.h)."""
    _fields_ = [(n, c_vp) for n in ("ln1_g", "ln1_b", "Wqs", "Wks", "Wvs", "Wos", "ln2_g", "ln2_b", "Wq", "Wk",
                                    "Wv", "Wo", "ln3_g", "ln3_b", "W1", "W2")]


class BlockShape(ctypes.Structure):
    """rs3_block_shape: sizes and row layouts of the block-sparse attention
    (block_shape() fills in the strides of packed tensors)."""
    _fields_ = [(n, c_i32) for n in ("n_obj", "n_q", "n_kv", "H", "H_kv", "d_h", "block", "top_k", "n_first",
                                     "n_last", "dt", "reserved")] + \
               [(n, c_i64) for n in ("q_stride", "q_obj_stride", "k_stride", "k_obj_stride", "v_stride",
                                     "v_obj_stride", "o_stride", "o_obj_stride")]


class Rs3Error(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (what, _status_str(status), status))


_SIGS = {
    "rs3_status_str": (ctypes.c_char_p, [c_i32]),
    "rs3_track_create": (c_i32, [c_i32, ctypes.POINTER(c_vp)]),
    "rs3_track_destroy": (None, [c_vp]),
    "rs3_track_export": (c_i32, [c_vp, c_vp]),
    "rs3_track_import": (c_i32, [c_vp, c_vp]),
    "rs3_layer_create": (c_i32, [c_i32, c_i32, c_i32, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, ctypes.POINTER(c_vp)]),
    "rs3_layer_destroy": (None, [c_vp]),
    "rs3_layer_set_rope": (c_i32, [c_vp, c_i32, c_i32, c_vp]),
    "rs3_layer_set_rope_axial": (c_i32, [c_vp, c_i32, c_i32, ctypes.c_double]),
    "rs3_bank_create": (c_i32, [c_vp, c_i32, c_i32, c_i32, ctypes.POINTER(c_vp)]),
    "rs3_bank_destroy": (None, [c_vp]),
    "rs3_bank_export": (c_i32, [c_vp, c_vp, c_vp, c_vp, c_vp, c_vp]),
    "rs3_bank_import": (c_i32, [c_vp, c_vp, c_vp, c_vp, c_vp, c_vp]),
    "rs3_attend_workspace_size": (c_i32, [c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, ctypes.POINTER(c_sz)]),
    "rs3_attend": (c_i32, [c_vp, c_vp, c_vp, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_vp, c_vp, c_sz, c_vp]),
    "rs3_bank_error": (c_i32, [c_vp, c_vp, c_i32]),
    "rs3_select_workspace_size": (c_i32, [ctypes.POINTER(Grid), c_i32, c_i64, ctypes.POINTER(c_sz)]),
    "rs3_select_queries": (c_i32, [ctypes.POINTER(Grid), c_i32, c_vp, c_vp, c_vp, c_i64, c_i32, c_i32, c_vp,
                                   ctypes.POINTER(SelectParams), c_vp, c_sz, c_vp, c_vp, c_vp, c_vp]),
    "rs3_readout_workspace_size": (c_i32, [c_vp, c_i32, c_i32, c_i32, ctypes.POINTER(c_sz)]),
    "rs3_readout": (c_i32, [c_vp, ctypes.POINTER(Grid), c_i32, c_vp, c_i64, c_vp, c_vp, c_vp, c_i32, c_i32,
                            c_i32, c_vp, c_i64, c_i32, c_vp, c_sz, c_vp]),
    "rs3_readout_noalloc": (c_i32, [c_vp, ctypes.POINTER(Grid), c_i32, c_vp, c_i64, c_vp, c_vp, c_vp, c_i32, c_i32,
                                    c_i32, c_vp, c_i64, c_i32, c_vp]),
    "rs3_readout_commit": (c_i32, [c_vp, ctypes.POINTER(Grid), c_i32, c_vp, c_i64, c_vp, c_vp, c_vp, c_i32, c_i32,
                                   c_i32, c_vp, c_i64, c_i32, c_vp, c_sz, c_vp, c_vp, c_i64, c_vp, c_i32, c_i32,
                                   c_i32, c_i32, c_vp, c_vp]),
    "rs3_commit": (c_i32, [c_vp, c_i32, ctypes.POINTER(Grid), c_vp, c_vp, c_i64, c_vp, c_i32, c_i32, c_i32,
                           c_i32, c_vp, c_vp]),
    "rs3_frame_workspace_size": (c_i32, [c_vp, ctypes.POINTER(Grid), c_i32, c_i64, c_i32, c_i32,
                                         ctypes.POINTER(c_sz)]),
    "rs3_frame": (c_i32, [c_vp, ctypes.POINTER(Grid), c_i32, c_vp, c_vp, ctypes.POINTER(FrameIO), c_vp, c_sz, c_vp]),
    "rs3_write_keepset": (c_i32, [ctypes.POINTER(Grid), c_i32, c_vp, c_i32, c_i32, c_i32, c_i32, c_vp, c_vp, c_vp]),
    "rs3_close_workspace_size": (c_i32, [c_i32, c_i32, c_i32, ctypes.POINTER(c_sz)]),
    "rs3_close_masks": (c_i32, [c_i32, c_i32, c_i32, c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_sz, c_vp]),
    "rs3_stack_create": (c_i32, [c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, ctypes.POINTER(StackWeights),
                                 ctypes.POINTER(c_vp)]),
    "rs3_stack_destroy": (None, [c_vp]),
    "rs3_stack_workspace_size": (c_i32, [c_vp, c_i32, c_i32, ctypes.POINTER(c_sz)]),
    "rs3_stack_readout": (c_i32, [c_vp, ctypes.POINTER(Grid), c_vp, c_vp, c_vp, c_vp, c_i32, c_i32, c_vp, c_i32,
                                  c_vp, c_sz, c_vp]),
    "rs3_qk_norm_rope": (c_i32, [c_i32, c_vp, c_i64, c_i32, c_vp, c_i64, c_i32, c_i32, c_i32, c_vp, c_vp,
                                 ctypes.c_float, c_vp, c_i32, c_i32, c_i32, c_vp, c_vp, c_i64, c_vp, c_i64, c_vp]),
    "rs3_block_means": (c_i32, [ctypes.POINTER(BlockShape), c_vp, c_vp, c_i32, c_vp, c_vp]),
    "rs3_block_select_workspace_size": (c_i32, [ctypes.POINTER(BlockShape), ctypes.POINTER(c_sz)]),
    "rs3_block_select": (c_i32, [ctypes.POINTER(BlockShape), c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]),
    "rs3_block_attend_workspace_size": (c_i32, [ctypes.POINTER(BlockShape), ctypes.POINTER(c_sz)]),
    "rs3_block_attend": (c_i32, [ctypes.POINTER(BlockShape), c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz,
                                 c_vp]),
    "rs3_profile_enable": (c_i32, [c_i32, c_i32]),
    "rs3_profile_report_n": (c_i32, [c_i32, c_vp, c_vp, c_vp]),
    "rs3_profile_report": (c_i32, [c_vp, c_vp, c_vp]),
    "rs3_profile_reset": (c_i32, []),
    "rs3_stream_read": (c_i32, [c_vp, c_sz, c_vp, c_vp]),
}

RS3_STREAM_READ_THREADS = 1024 * 256

KERNEL_NAMES = ["energy", "select", "commit", "commit_append", "copy", "qproj", "attn", "combine",
                "readout_f32", "merge_commit", "stack_gemm", "stack_merge", "stack_mlp", "stack_rows", "qk_norm",
                "block_means", "block_select", "block_attend"]

_lib = None


def lib():
    """Load librs3.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(lib_path):
            raise RuntimeError("librs3.so is not built; run `python -m paper_2608_22526_amd.build`")
        L = ctypes.CDLL(lib_path)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def exported_symbols():
    return list(_SIGS)


def _status_str(s: int) -> str:
    try:
        return lib().rs3_status_str(int(s)).decode()
    except Exception:  # library not loadable
        return "status"


def _check(status: int, what: str):
    if status != RS3_OK:
        raise Rs3Error(status, what)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream
    import torch
    return torch.cuda.current_stream().cuda_stream


# ---------------------------------------------------------------------------
class Track:
    """rs3_track: per-object (box, streak, has_box) state."""

    def __init__(self, n_obj: int):
        h = c_vp()
        _check(lib().rs3_track_create(n_obj, ctypes.byref(h)), "rs3_track_create")
        self.h, self.n_obj = h, n_obj

    def export(self) -> np.ndarray:
        out = np.zeros((self.n_obj, RS3_TRACK_WORDS), np.int32)
        _check(lib().rs3_track_export(self.h, out.ctypes.data), "rs3_track_export")
        return out

    def import_(self, state: np.ndarray):
        st = np.ascontiguousarray(state, dtype=np.int32)
        _check(lib().rs3_track_import(self.h, st.ctypes.data), "rs3_track_import")

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            _lib.rs3_track_destroy(self.h)
            self.h = None


class Layer:
    """rs3_layer: W_q [C][D], W_k/W_v [d_kv][D], W_o [D][C] host arrays
    (uint16 bf16 bits or float32).  absorb=True runs the single-head
    attention on the raw bank rows (see rs3.h)."""

    def __init__(self, C: int, H: int, d_kv: int, dtype: int, Wq, Wk, Wv, Wo, absorb: bool = False):
        arrs = [np.ascontiguousarray(w) for w in (Wq, Wk, Wv, Wo)]
        h = c_vp()
        _check(lib().rs3_layer_create(C, H, d_kv, dtype, int(absorb), *(a.ctypes.data for a in arrs),
                                      ctypes.byref(h)), "rs3_layer_create")
        self.h, self.C, self.H, self.d_kv, self.dtype, self.absorb = h, C, H, d_kv, dtype, bool(absorb)

    def set_rope(self, m: int, n: int, table=None):
        """Attach a rotary table: float32 host array [m*n][d_h/2][2] of
        (cos, sin) pairs; table=None with m = n = 0 removes it."""
        t = None if table is None else np.ascontiguousarray(table, dtype=np.float32)
        _check(lib().rs3_layer_set_rope(self.h, m, n, None if t is None else t.ctypes.data), "rs3_layer_set_rope")

    def set_rope_axial(self, m: int, n: int, theta: float):
        """Attach the axial rotary table built on the device."""
        _check(lib().rs3_layer_set_rope_axial(self.h, m, n, float(theta)), "rs3_layer_set_rope_axial")

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            _lib.rs3_layer_destroy(self.h)
            self.h = None


class Bank:
    """rs3_bank: one object's ring bank for `layer`."""

    def __init__(self, layer: Layer, cap: int, f_max: int, n_pin: int):
        h = c_vp()
        _check(lib().rs3_bank_create(layer.h, cap, f_max, n_pin, ctypes.byref(h)), "rs3_bank_create")
        self.h, self.layer, self.cap, self.f_max, self.n_pin = h, layer, cap, f_max, n_pin

    def export(self):
        es = 2 if self.layer.dtype == RS3_BF16 else 4
        npdt = np.uint16 if es == 2 else np.float32
        hdr = np.zeros(RS3_BANK_HDR_WORDS, np.int32)
        frames = np.zeros((self.f_max, 4), np.int32)
        K = np.zeros((self.cap, self.layer.d_kv), npdt)
        V = np.zeros((self.cap, self.layer.d_kv), npdt)
        pos = np.zeros(self.cap, np.int32)
        _check(lib().rs3_bank_export(self.h, hdr.ctypes.data, frames.ctypes.data, K.ctypes.data,
                                     V.ctypes.data, pos.ctypes.data), "rs3_bank_export")
        nf, nk = int(hdr[0]), int(hdr[3])
        return dict(hdr=hdr, n_frames=nf, pin_end=int(hdr[1]), err=int(hdr[2]), n_keys=nk,
                    frames=frames[:nf].copy(), K=K[:nk].copy(), V=V[:nk].copy(), pos=pos[:nk].copy())

    def import_snapshot(self, snap: dict):
        """Restore from a dict in the format of export() (synchronises)."""
        es = 2 if self.layer.dtype == RS3_BF16 else 4
        npdt = np.uint16 if es == 2 else np.float32
        hdr = np.ascontiguousarray(snap["hdr"], dtype=np.int32)
        frames = np.ascontiguousarray(snap["frames"], dtype=np.int32).reshape(-1, 4)
        K = np.ascontiguousarray(snap["K"], dtype=npdt)
        V = np.ascontiguousarray(snap["V"], dtype=npdt)
        pos = np.ascontiguousarray(snap["pos"], dtype=np.int32)
        _check(lib().rs3_bank_import(self.h, hdr.ctypes.data, frames.ctypes.data, K.ctypes.data, V.ctypes.data,
                                     pos.ctypes.data), "rs3_bank_import")

    def info(self) -> dict:
        """Header only (n_frames, pin_end, err, n_keys); synchronises."""
        hdr = np.zeros(RS3_BANK_HDR_WORDS, np.int32)
        _check(lib().rs3_bank_export(self.h, hdr.ctypes.data, None, None, None, None), "rs3_bank_export")
        return dict(n_frames=int(hdr[0]), pin_end=int(hdr[1]), err=int(hdr[2]), n_keys=int(hdr[3]))

    def error(self, clear: bool = False) -> int:
        e = np.zeros(1, np.int32)
        _check(lib().rs3_bank_error(self.h, e.ctypes.data, int(clear)), "rs3_bank_error")
        return int(e[0])

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            _lib.rs3_bank_destroy(self.h)
            self.h = None


def _grid(g) -> Grid:
    if isinstance(g, Grid):
        return g
    m, n, s = g
    return Grid(m, n, s)


def select_workspace_size(grid, n_obj: int, x_obj_stride: int) -> int:
    out = c_sz()
    _check(lib().rs3_select_workspace_size(ctypes.byref(_grid(grid)), n_obj, x_obj_stride, ctypes.byref(out)),
           "rs3_select_workspace_size")
    return out.value


def select_queries(grid, n_obj: int, masks, track: Track, X, x_obj_stride: int, C: int, dtype: int,
                   k: Sequence[int], params: SelectParams, ws, sel_idx, sel_count, prior_out=None,
                   stream=None):
    karr = np.ascontiguousarray(np.asarray(k, dtype=np.int32))
    _check(lib().rs3_select_queries(ctypes.byref(_grid(grid)), n_obj, _ptr(masks), track.h, _ptr(X),
                                    x_obj_stride, C, dtype, karr.ctypes.data, ctypes.byref(params), _ptr(ws),
                                    ws.numel() * ws.element_size(), _ptr(sel_idx), _ptr(sel_count),
                                    _ptr(prior_out), _stream(stream)), "rs3_select_queries")


def readout_workspace_size(layer: Layer, n_obj: int, max_sel: int, n_splits: int = 0) -> int:
    out = c_sz()
    _check(lib().rs3_readout_workspace_size(layer.h, n_obj, max_sel, n_splits, ctypes.byref(out)),
           "rs3_readout_workspace_size")
    return out.value


def readout(layer: Layer, grid, n_obj: int, X, x_obj_stride: int, banks: Sequence[Bank], sel_idx, sel_count,
            sel_stride: int, max_sel: int, n_splits: int, Y, y_obj_stride: int, y_fp32: int = 0, ws=None,
            stream=None):
    harr = (c_vp * len(banks))(*[b.h for b in banks])
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().rs3_readout(layer.h, ctypes.byref(_grid(grid)), n_obj, _ptr(X), x_obj_stride,
                             ctypes.cast(harr, c_vp), _ptr(sel_idx), _ptr(sel_count), sel_stride, max_sel,
                             n_splits, _ptr(Y), y_obj_stride, y_fp32, _ptr(ws), ws_bytes, _stream(stream)),
           "rs3_readout")


def readout_noalloc(layer: Layer, grid, n_obj: int, X, x_obj_stride: int, banks: Sequence[Bank], sel_idx, sel_count,
                    sel_stride: int, max_sel: int, n_splits: int, Y, y_obj_stride: int, y_fp32: int = 0, stream=None):
    """rs3_readout without a workspace: the library's fixed per-GPU scratch
    holds the split partials (nothing is allocated)."""
    harr = (c_vp * len(banks))(*[b.h for b in banks])
    _check(lib().rs3_readout_noalloc(layer.h, ctypes.byref(_grid(grid)), n_obj, _ptr(X), x_obj_stride,
                                     ctypes.cast(harr, c_vp), _ptr(sel_idx), _ptr(sel_count), sel_stride, max_sel,
                                     n_splits, _ptr(Y), y_obj_stride, y_fp32, _stream(stream)), "rs3_readout_noalloc")


def commit(banks: Sequence[Bank], grid, Kmem, Vmem, kv_obj_stride: int, masks, t: int, pin: int,
           fall_min: int, fall_max: int, kept_count=None, stream=None):
    harr = (c_vp * len(banks))(*[b.h for b in banks])
    _check(lib().rs3_commit(ctypes.cast(harr, c_vp), len(banks), ctypes.byref(_grid(grid)), _ptr(Kmem),
                            _ptr(Vmem), kv_obj_stride, _ptr(masks), t, pin, fall_min, fall_max,
                            _ptr(kept_count), _stream(stream)), "rs3_commit")


def readout_commit(layer: Layer, grid, n_obj: int, X, x_obj_stride: int, banks: Sequence[Bank], sel_idx, sel_count,
                   sel_stride: int, max_sel: int, n_splits: int, Y, y_obj_stride: int, y_fp32: int, ws, Kmem, Vmem,
                   kv_obj_stride: int, masks, t: int, pin: int, fall_min: int, fall_max: int, kept_count=None,
                   stream=None):
    """rs3_readout followed by rs3_commit, merged into fewer launches."""
    harr = (c_vp * len(banks))(*[b.h for b in banks])
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().rs3_readout_commit(layer.h, ctypes.byref(_grid(grid)), n_obj, _ptr(X), x_obj_stride,
                                    ctypes.cast(harr, c_vp), _ptr(sel_idx), _ptr(sel_count), sel_stride, max_sel,
                                    n_splits, _ptr(Y), y_obj_stride, y_fp32, _ptr(ws), ws_bytes, _ptr(Kmem),
                                    _ptr(Vmem), kv_obj_stride, _ptr(masks), t, pin, fall_min, fall_max,
                                    _ptr(kept_count), _stream(stream)), "rs3_readout_commit")


def frame_workspace_size(layer: Layer, grid, n_obj: int, x_obj_stride: int, max_sel: int, n_splits: int = 0) -> int:
    out = c_sz()
    _check(lib().rs3_frame_workspace_size(layer.h, ctypes.byref(_grid(grid)), n_obj, x_obj_stride, max_sel, n_splits,
                                          ctypes.byref(out)), "rs3_frame_workspace_size")
    return out.value


def frame(layer: Layer, grid, n_obj: int, track: Track, banks: Sequence[Bank], io: FrameIO, ws, stream=None):
    """One frame: rs3_select_queries then rs3_readout_commit in one call
    (`io` holds the arguments of both)."""
    harr = (c_vp * len(banks))(*[b.h for b in banks])
    _check(lib().rs3_frame(layer.h, ctypes.byref(_grid(grid)), n_obj, track.h, ctypes.cast(harr, c_vp),
                           ctypes.byref(io), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)), "rs3_frame")


def write_keepset(grid, n_obj: int, seed_masks, D_w: int, fall_min: int, fall_max: int, n_copies: int, keep,
                  counts=None, stream=None):
    """The fixed write keep-set K_w (u8 [n_copies][m*n]) from the seed masks."""
    _check(lib().rs3_write_keepset(ctypes.byref(_grid(grid)), n_obj, _ptr(seed_masks), D_w, fall_min, fall_max,
                                   n_copies, _ptr(keep), _ptr(counts), _stream(stream)), "rs3_write_keepset")


def close_workspace_size(n_obj: int, H: int, W: int) -> int:
    out = c_sz()
    _check(lib().rs3_close_workspace_size(n_obj, H, W, ctypes.byref(out)), "rs3_close_workspace_size")
    return out.value


def close_masks(n_obj: int, H: int, W: int, logits, dtype: int, k: int, closed=None, palette=None, ws=None,
                stream=None):
    """k x k closure of each object's decoded mask and the palette argmax."""
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().rs3_close_masks(n_obj, H, W, _ptr(logits), dtype, k, _ptr(closed), _ptr(palette), _ptr(ws),
                                 ws_bytes, _stream(stream)), "rs3_close_masks")


def attend_workspace_size(n_q: int, n_kv: int, H: int, d_h: int, dtype: int, n_splits: int = 0) -> int:
    out = c_sz()
    _check(lib().rs3_attend_workspace_size(n_q, n_kv, H, d_h, dtype, n_splits, ctypes.byref(out)),
           "rs3_attend_workspace_size")
    return out.value


def attend(Q, K, V, n_q: int, n_kv: int, H: int, d_h: int, dtype: int, O, ws=None, n_splits: int = 0,
           stream=None):
    """Bare attention core: O [n_q][H*d_h] fp32 from projected Q, K, V."""
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().rs3_attend(_ptr(Q), _ptr(K), _ptr(V), n_q, n_kv, H, d_h, dtype, n_splits, _ptr(O), _ptr(ws),
                            ws_bytes, _stream(stream)), "rs3_attend")


# ---- norm, rotation and block-sparse attention --------------------------------
def _check_tensor(name: str, t, numel: int, dtype, device):
    """Refuses a tensor that the kernels would read or write past, or that
    lies elsewhere than the call's other tensors."""
    if t.numel() < numel or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError("%s: %s of %s on %s%s, need %d contiguous elements of %s on %s"
                         % (name, tuple(t.shape), t.dtype, t.device, "" if t.is_contiguous() else " (strided)", numel,
                            dtype, device))


def _check_rows(name: str, t, last: int, dtype, device):
    """As _check_tensor for a tensor addressed by strides of its own: `last`
    elements must follow data_ptr() in its storage."""
    room = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
    if room < last or t.dtype != dtype or t.device != device:
        raise ValueError("%s: %d elements of %s on %s, need %d of %s on %s"
                         % (name, room, t.dtype, t.device, last, dtype, device))


def _call():
    """The current device and its current stream's handle."""
    import torch
    C = torch._C
    dev = C._cuda_getDevice()
    return torch, dev, C._cuda_getCurrentRawStream(dev)


def _tensor(torch, name: str, t, numel: int, dtype, dev: int):
    if t.numel() >= numel and t.dtype is dtype and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    _check_tensor(name, t, numel, dtype, torch.device("cuda", dev))
    return t.data_ptr()


def _rows(torch, name: str, t, last: int, dtype, dev: int):
    if not (t.numel() >= last and t.dtype is dtype and t.get_device() == dev and t.is_contiguous()):
        _check_rows(name, t, last, dtype, torch.device("cuda", dev))
    return t.data_ptr()


def _check_i32(*values: int):
    """ctypes would take them modulo 2^32."""
    for v in values:
        if not -2 ** 31 <= v < 2 ** 31:
            raise ValueError("%d is no 32-bit integer" % v)


def qk_norm_rope(n: int, Q, H: int, K, H_kv: int, d_h: int, dtype: int, Qo, Ko, gain_q=None, gain_k=None,
                 eps: float = 1e-6, table=None, d_rot: int = 0, pairing: int = RS3_PAIRS_ADJACENT, pos=None,
                 q_stride: Optional[int] = None, k_stride: Optional[int] = None, qo_stride: Optional[int] = None,
                 ko_stride: Optional[int] = None, stream=None):
    """RMS norm of each head of Q [n][H][d_h] and K [n][H_kv][d_h] (None with
    0 heads) and the rotation of its first d_rot channels by table[pos]."""
    if (n | H | H_kv | d_h | d_rot | pairing) >> 31:
        _check_i32(n, H, H_kv, d_h, d_rot, pairing)
    torch, dev, st = _call()
    dt, f32 = torch.bfloat16 if dtype == RS3_BF16 else torch.float32, torch.float32
    wq, wk = H * d_h, H_kv * d_h
    qs, ks = wq if q_stride is None else q_stride, wk if k_stride is None else k_stride
    qos, kos = wq if qo_stride is None else qo_stride, wk if ko_stride is None else ko_stride
    q = k = qo = ko = gq = gk = tab = ps = None
    n_pos = 0
    if n > 0 and wq > 0:
        if Q is not None:
            q = _rows(torch, "Q", Q, (n - 1) * qs + wq, dt, dev)
        if Qo is not None:
            qo = _rows(torch, "Qo", Qo, (n - 1) * qos + wq, dt, dev)
    if n > 0 and wk > 0:
        if K is not None:
            k = _rows(torch, "K", K, (n - 1) * ks + wk, dt, dev)
        if Ko is not None:
            ko = _rows(torch, "Ko", Ko, (n - 1) * kos + wk, dt, dev)
    if gain_q is not None:
        gq = _tensor(torch, "gain_q", gain_q, d_h, f32, dev)
    if gain_k is not None:
        gk = _tensor(torch, "gain_k", gain_k, d_h, f32, dev)
    if table is not None:
        n_pos = table.shape[0]
        tab = _tensor(torch, "table", table, n_pos * d_rot, f32, dev)
    if pos is not None:
        ps = _tensor(torch, "pos", pos, n, torch.int32, dev)
    _check(lib().rs3_qk_norm_rope(n, q, qs, H, k, ks, H_kv, d_h, dtype, gq, gk, eps, tab, n_pos, d_rot, pairing, ps,
                                  qo, qos, ko, kos, st if stream is None else stream), "rs3_qk_norm_rope")


def block_shape(dtype: int, n_obj: int, n_q: int, n_kv: int, H: int, H_kv: int, d_h: int, block: int, top_k: int,
                n_first: int = 0, n_last: int = 0, **strides) -> BlockShape:
    """A BlockShape for packed tensors [n_obj][rows][heads][d_h]; strides
    (q_stride=, q_obj_stride=, ...) replace the packed ones."""
    _check_i32(n_obj, n_q, n_kv, H, H_kv, d_h, block, top_k, n_first, n_last)
    s = BlockShape(n_obj, n_q, n_kv, H, H_kv, d_h, block, top_k, n_first, n_last, dtype, 0)
    for x, rows, heads in (("q", n_q, H), ("k", n_kv, H_kv), ("v", n_kv, H_kv), ("o", n_q, H)):
        row = strides.pop(x + "_stride", heads * d_h)
        setattr(s, x + "_stride", row)
        setattr(s, x + "_obj_stride", strides.pop(x + "_obj_stride", rows * row))
    if strides:
        raise TypeError("block_shape: unknown %s" % ", ".join(strides))
    return s


def _span(n_obj: int, obj: int, rows: int, row: int, width: int) -> int:
    """Elements from the first to the last of strided rows."""
    return (n_obj - 1) * obj + (rows - 1) * row + width if rows > 0 and n_obj > 0 else 0


def _means(torch, s: BlockShape, Kmean, dt, dev: int):
    n_blk = (s.n_kv + s.block - 1) // s.block if s.block > 0 else 0
    return _tensor(torch, "Kmean", Kmean, s.n_obj * s.H_kv * n_blk * s.d_h, dt, dev)


def _shape_dtype(torch, s: BlockShape):
    return torch.bfloat16 if s.dt == RS3_BF16 else torch.float32


def block_means(shape: BlockShape, K, Kmean, kv_len=None, n_new: int = 0, stream=None):
    """Kmean [n_obj][H_kv][n_blk][d_h]: the mean key of every block of K, or
    (n_new > 0) of the blocks that hold each object's last n_new keys."""
    if n_new >> 31:
        _check_i32(n_new)
    torch, dev, st = _call()
    s, dt = shape, _shape_dtype(torch, shape)
    k = _rows(torch, "K", K, _span(s.n_obj, s.k_obj_stride, s.n_kv, s.k_stride, s.H_kv * s.d_h), dt, dev)
    m = _means(torch, s, Kmean, dt, dev)
    n = None if kv_len is None else _tensor(torch, "kv_len", kv_len, s.n_obj, torch.int32, dev)
    _check(lib().rs3_block_means(s, k, n, n_new, m, st if stream is None else stream), "rs3_block_means")


def block_select_workspace_size(shape: BlockShape) -> int:
    out = c_sz()
    _check(lib().rs3_block_select_workspace_size(ctypes.byref(shape), ctypes.byref(out)),
           "rs3_block_select_workspace_size")
    return out.value


def _lists(torch, s: BlockShape, idx, count, n_vis, dev: int):
    rows, i32 = s.n_obj * s.n_q, torch.int32
    lists = rows * s.H_kv
    return (_tensor(torch, "idx", idx, lists * s.top_k, i32, dev), _tensor(torch, "count", count, lists, i32, dev),
            None if n_vis is None else _tensor(torch, "n_vis", n_vis, rows, i32, dev))


def _workspace(ws, dev: int):
    if ws is None:
        return None, 0
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError("ws: on %s, need contiguous memory on cuda:%d" % (ws.device, dev))
    return ws.data_ptr(), ws.numel() * ws.element_size()


def block_select(shape: BlockShape, Q, Kmean, idx, count, n_vis=None, ws=None, stream=None):
    """Each query's blocks by the scores of their mean keys: idx int32
    [n_obj][n_q][H_kv][top_k] ascending (-1 past the count), count int32."""
    torch, dev, st = _call()
    s, dt = shape, _shape_dtype(torch, shape)
    q = _rows(torch, "Q", Q, _span(s.n_obj, s.q_obj_stride, s.n_q, s.q_stride, s.H * s.d_h), dt, dev)
    m = _means(torch, s, Kmean, dt, dev)
    i, c, v = _lists(torch, s, idx, count, n_vis, dev)
    p, nbytes = _workspace(ws, dev)
    _check(lib().rs3_block_select(s, q, m, v, i, c, p, nbytes, st if stream is None else stream), "rs3_block_select")


def block_attend_workspace_size(shape: BlockShape) -> int:
    out = c_sz()
    _check(lib().rs3_block_attend_workspace_size(ctypes.byref(shape), ctypes.byref(out)),
           "rs3_block_attend_workspace_size")
    return out.value


def block_attend(shape: BlockShape, Q, K, V, idx, count, O, n_vis=None, ws=None, stream=None):
    """Softmax attention of every query over the keys of its listed blocks."""
    torch, dev, st = _call()
    s, dt = shape, _shape_dtype(torch, shape)
    n_obj, n_q, n_kv, wq, wk = s.n_obj, s.n_q, s.n_kv, s.H * s.d_h, s.H_kv * s.d_h
    q = _rows(torch, "Q", Q, _span(n_obj, s.q_obj_stride, n_q, s.q_stride, wq), dt, dev)
    k = _rows(torch, "K", K, _span(n_obj, s.k_obj_stride, n_kv, s.k_stride, wk), dt, dev)
    v = _rows(torch, "V", V, _span(n_obj, s.v_obj_stride, n_kv, s.v_stride, wk), dt, dev)
    o = _rows(torch, "O", O, _span(n_obj, s.o_obj_stride, n_q, s.o_stride, wq), dt, dev)
    i, c, vis = _lists(torch, s, idx, count, n_vis, dev)
    p, nbytes = _workspace(ws, dev)
    _check(lib().rs3_block_attend(s, q, k, v, i, c, vis, o, p, nbytes, st if stream is None else stream),
           "rs3_block_attend")


class Stack:
    """rs3_stack: the L-layer memory-attention stack on the kept queries.
    layers: one dict per layer with the keys of StackWeights (matrices uint16
    bf16 bits, row-major input dimension first; norm gains/shifts float32)."""

    def __init__(self, layers: Sequence[dict], C: int = 256, H_s: int = 1, d_kv: int = 64, F: int = 2048,
                 dtype: int = RS3_BF16):
        keep = []
        arr = (StackWeights * len(layers))()
        for i, w in enumerate(layers):
            for name, _ in StackWeights._fields_:
                a = np.ascontiguousarray(w[name], dtype=np.float32 if name.startswith("ln") else np.uint16)
                keep.append(a)
                setattr(arr[i], name, a.ctypes.data)
        h = c_vp()
        _check(lib().rs3_stack_create(len(layers), C, H_s, d_kv, F, dtype, arr, ctypes.byref(h)), "rs3_stack_create")
        self.h, self.n_layers, self.C, self.H_s, self.d_kv, self.F = h, len(layers), C, H_s, d_kv, F

    def workspace_size(self, max_sel: int, n_splits: int = 0) -> int:
        out = c_sz()
        _check(lib().rs3_stack_workspace_size(self.h, max_sel, n_splits, ctypes.byref(out)),
               "rs3_stack_workspace_size")
        return out.value

    def readout(self, grid, X, bank: Bank, sel_idx, sel_count, max_sel: int, Y, y_fp32: int = 0, ws=None,
                n_splits: int = 0, stream=None):
        ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
        _check(lib().rs3_stack_readout(self.h, ctypes.byref(_grid(grid)), _ptr(X), bank.h, _ptr(sel_idx),
                                       _ptr(sel_count), max_sel, n_splits, _ptr(Y), y_fp32, _ptr(ws), ws_bytes,
                                       _stream(stream)), "rs3_stack_readout")

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            _lib.rs3_stack_destroy(self.h)
            self.h = None


def profile_enable(on: bool, max_launches: int = 65536):
    _check(lib().rs3_profile_enable(int(on), max_launches), "rs3_profile_enable")


def profile_reset():
    _check(lib().rs3_profile_reset(), "rs3_profile_reset")


def stream_read(src, nbytes: int, out, stream=None):
    """rs3_stream_read: reads nbytes of device memory at src once; out
    (RS3_STREAM_READ_THREADS uint32) receives one xor word per thread."""
    _check(lib().rs3_stream_read(_ptr(src), nbytes, _ptr(out), _stream(stream)), "rs3_stream_read")


def profile_report() -> dict:
    """{kernel name: (total ms, launches)} accumulated since the last reset."""
    n = len(KERNEL_NAMES)
    ms = np.zeros(n, np.float64)
    cnt = np.zeros(n, np.int64)
    dropped = np.zeros(1, np.int64)
    _check(lib().rs3_profile_report_n(n, ms.ctypes.data, cnt.ctypes.data, dropped.ctypes.data), "rs3_profile_report_n")
    out = {KERNEL_NAMES[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}
    out["_dropped"] = (0.0, int(dropped[0]))
    return out
