"""ctypes binding of libvmoba.so: same names as the C ABI in include/vmoba.h, argument
marshalling only.  PyTorch supplies device memory and the stream; every step of the path runs
in the library's HIP kernels.  There is no fallback: if the library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import os
import struct

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libvmoba.so")

VMOBA_OK = 0
VMOBA_ERR_INVALID_ARG, VMOBA_ERR_UNSUPPORTED, VMOBA_ERR_WORKSPACE = -1, -2, -3
VMOBA_ERR_CAPACITY, VMOBA_ERR_HIP = -4, -5
VMOBA_F32, VMOBA_BF16 = 0, 1
OP_SELECT, OP_ATTN_FWD, OP_ATTN_BWD = 1, 2, 3

EXPORTS = ["vmoba_layer_kind", "vmoba_partition_dims", "vmoba_workspace_bytes", "vmoba_status_string",
           "vmoba_partition", "vmoba_select", "vmoba_select_static", "vmoba_attn_fwd", "vmoba_attn_bwd",
           "vmoba_profile_events", "vmoba_probe_mfma", "vmoba_probe_atomic_rows",
           "vmoba_rope_freqs", "vmoba_rope", "vmoba_rmsnorm_workspace_bytes", "vmoba_rmsnorm_fwd", "vmoba_rmsnorm_bwd",
           "vmoba_key_ranges", "vmoba_dense_workspace_bytes", "vmoba_dense_fwd", "vmoba_dense_bwd"]


class vmoba_grid(C.Structure):
    _fields_ = [("T", C.c_int32), ("H", C.c_int32), ("W", C.c_int32),
                ("bt", C.c_int32), ("bh", C.c_int32), ("bw", C.c_int32), ("chunk", C.c_int64)]


class vmoba_tensor(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("dtype", C.c_int32),
                ("stride_b", C.c_int64), ("stride_s", C.c_int64), ("stride_h", C.c_int64)]


class vmoba_scores(C.Structure):
    _fields_ = [("softmax_scale", C.c_float), ("cap", C.c_float), ("slopes", C.c_void_p), ("key_lo", C.c_void_p), ("key_hi", C.c_void_p),
                ("q_pos", C.c_void_p), ("q_first", C.c_int64)]


class VmobaError(RuntimeError):
    def __init__(self, fn, code):
        self.code = code
        super().__init__(f"{fn} failed: {code} ({status_string(code)})")


_lib = None


def lib():
    """The loaded library.  Raises if libvmoba.so has not been built (python -m
    paper_2506_23858_amd.build, or __graft_entry__.build())."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -m paper_2506_23858_amd.build)")
    L = C.CDLL(LIB_PATH)
    P = C.c_void_p
    L.vmoba_layer_kind.argtypes = [C.c_int]
    L.vmoba_layer_kind.restype = C.c_int
    L.vmoba_partition_dims.argtypes = [C.POINTER(vmoba_grid), C.POINTER(C.c_int64), C.POINTER(C.c_int32)]
    L.vmoba_partition_dims.restype = C.c_int
    L.vmoba_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int, C.c_int32, C.c_int64, C.c_int]
    L.vmoba_workspace_bytes.restype = C.c_size_t
    L.vmoba_status_string.argtypes = [C.c_int]
    L.vmoba_status_string.restype = C.c_char_p
    # (tensor descriptors: pointers to vmoba_tensor, as bytes or ctypes objects)
    L.vmoba_partition.argtypes = [C.POINTER(vmoba_grid), C.c_int, C.c_int, C.c_int, C.c_int, C.c_int,
                                  P, P, P, P, P, P]
    L.vmoba_partition.restype = C.c_int
    L.vmoba_select.argtypes = [C.c_int, C.c_int, C.c_int64, C.c_int, C.c_int32, P,
                               P, P, C.c_float, C.c_float, C.c_int,
                               C.c_int32, P, P, P, P, P, P, P, P, C.c_int64, P, P, P, P, P, P, C.c_size_t, P]
    L.vmoba_select.restype = C.c_int
    L.vmoba_select_static.argtypes = L.vmoba_select.argtypes[:-3] + [P]      # no workspace pointer / size
    L.vmoba_select_static.restype = C.c_int
    L.vmoba_attn_fwd.argtypes = [C.c_int, C.c_int, C.c_int64, C.c_int, C.c_int32, P,
                                 P, P, P,
                                 P, P, P, P, C.c_int64, C.c_float, P, P, P, P, P, C.c_size_t, P]
    L.vmoba_attn_fwd.restype = C.c_int
    L.vmoba_attn_bwd.argtypes = [C.c_int, C.c_int, C.c_int64, C.c_int, C.c_int32, P,
                                 P, P, P,
                                 P, P, P,
                                 P, P, P, P, C.c_int64, C.c_float,
                                 P, P, P,
                                 P, P, P, P, C.c_size_t, P]
    L.vmoba_attn_bwd.restype = C.c_int
    L.vmoba_profile_events.argtypes = [C.c_int, P, P]
    L.vmoba_profile_events.restype = C.c_int
    L.vmoba_probe_mfma.argtypes = [C.c_int64, C.c_int, P, C.POINTER(C.c_double), P]
    L.vmoba_probe_mfma.restype = C.c_int
    L.vmoba_probe_atomic_rows.argtypes = [P, P, C.c_int, C.c_int, C.c_int64, C.c_int, C.c_int, P]
    L.vmoba_probe_atomic_rows.restype = C.c_int
    L.vmoba_rope_freqs.argtypes = [C.c_int, C.POINTER(C.c_int32), C.c_double, C.c_int, C.c_double, C.c_int64, P, C.POINTER(C.c_float)]
    L.vmoba_rope_freqs.restype = C.c_int
    L.vmoba_rope.argtypes = [C.c_int, C.c_int64, C.c_int, C.c_int, C.POINTER(C.c_int32), P, P, P, C.c_int, C.POINTER(C.c_int32), C.c_int, C.c_int, C.c_float,
                             C.POINTER(vmoba_grid), C.c_int64, P, C.c_int64, P]
    L.vmoba_rope.restype = C.c_int
    L.vmoba_rmsnorm_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int64, C.c_int]
    L.vmoba_rmsnorm_workspace_bytes.restype = C.c_size_t
    L.vmoba_rmsnorm_fwd.argtypes = [C.c_int, C.c_int, C.c_int64, C.c_int, P, P, P, C.c_int, C.c_float, P, P, P, P, P]
    L.vmoba_rmsnorm_fwd.restype = C.c_int
    L.vmoba_rmsnorm_bwd.argtypes = [C.c_int, C.c_int, C.c_int64, C.c_int, P, P, C.c_int, P, P, P, P, P, P, C.c_size_t, P]
    L.vmoba_rmsnorm_bwd.restype = C.c_int
    L.vmoba_key_ranges.argtypes = [C.c_int, C.c_int64, C.c_int64, P, C.c_int64, C.c_int32, P, C.c_int64, C.c_int, P, C.c_int64, P, P, P]
    L.vmoba_key_ranges.restype = C.c_int
    L.vmoba_dense_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int64, C.c_int, C.c_int]
    L.vmoba_dense_workspace_bytes.restype = C.c_size_t
    L.vmoba_dense_fwd.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int64, C.c_int, P, P, P, C.POINTER(vmoba_scores), P, P, P, C.c_size_t, P]
    L.vmoba_dense_fwd.restype = C.c_int
    L.vmoba_dense_bwd.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int64, C.c_int, P, P, P, C.POINTER(vmoba_scores), P, P, P, P, P, P, P, C.c_size_t, P]
    L.vmoba_dense_bwd.restype = C.c_int
    _lib = L
    return L


def status_string(code: int) -> str:
    return lib().vmoba_status_string(int(code)).decode()


def _check(fn, rc):
    if rc != VMOBA_OK:
        raise VmobaError(fn, rc)


_DTYPE_CODES = {torch.float32: VMOBA_F32, torch.bfloat16: VMOBA_BF16}


# A short call is bound by the host: a training step with every tensor in block order describes 30 tensors and passes 50 pointers beside
# its 15 launches.  So a tensor is asked once for its strides, its descriptor is packed as bytes (1.1 -> 0.7 us against a ctypes structure), addresses are
# plain integers, which the argument types turn into pointers, and the current stream is asked for as a number, not as an
# object.  2 heads x 512 tokens x 64, float32, forward and backward: 104 -> 85 us (host alone 108 -> 80, half of it the launches).
def _dtype_code(t: torch.Tensor) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


_pack_desc = struct.Struct("Pi4xqqq").pack        # the fields of vmoba_tensor
assert struct.calcsize("Pi4xqqq") == C.sizeof(vmoba_tensor)


def _desc(t: torch.Tensor) -> bytes:
    """Descriptor of a 4-D tensor indexed (b, s, h, d) -- any strides with d contiguous -- as the bytes of a vmoba_tensor."""
    strides = t.stride()
    assert len(strides) == 4 and strides[3] == 1, "expect a (b, s, h, d) view with contiguous d"
    code = _DTYPE_CODES.get(t.dtype)
    return _pack_desc(t.data_ptr(), _dtype_code(t) if code is None else code, strides[0], strides[1], strides[2])


def tensor_desc(t: torch.Tensor) -> vmoba_tensor:
    """The same as a ctypes structure, for programs that call the library themselves."""
    return vmoba_tensor.from_buffer_copy(_desc(t))


def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(_device()) if _raw_stream and _device else torch.cuda.current_stream().cuda_stream


def make_grid(T, H, W, bt=0, bh=0, bw=0, chunk=0) -> vmoba_grid:
    return vmoba_grid(T, H, W, bt, bh, bw, chunk)


# ------------------------------------------------------------------------------- host helpers
def vmoba_layer_kind(layer: int) -> int:
    return lib().vmoba_layer_kind(int(layer))


def vmoba_partition_dims(g: vmoba_grid):
    S, nb = C.c_int64(0), C.c_int32(0)
    _check("vmoba_partition_dims", lib().vmoba_partition_dims(C.byref(g), C.byref(S), C.byref(nb)))
    return S.value, nb.value


def vmoba_workspace_bytes(op, B, Hh, S, D, n_blocks, nnz_capacity, dtype) -> int:
    return lib().vmoba_workspace_bytes(op, B, Hh, S, D, n_blocks, nnz_capacity, dtype)


def nnz_capacity_for(S: int, n_blocks: int, tau: float) -> int:
    """Per-head list capacity (buffer sizing only): in exact arithmetic the selection keeps at most
    ceil(tau * S * N_b) pairs.  tau is taken as the float32 the library receives, and a margin covers
    the float32 rounding of P (rows sum to 1 within ~1e-6, so the pool can fall short of S by that
    fraction and the cut move by as much)."""
    n = S * n_blocks
    tau32 = struct.unpack("f", struct.pack("f", float(tau)))[0]
    return max(1, min(n, math.ceil(tau32 * n * (1.0 + 2.0 ** -18)) + 16))


def vmoba_profile_events(slot: int, start_event=None, stop_event=None):
    """start_event / stop_event: raw hipEvent_t handles (ints) or None."""
    _check("vmoba_profile_events", lib().vmoba_profile_events(
        int(slot), C.c_void_p(start_event) if start_event else None,
        C.c_void_p(stop_event) if stop_event else None))


def vmoba_probe_mfma(iters: int, workgroups: int, sink, stream=None) -> float:
    """Launches the matrix-rate probe; returns the FLOP count of the launch (time it with events)."""
    flop = C.c_double(0.0)
    _check("vmoba_probe_mfma", lib().vmoba_probe_mfma(int(iters), int(workgroups), _ptr(sink), C.byref(flop), _stream(stream)))
    return flop.value


def vmoba_probe_atomic_rows(dq, lists, cnt, S, runs, heads, stream=None):
    """dq: float32 [heads, S, 128] (zeroed); lists: int32 [n_lists, cnt] ascending rows."""
    _check("vmoba_probe_atomic_rows", lib().vmoba_probe_atomic_rows(_ptr(dq), _ptr(lists), int(lists.shape[0]), int(cnt),
                                                                     int(S), int(runs), int(heads), _stream(stream)))


# ------------------------------------------------------------------------------- entry points
def vmoba_partition(g, inverse, B, Hh, D, ins, outs, perm, inv_perm, blk_off, stream=None):
    """ins / outs: lists of (b, s, h, d) views."""
    n = len(ins)
    assert len(outs) == n
    rc = lib().vmoba_partition(C.byref(g), int(inverse), B, Hh, D, n, b"".join(map(_desc, ins)), b"".join(map(_desc, outs)),
                               _ptr(perm), _ptr(inv_perm), _ptr(blk_off), _stream(stream))
    _check("vmoba_partition", rc)


GLOBAL_THRESHOLD, LOCAL_TOPK, LOCAL_THRESHOLD, GLOBAL_TOPK, POOL_SOFTMAX_THRESHOLD = 0, 1, 2, 3, 4
SELECT_OWN_BLOCK = 0x100


def vmoba_select(B, Hh, S, D, n_blocks, blk_off, Qp, Kp, tau, score_scale, mode, topk, Bmean, P, mask,
                 blk_ptr, q_idx, row_ptr, col_idx, pair_pos, nnz_capacity, k_out, theta_out, dev_status,
                 workspace, stream=None, query_pos=None, kv_rows=None):
    rc = lib().vmoba_select(B, Hh, S, D, n_blocks, _ptr(blk_off), _desc(Qp), _desc(Kp),
                            float(tau), float(score_scale), int(mode), int(topk), _ptr(Bmean), _ptr(P), _ptr(mask),
                            _ptr(blk_ptr), _ptr(q_idx), _ptr(row_ptr), _ptr(col_idx), _ptr(pair_pos),
                            int(nnz_capacity), _ptr(k_out), _ptr(theta_out), _ptr(dev_status), _ptr(query_pos),
                            _ptr(kv_rows), _ptr(workspace), workspace.nbytes, _stream(stream))
    _check("vmoba_select", rc)


SELECT_STATIC_MAX_BYTES = 32 << 20


def vmoba_select_static(B, Hh, S, D, n_blocks, blk_off, Qp, Kp, tau, score_scale, mode, topk, Bmean, P, mask,
                        blk_ptr, q_idx, row_ptr, col_idx, pair_pos, nnz_capacity, k_out, theta_out, dev_status,
                        stream=None, query_pos=None, kv_rows=None):
    """vmoba_select on the library's static scratch array (no workspace argument, nothing allocated)."""
    rc = lib().vmoba_select_static(B, Hh, S, D, n_blocks, _ptr(blk_off), _desc(Qp), _desc(Kp),
                                   float(tau), float(score_scale), int(mode), int(topk), _ptr(Bmean), _ptr(P),
                                   _ptr(mask), _ptr(blk_ptr), _ptr(q_idx), _ptr(row_ptr), _ptr(col_idx),
                                   _ptr(pair_pos), int(nnz_capacity), _ptr(k_out), _ptr(theta_out),
                                   _ptr(dev_status), _ptr(query_pos), _ptr(kv_rows), _stream(stream))
    _check("vmoba_select_static", rc)


def vmoba_attn_fwd(B, Hh, S, D, n_blocks, blk_off, Qp, Kp, Vp, blk_ptr, q_idx, row_ptr, pair_pos,
                   nnz_capacity, softmax_scale, O, LSE, workspace, stream=None, out_rows=None, kv_rows=None):
    rc = lib().vmoba_attn_fwd(B, Hh, S, D, n_blocks, _ptr(blk_off), _desc(Qp), _desc(Kp), _desc(Vp),
                              _ptr(blk_ptr), _ptr(q_idx), _ptr(row_ptr), _ptr(pair_pos), int(nnz_capacity),
                              float(softmax_scale), _desc(O), _ptr(LSE), _ptr(out_rows), _ptr(kv_rows), _ptr(workspace),
                              workspace.nbytes, _stream(stream))
    _check("vmoba_attn_fwd", rc)


def vmoba_attn_bwd(B, Hh, S, D, n_blocks, blk_off, Qp, Kp, Vp, O, LSE, dO, blk_ptr, q_idx, row_ptr,
                   pair_pos, nnz_capacity, softmax_scale, dQ, dK, dV, workspace, stream=None, rows=None, key_rows=None,
                   kv_rows=None):
    rc = lib().vmoba_attn_bwd(B, Hh, S, D, n_blocks, _ptr(blk_off), _desc(Qp), _desc(Kp), _desc(Vp),
                              _desc(O), _ptr(LSE), _desc(dO), _ptr(blk_ptr), _ptr(q_idx),
                              _ptr(row_ptr), _ptr(pair_pos), int(nnz_capacity), float(softmax_scale),
                              _desc(dQ), _desc(dK), _desc(dV), _ptr(rows), _ptr(key_rows), _ptr(kv_rows),
                              _ptr(workspace),
                              workspace.nbytes, _stream(stream))
    _check("vmoba_attn_bwd", rc)


# ------------------------------------------------------------------------------- around the sparse layer: positions, norms, dense attention
# A call on a few tokens is bound by the host: checks are comparisons on what a tensor hands out at once.
def _on_device(*tensors):
    """The kernels run on the current device's stream: every tensor (None: left out) has to lie there."""
    here = -2
    for t in tensors:
        if t is not None:
            at = t.get_device()
            if at != here:
                if here == -2 and at >= 0:
                    here = _device() if _device else torch.cuda.current_device()
                if at != here:
                    raise ValueError(f"a tensor of shape {tuple(t.shape)} lies on {t.device}, not on the current GPU")


def _shaped(name, t, shape):
    if t is not None and t.shape != shape:
        raise ValueError(f"{name} has the shape {tuple(t.shape)}, not {tuple(shape)}")


def _packed_array(t, name, dtype):
    """Address of a contiguous array of `dtype`, or None."""
    if t is None:
        return None
    if t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} has to be a contiguous {dtype} tensor")
    return t.data_ptr()


@functools.lru_cache(maxsize=256)
def _int_array(values):
    return (C.c_int32 * max(1, len(values)))(*values)


ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_NTK, ROPE_YARN = 0, 1, 2, 3
VMOBA_F8E4M3 = 2


def vmoba_rope_freqs(dims, base=10000.0, scaling=ROPE_PLAIN, factor=1.0, train_len=0):
    """dims: channels rotated per axis.  Returns (float64 CPU tensor [sum(dims) / 2], mscale)."""
    dims = tuple(int(d) for d in dims)
    freqs, m = torch.empty(max(1, sum(dims) // 2), dtype=torch.float64), C.c_float(0.0)
    _check("vmoba_rope_freqs", lib().vmoba_rope_freqs(len(dims), _int_array(dims), float(base), int(scaling), float(factor), int(train_len),
                                                      freqs.data_ptr(), C.byref(m)))
    return freqs, m.value


def vmoba_rope(B, S, D, ins, outs, freqs, dims, layout=ROPE_HALF, inverse=False, mscale=1.0, grid=None, first=0, positions=None, stream=None):
    """ins / outs: lists of (b, s, h, d) views, each with its own number of heads; freqs: float64 [sum(dims) / 2] on the device; grid: (T, H, W);
    positions: int32 [B or 1, S, len(dims)]."""
    n, dims = len(ins), tuple(dims)
    if len(outs) != n:
        raise ValueError("as many outputs as inputs")
    _on_device(freqs, positions, *ins, *outs)
    heads = []
    for x, y in zip(ins, outs):
        shape = x.shape
        if len(shape) != 4 or shape[0] != B or shape[1] != S or shape[3] != D or y.shape != shape:
            raise ValueError(f"inputs and outputs have the shapes {tuple(shape)} and {tuple(y.shape)}, not [{B}, {S}, heads, {D}]")
        heads.append(shape[2])
    _shaped("freqs", freqs, (sum(dims) // 2,))
    shared = positions is not None and positions.shape[0] == 1
    _shaped("positions", positions, (1 if shared else B, S, len(dims)))
    rc = lib().vmoba_rope(B, S, D, n, _int_array(tuple(heads)), b"".join(map(_desc, ins)), b"".join(map(_desc, outs)),
                          _packed_array(freqs, "freqs", torch.float64), len(dims), _int_array(dims), int(layout), int(inverse),
                          mscale, None if grid is None else make_grid(*grid), first, _packed_array(positions, "positions", torch.int32),
                          0 if shared else S * len(dims), _stream(stream))
    _check("vmoba_rope", rc)


def vmoba_rmsnorm_workspace_bytes(B, Hh, S, D) -> int:
    return lib().vmoba_rmsnorm_workspace_bytes(B, Hh, S, D)


def _weight(w, D):
    if w is None:
        return None, VMOBA_F32
    _shaped("weight", w, (D,))
    if not w.is_contiguous():
        raise ValueError("weight has to be contiguous")
    return w.data_ptr(), _dtype_code(w)


def _desc8(t):
    """Descriptor of a tensor that may be float8_e4m3fn."""
    if t.dtype != torch.float8_e4m3fn:
        return _desc(t)
    strides = t.stride()
    assert len(strides) == 4 and strides[3] == 1, "expect a (b, s, h, d) view with contiguous d"
    return _pack_desc(t.data_ptr(), VMOBA_F8E4M3, strides[0], strides[1], strides[2])


def vmoba_rmsnorm_fwd(B, Hh, S, D, x, residual, weight, eps, total, y, y_scale, inv_rms, stream=None):
    """x, residual, total, y: (b, s, h, d) views; y of x's type or float8_e4m3fn (then with y_scale [B, S, Hh]); residual and total, y_scale and
    inv_rms may be None."""
    _on_device(x, residual, weight, total, y, y_scale, inv_rms)
    shape, rows = (B, S, Hh, D), (B, S, Hh)
    for name, t in (("x", x), ("residual", residual), ("total", total), ("y", y)):
        _shaped(name, t, shape)
    _shaped("y_scale", y_scale, rows)
    _shaped("inv_rms", inv_rms, rows)
    w, code = _weight(weight, D)
    rc = lib().vmoba_rmsnorm_fwd(B, Hh, S, D, _desc(x), None if residual is None else _desc(residual), w, code, eps,
                                 None if total is None else _desc(total), _desc8(y), _packed_array(y_scale, "y_scale", torch.float32),
                                 _packed_array(inv_rms, "inv_rms", torch.float32), _stream(stream))
    _check("vmoba_rmsnorm_fwd", rc)


def vmoba_rmsnorm_bwd(B, Hh, S, D, x, weight, inv_rms, dy, dtotal, dx, dweight, workspace, stream=None):
    """x: what was normalised (the forward call's total, if there was a residual).  dtotal and dweight (then also workspace) may be None."""
    _on_device(x, weight, inv_rms, dy, dtotal, dx, dweight, workspace)
    shape = (B, S, Hh, D)
    for name, t in (("x", x), ("dy", dy), ("dtotal", dtotal), ("dx", dx)):
        _shaped(name, t, shape)
    _shaped("inv_rms", inv_rms, shape[:3])
    _shaped("dweight", dweight, (D,))
    w, code = _weight(weight, D)
    rc = lib().vmoba_rmsnorm_bwd(B, Hh, S, D, _desc(x), w, code, _packed_array(inv_rms, "inv_rms", torch.float32), _desc(dy),
                                 None if dtotal is None else _desc(dtotal), _desc(dx), _packed_array(dweight, "dweight", torch.float32),
                                 _ptr(workspace), 0 if workspace is None else workspace.nbytes, _stream(stream))
    _check("vmoba_rmsnorm_bwd", rc)


def vmoba_key_ranges(B, Sq, Sk, key_lo, key_hi, doc_off=None, prefix=None, causal=False, q_pos=None, q_first=0, stream=None):
    """key_lo, key_hi: int32 [B, Sq]; doc_off: int32 [B or 1, documents + 1]; prefix: int32 [B or 1, documents]; q_pos: int32 [B, Sq]."""
    _on_device(key_lo, key_hi, doc_off, prefix, q_pos)
    docs = 1 if doc_off is None else doc_off.shape[-1] - 1
    doc_rows, prefix_rows = (1 if t is not None and t.shape[0] == 1 else B for t in (doc_off, prefix))
    for name, t, shape in (("key_lo", key_lo, (B, Sq)), ("key_hi", key_hi, (B, Sq)), ("q_pos", q_pos, (B, Sq)), ("doc_off", doc_off, (doc_rows, docs + 1)),
                           ("prefix", prefix, (prefix_rows, docs))):
        _shaped(name, t, shape)
    i32 = torch.int32
    rc = lib().vmoba_key_ranges(B, Sq, Sk, _packed_array(doc_off, "doc_off", i32), 0 if doc_rows == 1 else docs + 1, docs,
                                _packed_array(prefix, "prefix", i32), 0 if prefix_rows == 1 else docs, int(causal), _packed_array(q_pos, "q_pos", i32),
                                q_first, _packed_array(key_lo, "key_lo", i32), _packed_array(key_hi, "key_hi", i32), _stream(stream))
    _check("vmoba_key_ranges", rc)


def vmoba_dense_workspace_bytes(op, B, Hq, Hkv, Sq, Sk, D, dtype) -> int:
    return lib().vmoba_dense_workspace_bytes(op, B, Hq, Hkv, Sq, Sk, D, dtype)


def _scores(B, Hq, Sq, softmax_scale, cap, slopes, key_lo, key_hi, q_pos, q_first):
    _on_device(slopes, key_lo, key_hi, q_pos)
    _shaped("slopes", slopes, (Hq,))
    for name, t in (("key_lo", key_lo), ("key_hi", key_hi), ("q_pos", q_pos)):
        _shaped(name, t, (B, Sq))
    i32 = torch.int32
    return vmoba_scores(softmax_scale, cap, _packed_array(slopes, "slopes", torch.float32), _packed_array(key_lo, "key_lo", i32),
                        _packed_array(key_hi, "key_hi", i32), _packed_array(q_pos, "q_pos", i32), q_first)


def vmoba_dense_fwd(B, Hq, Hkv, Sq, Sk, D, Q, K, V, O, LSE, workspace, softmax_scale, cap=0.0, slopes=None, key_lo=None, key_hi=None, q_pos=None,
                    q_first=0, stream=None):
    """Q, O: (b, s, h, d) views of Hq heads, K, V of Hkv; LSE: float32 [B, Hq, Sq]."""
    _on_device(Q, K, V, O, LSE, workspace)
    q, k = (B, Sq, Hq, D), (B, Sk, Hkv, D)
    for name, t, shape in (("Q", Q, q), ("K", K, k), ("V", V, k), ("O", O, q), ("LSE", LSE, (B, Hq, Sq))):
        _shaped(name, t, shape)
    how = _scores(B, Hq, Sq, softmax_scale, cap, slopes, key_lo, key_hi, q_pos, q_first)
    rc = lib().vmoba_dense_fwd(B, Hq, Hkv, Sq, Sk, D, _desc(Q), _desc(K), _desc(V), how, _desc(O), _packed_array(LSE, "LSE", torch.float32),
                               _ptr(workspace), workspace.nbytes, _stream(stream))
    _check("vmoba_dense_fwd", rc)


def vmoba_dense_bwd(B, Hq, Hkv, Sq, Sk, D, Q, K, V, O, LSE, dO, dQ, dK, dV, workspace, softmax_scale, cap=0.0, slopes=None, key_lo=None,
                    key_hi=None, q_pos=None, q_first=0, stream=None):
    _on_device(Q, K, V, O, LSE, dO, dQ, dK, dV, workspace)
    q, k = (B, Sq, Hq, D), (B, Sk, Hkv, D)
    for name, t, shape in (("Q", Q, q), ("K", K, k), ("V", V, k), ("O", O, q), ("LSE", LSE, (B, Hq, Sq)), ("dO", dO, q), ("dQ", dQ, q), ("dK", dK, k),
                           ("dV", dV, k)):
        _shaped(name, t, shape)
    how = _scores(B, Hq, Sq, softmax_scale, cap, slopes, key_lo, key_hi, q_pos, q_first)
    rc = lib().vmoba_dense_bwd(B, Hq, Hkv, Sq, Sk, D, _desc(Q), _desc(K), _desc(V), how, _desc(O), _packed_array(LSE, "LSE", torch.float32), _desc(dO),
                               _desc(dQ), _desc(dK), _desc(dV), _ptr(workspace), workspace.nbytes, _stream(stream))
    _check("vmoba_dense_bwd", rc)


# ------------------------------------------------------------------------------- buffer plan
class LayerPlan:
    """All device buffers of one layer geometry, allocated once (PyTorch is only the allocator).
    The methods call the C ABI in the order partition -> select -> attn_fwd -> attn_bwd ->
    inverse partition and allocate nothing.  With fused_io the attention calls read dO and write O,
    dQ, dK, dV in the caller's token order themselves (row map = perm): no partition of dO, no
    inverse partitions, and the block-order copies Op, dOp, dQp, dKp, dVp do not exist.
    With q_in_place (implies fused_io) only K and V are rearranged, as in the paper's Eq. 1: Q is read
    where the caller has it, a query's id is its token index everywhere (P, mask, lists, LSE), and O,
    dO, dQ need no row map at all; dK and dV go back through key_rows = perm.
    With kv_in_place (implies q_in_place) nothing is rearranged in memory at all: the partition call only
    builds the index arrays and every kernel finds key position k at row perm[k] of the caller's K and V.
    prepare: a QueryKeyPlan whose norms and rotary positions Q and K pass through first; backward() then returns the gradients of
    what was given to forward()."""

    def __init__(self, B, Hh, D, grid, block=(0, 0, 0), chunk=0, tau=0.25, dtype=torch.bfloat16,
                 device="cuda", score_scale=None, softmax_scale=None, need_bwd=True, mode=GLOBAL_THRESHOLD, topk=0,
                 fused_io=False, q_in_place=False, kv_in_place=False, prepare=None):
        T, H, W = grid
        self.prepare = prepare
        self.kv_in_place = bool(kv_in_place)
        self.q_in_place = bool(q_in_place) or self.kv_in_place
        self.fused_io = bool(fused_io) or self.q_in_place
        fused_io = self.fused_io
        self.Qin = None
        self.g = make_grid(T, H, W, *block, chunk)
        self.B, self.Hh, self.D, self.tau, self.dtype, self.dev = B, Hh, D, float(tau), dtype, device
        self.S, self.nb = vmoba_partition_dims(self.g)
        self.score_scale = score_scale if score_scale is not None else 1.0 / math.sqrt(D)
        self.softmax_scale = softmax_scale if softmax_scale is not None else 1.0 / math.sqrt(D)
        self.mode, self.topk = int(mode), int(topk)
        base_mode = self.mode & ~SELECT_OWN_BLOCK
        if base_mode == GLOBAL_THRESHOLD:
            self.cap = nnz_capacity_for(self.S, self.nb, tau)
        elif base_mode in (LOCAL_THRESHOLD, POOL_SOFTMAX_THRESHOLD):   # no bound below the whole pool
            self.cap = self.S * self.nb
        else:
            self.cap = self.S * min(self.topk, self.nb)
        if self.mode & SELECT_OWN_BLOCK:
            self.cap = min(self.cap + self.S, self.S * self.nb)
        S, nb, BH, cap = self.S, self.nb, B * Hh, self.cap
        dc = VMOBA_BF16 if dtype == torch.bfloat16 else VMOBA_F32
        i32 = dict(dtype=torch.int32, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        self.perm = torch.empty(S, **i32)
        self.inv_perm = torch.empty(S, **i32)
        self.blk_off = torch.empty(nb + 1, **i32)

        def blk_tensor(dt=dtype):   # block-order storage [B, Hh, S, D], handed out as a (b, s, h, d) view
            return torch.empty(B, Hh, S, D, dtype=dt, device=device).permute(0, 2, 1, 3)

        self.Kp, self.Vp = (None, None) if self.kv_in_place else (blk_tensor() for _ in range(2))
        self.Qp = None if self.q_in_place else blk_tensor()
        self.Op = None if fused_io else blk_tensor()
        self.LSE = torch.empty(B, Hh, S, **f32)
        self.Bmean = torch.empty(B, Hh, nb, D, **f32)
        self.P = torch.empty(B, Hh, S, nb, **f32)
        self.words = (nb + 31) // 32
        self.mask = torch.empty(B, Hh, S, self.words, **i32)
        self.blk_ptr = torch.empty(BH, nb + 1, **i32)
        self.row_ptr = torch.empty(BH, S + 1, **i32)
        self.q_idx = torch.empty(BH * cap, **i32)
        self.col_idx = torch.empty(BH * cap, **i32)
        self.pair_pos = torch.empty(BH * cap, **i32)
        self.k_out = torch.empty(BH, dtype=torch.int64, device=device)
        self.theta = torch.empty(BH, **f32)
        self.dev_status = torch.zeros(1, **i32)
        n_sel = vmoba_workspace_bytes(OP_SELECT, B, Hh, S, D, nb, cap, dc)
        n_fwd = vmoba_workspace_bytes(OP_ATTN_FWD, B, Hh, S, D, nb, cap, dc)
        n_bwd = vmoba_workspace_bytes(OP_ATTN_BWD, B, Hh, S, D, nb, cap, dc) if need_bwd else 0
        self.ws_select = torch.empty(n_sel, dtype=torch.uint8, device=device)
        # forward partials are dead once O is merged, so forward and backward share one workspace
        self.ws_attn = torch.empty(max(n_fwd, n_bwd), dtype=torch.uint8, device=device)
        self.O = torch.empty(B, S, Hh, D, dtype=dtype, device=device)
        if need_bwd:
            if not fused_io:
                self.dOp, self.dQp, self.dKp, self.dVp = (blk_tensor() for _ in range(4))
            self.dQ, self.dK, self.dV = (torch.empty(B, S, Hh, D, dtype=dtype, device=device) for _ in range(3))

    # -- the hot path, one method per C-ABI call -------------------------------------------
    def partition(self, Q, K, V):
        if self.kv_in_place:         # index arrays only; the blocks of Eq. 1 are addressed where they lie
            self.Qin, self.Kp, self.Vp = Q, K, V
            vmoba_partition(self.g, 0, self.B, self.Hh, self.D, [], [], self.perm, self.inv_perm, self.blk_off)
            return
        if self.q_in_place:          # Eq. 1 as written: only the keys (and their values) are rearranged
            self.Qin = Q
            vmoba_partition(self.g, 0, self.B, self.Hh, self.D, [K, V], [self.Kp, self.Vp],
                            self.perm, self.inv_perm, self.blk_off)
            return
        vmoba_partition(self.g, 0, self.B, self.Hh, self.D, [Q, K, V], [self.Qp, self.Kp, self.Vp],
                        self.perm, self.inv_perm, self.blk_off)

    def _q(self):
        return self.Qin if self.q_in_place else self.Qp

    def select(self):
        vmoba_select(self.B, self.Hh, self.S, self.D, self.nb, self.blk_off, self._q(), self.Kp, self.tau,
                     self.score_scale, self.mode, self.topk, self.Bmean, self.P, self.mask, self.blk_ptr, self.q_idx,
                     self.row_ptr, self.col_idx, self.pair_pos, self.cap, self.k_out, self.theta,
                     self.dev_status, self.ws_select, query_pos=self.inv_perm if self.q_in_place else None,
                     kv_rows=self.perm if self.kv_in_place else None)

    def attn_fwd(self):
        if self.q_in_place:
            vmoba_attn_fwd(self.B, self.Hh, self.S, self.D, self.nb, self.blk_off, self.Qin, self.Kp, self.Vp,
                           self.blk_ptr, self.q_idx, self.row_ptr, self.pair_pos, self.cap, self.softmax_scale,
                           self.O, self.LSE, self.ws_attn, kv_rows=self.perm if self.kv_in_place else None)
            return
        vmoba_attn_fwd(self.B, self.Hh, self.S, self.D, self.nb, self.blk_off, self.Qp, self.Kp, self.Vp,
                       self.blk_ptr, self.q_idx, self.row_ptr, self.pair_pos, self.cap, self.softmax_scale,
                       self.O if self.fused_io else self.Op, self.LSE, self.ws_attn,
                       out_rows=self.perm if self.fused_io else None)

    def unpartition_out(self):
        vmoba_partition(self.g, 1, self.B, self.Hh, self.D, [self.Op], [self.O], self.perm, None, None)

    def partition_dO(self, dO):
        vmoba_partition(self.g, 0, self.B, self.Hh, self.D, [dO], [self.dOp], self.perm, None, None)

    def attn_bwd(self, dO=None):
        """dO: the caller-layout gradient (fused_io only; otherwise partition_dO() has run)."""
        if self.q_in_place:
            vmoba_attn_bwd(self.B, self.Hh, self.S, self.D, self.nb, self.blk_off, self.Qin, self.Kp, self.Vp,
                           self.O, self.LSE, dO, self.blk_ptr, self.q_idx, self.row_ptr, self.pair_pos,
                           self.cap, self.softmax_scale, self.dQ, self.dK, self.dV, self.ws_attn, key_rows=self.perm,
                           kv_rows=self.perm if self.kv_in_place else None)
            return
        if self.fused_io:
            vmoba_attn_bwd(self.B, self.Hh, self.S, self.D, self.nb, self.blk_off, self.Qp, self.Kp, self.Vp,
                           self.O, self.LSE, dO, self.blk_ptr, self.q_idx, self.row_ptr, self.pair_pos,
                           self.cap, self.softmax_scale, self.dQ, self.dK, self.dV, self.ws_attn, rows=self.perm)
            return
        vmoba_attn_bwd(self.B, self.Hh, self.S, self.D, self.nb, self.blk_off, self.Qp, self.Kp, self.Vp,
                       self.Op, self.LSE, self.dOp, self.blk_ptr, self.q_idx, self.row_ptr, self.pair_pos,
                       self.cap, self.softmax_scale, self.dQp, self.dKp, self.dVp, self.ws_attn)

    def unpartition_grads(self):
        vmoba_partition(self.g, 1, self.B, self.Hh, self.D, [self.dQp, self.dKp, self.dVp],
                        [self.dQ, self.dK, self.dV], self.perm, None, None)

    def forward(self, Q, K, V):
        if self.prepare is not None:
            Q, K = self.prepare.forward(Q, K)
        self.partition(Q, K, V)
        self.select()
        self.attn_fwd()
        if not self.fused_io:
            self.unpartition_out()
        return self.O

    def backward(self, dO):
        if self.fused_io:
            self.attn_bwd(dO)
        else:
            self.partition_dO(dO)
            self.attn_bwd()
            self.unpartition_grads()
        if self.prepare is not None:
            return *self.prepare.backward(self.dQ, self.dK), self.dV
        return self.dQ, self.dK, self.dV


class QueryKeyPlan:
    """What queries and keys pass through between the projections and the attention: a root-mean-square norm with a weight each, and rotary
    positions on the latent grid (or given ones).  All buffers are allocated once; the methods allocate nothing.
    dims: channels rotated per axis, None: no rotation.  norm: None, "head" (over the D channels of every head, weights [D]) or "token" (over all
    heads of a token, weights [heads * D]).  The weights wq, wk are the caller's; gradients of theirs are in dwq, dwk after backward()."""

    def __init__(self, B, Hq, Hkv, S, D, dims=None, grid=None, layout=ROPE_HALF, base=10000.0, scaling=ROPE_PLAIN, factor=1.0, train_len=0,
                 norm="head", wq=None, wk=None, eps=1e-6, dtype=torch.bfloat16, device="cuda", need_bwd=True):
        if norm not in (None, "head", "token"):
            raise ValueError("norm is None, 'head' or 'token'")
        self.B, self.S, self.D, self.heads, self.dims, self.grid, self.layout = B, S, D, (Hq, Hkv), dims, grid, layout
        self.norm, self.weights, self.eps = norm, (wq, wk), eps
        if dims is not None:
            freqs, self.mscale = vmoba_rope_freqs(dims, base, scaling, factor, train_len)
            self.freqs = freqs.to(device)
        new = lambda: [torch.empty(B, S, h, D, dtype=dtype, device=device) for h in self.heads]      # noqa: E731
        self.out, self.grads = new(), new() if need_bwd else None
        if norm is not None:
            sizes = [self._rows(h) for h in self.heads]
            self.inv_rms = [torch.empty(B, S, n, device=device) for n, _ in sizes]
            if need_bwd:
                self.dwq, self.dwk = (torch.empty(d, device=device) for _, d in sizes)
                n = max(vmoba_rmsnorm_workspace_bytes(B, n, S, d) for n, d in sizes)
                self.workspace = torch.empty(n, dtype=torch.uint8, device=device)

    def _rows(self, heads):
        """Rows per token and channels per row of the norm."""
        return (heads, self.D) if self.norm == "head" else (1, heads * self.D)

    def _view(self, t, heads):
        return t.view(self.B, self.S, *self._rows(heads))

    def _rotate(self, src, dst, inverse, first, positions):
        vmoba_rope(self.B, self.S, self.D, src, dst, self.freqs, self.dims, self.layout, inverse, self.mscale, self.grid, first, positions)

    def forward(self, Q, K, first=0, positions=None):
        """Q: [B, S, Hq, D], K: [B, S, Hkv, D]; first, positions: as in vmoba_rope.  Q and K are read again by backward()."""
        self.inputs, self.at = (Q, K), (first, positions)
        src = [Q, K]
        if self.norm is not None:
            for x, y, w, inv, h in zip(src, self.out, self.weights, self.inv_rms, self.heads):
                n, d = self._rows(h)
                vmoba_rmsnorm_fwd(self.B, n, self.S, d, self._view(x, h), None, w, self.eps, None, self._view(y, h), None, inv)
            src = self.out
        if self.dims is not None:
            self._rotate(src, self.out, False, *self.at)
            src = self.out
        return src[0], src[1]

    def backward(self, dQ, dK):
        """Gradients of forward()'s inputs, from those of its outputs."""
        src = [dQ, dK]
        if self.dims is not None:
            self._rotate(src, self.grads, True, *self.at)
            src = self.grads
        if self.norm is not None:
            for x, dy, dx, w, inv, h, dw in zip(self.inputs, src, self.grads, self.weights, self.inv_rms, self.heads, (self.dwq, self.dwk)):
                n, d = self._rows(h)
                vmoba_rmsnorm_bwd(self.B, n, self.S, d, self._view(x, h), w, inv, self._view(dy, h), None, self._view(dx, h),
                                  None if w is None else dw, self.workspace)
            src = self.grads
        return src[0], src[1]


class DensePlan:
    """Dense attention in the place of a sparse layer -- the layers and sampling steps that stay dense, packed clips, a prefix of text, a cache -- with all
    buffers allocated once.  doc_off, prefix: int32 tensors on the device, read at every forward() (see vmoba_key_ranges).  prepare: as in LayerPlan."""

    def __init__(self, B, Hq, Hkv, Sq, Sk, D, dtype=torch.bfloat16, device="cuda", softmax_scale=None, cap=0.0, slopes=None, doc_off=None, prefix=None,
                 causal=False, need_bwd=True, prepare=None):
        self.size, self.prepare = (B, Hq, Hkv, Sq, Sk, D), prepare
        self.ranges = dict(doc_off=doc_off, prefix=prefix, causal=causal)
        self.ranged = doc_off is not None or prefix is not None or causal
        self.scores = dict(softmax_scale=1.0 / math.sqrt(D) if softmax_scale is None else softmax_scale, cap=cap, slopes=slopes)
        code = VMOBA_BF16 if dtype == torch.bfloat16 else VMOBA_F32
        n = max(vmoba_dense_workspace_bytes(op, *self.size, code) for op in ([OP_ATTN_FWD, OP_ATTN_BWD] if need_bwd else [OP_ATTN_FWD]))
        if n == 0:
            raise VmobaError("vmoba_dense_workspace_bytes", -2)
        self.workspace = torch.empty(n, dtype=torch.uint8, device=device)
        self.O = torch.empty(B, Sq, Hq, D, dtype=dtype, device=device)
        self.LSE = torch.empty(B, Hq, Sq, device=device)
        self.key_lo, self.key_hi = (torch.empty(B, Sq, dtype=torch.int32, device=device) for _ in range(2))
        if need_bwd:
            self.dQ, self.dK, self.dV = (torch.empty(B, s, h, D, dtype=dtype, device=device) for s, h in ((Sq, Hq), (Sk, Hkv), (Sk, Hkv)))

    def forward(self, Q, K, V, q_pos=None):
        """q_pos: int32 [B, Sq], positions of the queries among the keys; None: the last Sq ones."""
        B, _, _, Sq, Sk, _ = self.size
        if self.prepare is not None:
            Q, K = self.prepare.forward(Q, K)
        self.inputs, self.how = (Q, K, V), dict(self.scores, q_pos=q_pos, q_first=Sk - Sq)
        if self.ranged:
            vmoba_key_ranges(B, Sq, Sk, self.key_lo, self.key_hi, q_pos=q_pos, q_first=Sk - Sq, **self.ranges)
            self.how.update(key_lo=self.key_lo, key_hi=self.key_hi)
        vmoba_dense_fwd(*self.size, Q, K, V, self.O, self.LSE, self.workspace, **self.how)
        return self.O

    def backward(self, dO):
        vmoba_dense_bwd(*self.size, *self.inputs, self.O, self.LSE, dO, self.dQ, self.dK, self.dV, self.workspace, **self.how)
        if self.prepare is not None:
            return *self.prepare.backward(self.dQ, self.dK), self.dV
        return self.dQ, self.dK, self.dV
