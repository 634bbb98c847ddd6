"""Front end of the C-ABI library (``include/unionsparse.h``): argument marshalling only. Encoding and the host
calls go through ctypes; the calls made per product go through a native module (``csrc/us_torch.cpp``), because
marshalling them in Python takes longer than a small product takes on the GPU.

Every step of the SpMM runs in the CUDA library; there is no CPU fallback. Importing this module
fails loudly when the compiled library is missing, and the first call that takes tensors when the native
module is (build them with ``python -m paper_2608_09291_b200.build`` or ``__graft_entry__.build()``).
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import numpy as np

_LIB_PATH = Path(__file__).resolve().parent / "libunionsparse.so"
_EXT_PATH = _LIB_PATH.with_name("_us_torch.so")
if not _LIB_PATH.exists():
    raise ImportError(f"{_LIB_PATH} is missing: build the CUDA library first "
                      "(python -m paper_2608_09291_b200.build)")
_lib = ctypes.CDLL(str(_LIB_PATH))

US_OK = 0
US_ENCODE_HOST_ONLY = 1
US_ENCODE_SORT_ROWS = 2
US_ENCODE_PAIR_ROWS = 4
US_ENCODE_W2 = 8

EXPORTS = ["us_encode", "us_get_stats", "us_decode", "us_get_row_order", "us_spmm", "us_spmm_static_scratch",
           "us_spmm_requant", "us_absmax_f16", "us_quantize_f16",
           "us_last_error", "us_debug_withhold_copy", "us_stage_timers", "us_destroy", "us_spmm_bytes", "us_launch_info", "us_launch_kernel",
           "us_mx4_bytes", "us_mx4_quantize", "us_mx4_dequantize", "us_mx4_pack", "us_mx4_unpack", "us_mx4_matmul",
           "us_mx4_linear_scratch", "us_mx4_linear", "us_mx4_matmul_epilogue", "us_mx4_linear_epilogue", "us_mx4_last_error",
           "us_kv_create", "us_kv_append", "us_kv_append_granted", "us_kv_read", "us_kv_attention_scratch", "us_kv_attention", "us_kv_shared_attention_scratch",
           "us_kv_shared_attention", "us_kv_last_error", "us_kv_destroy",
           "us_kv_fork", "us_kv_release", "us_kv_extend_scratch", "us_kv_extend", "us_kv_extend_granted", "us_kv_compact_scratch", "us_kv_compact", "us_kv_remap", "us_kv_copy_blocks",
           "us_qk_norm_rope",
           "us_status_string"]


class us_format(ctypes.Structure):
    _fields_ = [("H_L", ctypes.c_int32), ("K_L", ctypes.c_int32),
                ("R_A", ctypes.c_int32), ("C_A", ctypes.c_int32)]


class us_stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "M", "K", "Mp", "Kp", "nnz", "n_tiles", "sum_P", "bytes_payload", "bytes_payload_padded",
        "bytes_bitmap", "bytes_offsets", "bytes_total")] + [
        ("pmr", ctypes.c_double), ("fill", ctypes.c_double), ("fmt", us_format),
        ("weight_bits", ctypes.c_int32), ("reserved", ctypes.c_int32)]


_vp = ctypes.c_void_p
_lib.us_encode.argtypes = [_vp, ctypes.c_int64, ctypes.c_int64, _vp, ctypes.POINTER(us_format),
                           ctypes.c_int32, ctypes.c_uint32, ctypes.POINTER(_vp)]
_lib.us_get_stats.argtypes = [_vp, ctypes.POINTER(us_stats)]
_lib.us_decode.argtypes = [_vp, _vp]
_lib.us_get_row_order.argtypes = [_vp, _vp]
_lib.us_spmm.argtypes = [_vp, _vp, ctypes.c_int32, _vp, _vp, _vp]
_lib.us_last_error.argtypes = [_vp]
_lib.us_spmm_static_scratch.argtypes = [_vp, _vp, ctypes.c_int32, _vp, _vp, _vp]
_lib.us_spmm_requant.argtypes = [_vp, _vp, ctypes.c_int64, _vp, ctypes.c_int32, _vp, _vp, ctypes.c_int64,
                                 ctypes.c_int64, _vp]
_lib.us_absmax_f16.argtypes = [_vp, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, _vp, _vp]
_lib.us_quantize_f16.argtypes = [_vp, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, _vp, _vp, _vp, _vp]
_lib.us_destroy.argtypes = [_vp]
_lib.us_stage_timers.argtypes = [_vp, ctypes.c_int32, _vp, ctypes.c_int32]
_lib.us_debug_withhold_copy.argtypes = [_vp, ctypes.c_int64, ctypes.c_int64]
_lib.us_spmm_bytes.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32]
_lib.us_spmm_bytes.restype = ctypes.c_int64
_lib.us_launch_info.argtypes = [_vp, ctypes.c_int32] + [ctypes.POINTER(ctypes.c_int32)] * 3
_lib.us_launch_kernel.argtypes = [_vp, ctypes.c_int32, _vp]
_lib.us_launch_kernel.restype = ctypes.c_char_p
_i32, _i64 = ctypes.c_int32, ctypes.c_int64
_lib.us_mx4_bytes.argtypes = [_i64, _i64]
_lib.us_mx4_bytes.restype = _i64
_lib.us_mx4_quantize.argtypes = [_vp, _i32, _i64, _i64, _i64, _vp, _vp]
_lib.us_mx4_dequantize.argtypes = [_vp, _i64, _i64, _vp, _i32, _i64, _vp]
_lib.us_mx4_pack.argtypes = [_vp, _i64, _vp, _i64, _i64, _i64, _vp, _vp]
_lib.us_mx4_unpack.argtypes = [_vp, _i64, _i64, _vp, _i64, _vp, _i64, _vp]
_lib.us_mx4_matmul.argtypes = [_vp, _i64, _vp, _i64, _i64, _vp, _i32, _i64, ctypes.c_uint32, _vp]
_lib.us_mx4_linear_scratch.argtypes = [_i64, _i64, _i64]
_lib.us_mx4_linear_scratch.restype = _i64
_lib.us_mx4_linear.argtypes = [_vp, _i32, _i64, _i64, _vp, _i64, _i64, _vp, _i32, _i64, _vp, _i64, ctypes.c_uint32, _vp]


class us_mx4_epilogue(ctypes.Structure):
    _fields_ = [("bias", _vp), ("residual", _vp), ("ldr", _i64), ("bias_type", _i32), ("residual_type", _i32), ("act", _i32), ("gated", _i32)]


_lib.us_mx4_matmul_epilogue.argtypes = [_vp, _i64, _vp, _i64, _i64, ctypes.POINTER(us_mx4_epilogue), _vp, _i32, _i64, ctypes.c_uint32, _vp]
_lib.us_mx4_linear_epilogue.argtypes = [_vp, _i32, _i64, _i64, _vp, _i64, _i64, ctypes.POINTER(us_mx4_epilogue), _vp, _i32, _i64, _vp, _i64, ctypes.c_uint32, _vp]
_lib.us_mx4_last_error.argtypes = []


class us_kv_seqs(ctypes.Structure):
    _fields_ = [("block_table", _vp), ("table_stride", _i64), ("lengths", _vp), ("cu_tokens", _vp), ("n_seqs", _i32), ("table_width", _i32)]


_seqs = ctypes.POINTER(us_kv_seqs)
_lib.us_kv_create.argtypes = [_vp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, ctypes.POINTER(_vp)]
_lib.us_kv_append.argtypes = [_vp, _seqs, _i64, _vp, _vp, _i32, _i64, _i64, _i64, _i64, _vp]
_lib.us_kv_append_granted.argtypes = [_vp, _seqs, _i64, _vp, _vp, _i32, _i64, _i64, _i64, _i64, _vp, _vp]
_lib.us_kv_read.argtypes = [_vp, _seqs, _i64, _vp, _vp, _i32, _vp]
_lib.us_kv_attention_scratch.argtypes = [_vp, _seqs, _i64, _i32]
_lib.us_kv_attention_scratch.restype = _i64
_lib.us_kv_attention.argtypes = [_vp, _seqs, _i64, _vp, _i32, _i32, _i64, _i64, ctypes.c_float, _i32, _i32, _vp, _i64, _i64, _vp, _vp, _i64, _vp]
_lib.us_kv_shared_attention_scratch.argtypes = [_vp, _seqs, _seqs, _i64, _i32]
_lib.us_kv_shared_attention_scratch.restype = _i64
_lib.us_kv_shared_attention.argtypes = [_vp, _seqs, _seqs, _i64, _vp, _i32, _i32, _i64, _i64, ctypes.c_float, _i32, _vp, _i64, _i64, _vp, _vp, _i64, _vp]
_lib.us_kv_last_error.argtypes = []
_lib.us_kv_destroy.argtypes = [_vp]
_lib.us_kv_fork.argtypes = [_vp, _vp, _seqs, _vp, _i32, _vp, _i64, _vp, _i32, _vp]
_lib.us_kv_release.argtypes = [_vp, _vp, _seqs, _vp]
_lib.us_kv_extend_scratch.argtypes = [_vp, _i32]
_lib.us_kv_extend_scratch.restype = _i64
_lib.us_kv_extend.argtypes = [_vp, _vp, _vp, _i64, _i32, _vp, _i32, _vp, _i32, _vp, _i64, _vp]
_lib.us_kv_extend_granted.argtypes = [_vp, _vp, _vp, _i64, _i32, _vp, _i32, _vp, _i32, _vp, _vp, _i64, _vp]
_lib.us_kv_compact_scratch.argtypes = [_vp]
_lib.us_kv_compact_scratch.restype = _i64
_lib.us_kv_compact.argtypes = [_vp, _vp, _seqs, _i32, _vp, _vp, _vp, _i64, _vp]
_lib.us_kv_remap.argtypes = [_vp, _vp, _seqs, _vp]
_lib.us_kv_copy_blocks.argtypes = [_vp, _vp, _vp, _i64, _vp]


class us_rotary(ctypes.Structure):
    _fields_ = [("turns", _vp), ("axis", _vp), ("rotary_dim", _i32), ("axes", _i32), ("interleaved", _i32)]


class us_heads(ctypes.Structure):
    _fields_ = [("x", _vp), ("token_stride", _i64), ("head_stride", _i64), ("out", _vp), ("out_token_stride", _i64), ("out_head_stride", _i64),
                ("weight", _vp), ("weight_type", _i32), ("heads", _i32)]


_lib.us_qk_norm_rope.argtypes = [ctypes.POINTER(us_rotary), _vp, _i64, _i64, _i32, _i32, ctypes.POINTER(us_heads), ctypes.POINTER(us_heads), ctypes.c_float, _vp]
_lib.us_status_string.argtypes = [ctypes.c_int]
_lib.us_status_string.restype = ctypes.c_char_p


class UsError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {_lib.us_status_string(status).decode()} (status {status})")


def _check(status: int, where: str):
    if status != US_OK:
        raise UsError(status, where)


_ext = None   # the native module: imported with the first tensor call, so that host-only use needs no torch


def _native():
    global _ext
    if _ext is None:
        import torch  # noqa: F401  (its libraries have to be loaded first)
        if not _EXT_PATH.exists():
            raise ImportError(f"{_EXT_PATH} is missing: build it first (python -m paper_2608_09291_b200.build)")
        from . import _us_torch
        _us_torch.set_error(UsError)
        _ext = _us_torch
    return _ext


def us_status_string(status: int) -> str:
    return _lib.us_status_string(int(status)).decode()


def us_encode(W: np.ndarray, w_scale: np.ndarray | None = None, fmt: tuple | None = None,
              max_N: int = 64, flags: int = 0) -> int:
    """W: host int8 (M, K); w_scale: host float16 (M,) or None. Returns the handle."""
    W = np.ascontiguousarray(W, dtype=np.int8)
    M, K = W.shape
    ws = None
    if w_scale is not None:
        ws = np.ascontiguousarray(w_scale, dtype=np.float16)
        assert ws.shape == (M,)
    f = us_format(*fmt) if fmt is not None else None
    h = _vp()
    st = _lib.us_encode(W.ctypes.data, M, K, ws.ctypes.data if ws is not None else None,
                        ctypes.byref(f) if f is not None else None, int(max_N), int(flags),
                        ctypes.byref(h))
    _check(st, "us_encode")
    return h.value


def us_get_stats(h: int) -> dict:
    st = us_stats()
    _check(_lib.us_get_stats(h, ctypes.byref(st)), "us_get_stats")
    d = {n: getattr(st, n) for n, _ in us_stats._fields_ if n != "fmt"}
    d["fmt"] = (st.fmt.H_L, st.fmt.K_L, st.fmt.R_A, st.fmt.C_A)
    return d


def us_decode(h: int) -> np.ndarray:
    st = us_get_stats(h)
    out = np.zeros((st["M"], st["K"]), dtype=np.int8)
    _check(_lib.us_decode(h, out.ctypes.data), "us_decode")
    return out


def us_get_row_order(h: int) -> np.ndarray:
    st = us_get_stats(h)
    out = np.zeros(st["Mp"], dtype=np.int32)
    _check(_lib.us_get_row_order(h, out.ctypes.data), "us_get_row_order")
    return out


def us_spmm(h: int, X_ptr: int, N: int, x_scale_ptr: int | None, Y_ptr: int, stream: int | None = None):
    """Raw call: device pointers as integers, stream as a cudaStream_t integer (None = default)."""
    _check(_lib.us_spmm(h, X_ptr, int(N), x_scale_ptr, Y_ptr, stream), "us_spmm")


US_STATIC_SCRATCH_BYTES = 4 << 20
US_ERR_SCRATCH_TOO_SMALL = 8


def us_spmm_static_scratch(h: int, X_ptr: int, N: int, x_scale_ptr: int | None, Y_ptr: int,
                           stream: int | None = None):
    """us_spmm for callers that may not allocate device memory around the call: the kernel's
    scratch (strip sums and arrival counters) is a fixed 4 MiB array inside the library image,
    shared by all calls on the GPU -- overlapping calls race, and a problem that does not fit
    is refused with status US_ERR_SCRATCH_TOO_SMALL. Same arguments as us_spmm."""
    _check(_lib.us_spmm_static_scratch(h, X_ptr, int(N), x_scale_ptr, Y_ptr, stream),
           "us_spmm_static_scratch")


def us_spmm_requant(h: int, X16_ptr: int, ldx: int, x_amax_ptr: int, N: int, Y16_ptr: int,
                    y_amax_ptr: int | None = None, amax_m0: int = 0, amax_m1: int = 0,
                    stream: int | None = None):
    """Chained call: fp16 activations (row stride ldx elements) quantised per token to INT4 with
    the step max|x| / 7 while they are staged, fp16 output, and optionally the per-token absmax
    of output columns [amax_m0, amax_m1) for the next call. Device pointers as integers."""
    _check(_lib.us_spmm_requant(h, X16_ptr, int(ldx), x_amax_ptr, int(N), Y16_ptr, y_amax_ptr,
                                int(amax_m0), int(amax_m1), stream), "us_spmm_requant")


def us_absmax_f16(X16_ptr: int, ldx: int, N: int, K: int, amax_ptr: int, stream: int | None = None):
    """Fills the absmax buffer at amax_ptr with max_k |X16[n][k]| per token."""
    _check(_lib.us_absmax_f16(X16_ptr, int(ldx), int(N), int(K), amax_ptr, stream), "us_absmax_f16")


def us_quantize_f16(X16_ptr: int, ldx: int, N: int, K: int, amax_ptr: int, Xq_ptr: int,
                    x_scale_ptr: int | None = None, stream: int | None = None):
    """The INT4 codes of the chained call's quantiser, packed as us_spmm expects X, and the steps."""
    _check(_lib.us_quantize_f16(X16_ptr, int(ldx), int(N), int(K), amax_ptr, Xq_ptr, x_scale_ptr, stream),
           "us_quantize_f16")


def us_last_error(h: int) -> int:
    return int(_lib.us_last_error(h))


def us_debug_withhold_copy(h: int, position: int, wait_us: int = 1000):
    """Test hook: later us_spmm calls on the handle never copy the tile at `position` and bound
    their waits to wait_us microseconds (position < 0: back to normal)."""
    _check(_lib.us_debug_withhold_copy(h, int(position), int(wait_us)), "us_debug_withhold_copy")


def us_stage_timers(h: int, enable: int = -1, read: bool = False, per_cta: int = 0):
    """Switch the kernel's stage timers on/off; with read=True return (and clear) the sums
    {wait, decode, epilogue, lifetime, prologue} in SM cycles, the number of warps, the
    longest warp lifetime and the first-start-to-last-end span in ns; with per_cta = n also the
    prologue checkpoints and, for the first n CTAs, the time stamps (start, first warp end,
    activations staged, end, past the dependency wait) in ns."""
    n = 8 + (4 + 5 * per_cta if per_cta else 0)
    out = (ctypes.c_uint64 * n)() if read else None
    _check(_lib.us_stage_timers(h, int(enable), out, n if read else 0), "us_stage_timers")
    if read:
        d = dict(zip(("wait", "decode", "epilogue", "lifetime", "warps", "prologue", "max_lifetime", "span_ns"),
                     [int(v) for v in out[:8]]))
        if per_cta:
            d["checkpoints"] = [int(v) for v in out[8:12]]
            d["ctas"] = [tuple(int(v) for v in out[12 + 5 * c: 17 + 5 * c]) for c in range(per_cta)]
        return d
    return None


def us_destroy(h: int):
    _check(_lib.us_destroy(h), "us_destroy")


def us_spmm_bytes(h: int, N: int, fp16_out: bool) -> int:
    return int(_lib.us_spmm_bytes(h, int(N), int(bool(fp16_out))))


def us_launch_info(h: int, N: int) -> dict:
    g, b, s = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check(_lib.us_launch_info(h, int(N), ctypes.byref(g), ctypes.byref(b), ctypes.byref(s)),
           "us_launch_info")
    return {"grid": g.value, "block": b.value, "smem_bytes": s.value}


def us_launch_kernel(h: int, N: int, stream: int | None = None) -> str:
    """Name of the kernel that this thread's next us_spmm for N tokens on the stream would launch."""
    name = _lib.us_launch_kernel(h, int(N), stream)
    if name is None:
        us_launch_info(h, N)   # (raises with the reason)
    return name.decode()


def pack_int4(X: np.ndarray) -> np.ndarray:
    """(N, K) int8 values in [-8, 7] -> (N, ceil(K/2)) bytes, k even in the low nibble."""
    X = np.ascontiguousarray(X, dtype=np.int8)
    N, K = X.shape
    if K % 2:
        X = np.concatenate([X, np.zeros((N, 1), np.int8)], axis=1)
    u = X.view(np.uint8) & 0xF
    return np.ascontiguousarray(u[:, 0::2] | (u[:, 1::2] << 4))


US_AMAX_BYTES = 4 * 64 * (1 + 192)


def new_amax(device="cuda"):
    """An absmax buffer (device int32 tensor) for the chained calls."""
    import torch
    return torch.zeros(US_AMAX_BYTES // 4, device=device, dtype=torch.int32)


def amax_values(buf, N: int):
    """The per-token absmax an absmax buffer holds, as a host uint16 array of fp16 bit patterns."""
    w = buf.cpu().numpy()
    parts = int(w[0])
    return w[64:64 + 64 * parts].reshape(parts, 64)[:, :N].max(axis=0).astype(np.uint16)


def absmax_f16(X16, out=None, stream=None):
    """Per-token absmax of a device float16 (N, K) tensor or view (unit column stride), as the
    absmax buffer the chained call takes."""
    if out is None:
        out = new_amax(X16.device)
    (_ext or _native()).absmax_f16(X16, out, stream)
    return out


def quantize_f16(X16, amax, stream=None):
    """(packed INT4 codes uint8 (N, ceil(K/2)), steps float16 (N,)) of a device float16 (N, K)."""
    import torch
    assert X16.dtype == torch.float16 and X16.stride(1) == 1
    N, K = X16.shape
    Xq = torch.empty((N, (K + 1) // 2), device=X16.device, dtype=torch.uint8)
    sc = torch.empty(N, device=X16.device, dtype=torch.float16)
    if stream is None:
        stream = torch.cuda.current_stream(X16.device).cuda_stream
    us_quantize_f16(X16.data_ptr(), X16.stride(0), N, K, amax.data_ptr(), Xq.data_ptr(), sc.data_ptr(), stream)
    return Xq, sc


class SparseWeight:
    """An encoded weight on the current CUDA device. Torch tensors are used only as device memory."""

    def __init__(self, W: np.ndarray, w_scale: np.ndarray | None = None, fmt: tuple | None = None,
                 max_N: int = 64, flags: int = 0):
        _native()
        self.handle = us_encode(W, w_scale, fmt, max_N, flags)
        self.stats = us_get_stats(self.handle)
        self.M, self.K = self.stats["M"], self.stats["K"]
        self.has_scale = w_scale is not None

    def spmm(self, X, N: int, x_scale=None, out=None, stream=None):
        """X: device uint8 tensor (N, ceil(K/2)); x_scale: device float16 (N,) or None.
        Returns a device tensor (N, M): int32, or float16 when x_scale is given."""
        return _ext.spmm(self.handle, self.M, X, N, x_scale, out, stream)

    def spmm_requant(self, X16, N: int, x_amax, out=None, y_amax=None, amax_range=None, stream=None):
        """X16: device float16 tensor or view, (N, K) with unit column stride; x_amax: absmax buffer
        from absmax_f16 or an earlier call's y_amax. Returns the (N, M) float16 output; if y_amax
        (an absmax buffer) is given it receives the absmax of columns amax_range of the output."""
        m0, m1 = amax_range if amax_range is not None else (0, self.M)
        return _ext.spmm_requant(self.handle, self.M, self.K, X16, N, x_amax, out, y_amax, m0, m1, stream)

    def check(self):
        st = us_last_error(self.handle)
        _check(st, "us_last_error")

    def close(self):
        if self.handle:
            us_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- MX4: dense matrices in microscaled 4-bit floating point ----

def mx4_bytes(rows: int, K: int) -> int:
    """Bytes of device memory that the tiles of a rows x K matrix take."""
    n = int(_lib.us_mx4_bytes(int(rows), int(K)))
    if n < 0:
        raise UsError(1, "us_mx4_bytes")
    return n


class Mx4:
    """A dense (rows, K) matrix of E2M1 values with a power-of-two scale for 32 columns of a row, on a CUDA device, in the library's
    tiles (``data``, uint8). Made by ``mx4_quantize`` and ``mx4_from_codes``."""

    __slots__ = ("rows", "K", "data", "frozen", "__weakref__")

    def __init__(self, rows: int, K: int, data=None, device="cuda"):
        import torch
        _native()
        need = mx4_bytes(rows, K)
        if data is None:
            data = torch.empty(need, device=device, dtype=torch.uint8)
        elif data.dtype != torch.uint8 or data.numel() != need or not data.is_contiguous() or not data.is_cuda:
            raise ValueError(f"data must be {need} contiguous bytes (uint8) on a CUDA device")
        self.rows, self.K, self.data, self.frozen = int(rows), int(K), data, False

    def freeze(self):
        """Declares the matrix complete and constant (a weight): waits for its device, and from then on products may read it while
        the stream's earlier work still runs. Not during a stream capture. Returns the matrix."""
        import torch
        torch.cuda.synchronize(self.data.device)
        self.frozen = True
        return self

    def dequantize(self, dtype=None, out=None, stream=None):
        """The (rows, K) values, float32 unless another type is asked for (float16 may overflow). bfloat16 holds them exactly."""
        return _ext.mx4_dequantize(self.data, self.rows, self.K, dtype, out, stream)

    def codes(self, stream=None):
        """(codes uint8 (rows, ceil(K/2)), even column in the low nibble; scale bytes uint8 (rows, ceil(K/32)))."""
        return _ext.mx4_unpack(self.data, self.rows, self.K, stream)


def mx4_quantize(X, out: Mx4 | None = None, stream=None) -> Mx4:
    """MX4 form of a device float16, bfloat16 or float32 (rows, K) tensor or view (unit column stride). An `out` that is given is
    written over (not one that is frozen)."""
    ext = _ext or _native()
    if out is None:
        m = Mx4.__new__(Mx4)
        m.data, m.rows, m.K = ext.mx4_quantize(X, None, stream)
        m.frozen = False
        return m
    if out.frozen or (out.rows, out.K) != tuple(X.shape):
        raise ValueError("out must be an unfrozen Mx4 of X's shape")
    ext.mx4_quantize(X, out.data, stream)
    return out


def mx4_from_codes(codes, scales, K: int, stream=None) -> Mx4:
    """A matrix from E2M1 codes (uint8 (rows, ceil(K/2)), even column in the low nibble) and scale bytes (uint8 (rows, ceil(K/32))),
    both on the device with unit column stride: a checkpoint's weight. The result is frozen (the call waits for the device)."""
    m = Mx4.__new__(Mx4)
    m.rows, m.K, m.frozen = int(codes.shape[0]), int(K), False
    m.data = (_ext or _native()).mx4_pack(codes, scales, K, stream)
    return m.freeze()


ACTIVATIONS = {None: 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


def mx4_linear(X, w: Mx4, out=None, dtype=None, stream=None, bias=None, act=None, gated=False, residual=None):
    """(N, M) product of activations and the transposed (M, K) weight. X: device float16, bfloat16 or float32 (N, K) tensor or view
    (unit column stride), quantised to MX4 within the call, or an Mx4. The result has `dtype`, by default X's (float16 for an Mx4);
    `out` may have any row stride.

    What follows the product is done on its sums: y = act(x w^T + bias) + residual. act: None, "relu", "silu", "gelu" or "gelu_tanh". gated: rows
    2 j and 2 j + 1 of w (and of bias) are gate and up projection of column j, y = act(gate) * up + residual, (N, M / 2). bias (M,) and residual (N, columns of the
    result; any row stride) may be of any of the three types; the residual may be `out` itself, and otherwise does not overlap it."""
    ext = _ext or _native()
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {list(ACTIVATIONS)}")
    if isinstance(X, Mx4):
        if X.K != w.K:
            raise ValueError("X and w differ in K")
        return ext.mx4_linear(X.data, X.rows, w.data, w.rows, w.K, out, dtype, w.frozen, stream, bias, ACTIVATIONS[act], gated, residual)
    return ext.mx4_linear(X, -1, w.data, w.rows, w.K, out, dtype, w.frozen, stream, bias, ACTIVATIONS[act], gated, residual)


def mx4_check():
    """Waits for the current device and raises if a product on it gave up a bounded wait."""
    _check(_lib.us_mx4_last_error(), "us_mx4_last_error")


# ---- norms and rotation of heads ----

class Rotary:
    """How positions turn the heads of queries and keys: pair i of the first `rotary_dim` values (all `head_dim` unless given) by position * base ** (-2 i /
    rotary_dim), or by `frequencies` (radians a place, one for each pair). Pairs are (i, i + rotary_dim / 2), or neighbours (2 i, 2 i + 1) if `interleaved`.

    Positions with several axes (time, height, width): `sections`, how many pairs each axis turns, in order (a list of rotary_dim / 2 in all), or
    `pair_axis`, the axis of each pair. The table lies on the device, complete and constant (the constructor waits for it)."""

    def __init__(self, head_dim: int, base: float = 10000.0, rotary_dim: int | None = None, interleaved: bool = False, sections=None, pair_axis=None,
                 frequencies=None, device="cuda"):
        import torch
        rotary_dim = head_dim if rotary_dim is None else int(rotary_dim)
        if not 2 <= head_dim <= 256 or head_dim % 2 or not 2 <= rotary_dim <= head_dim or rotary_dim % 2:
            raise ValueError("head_dim must be even and at most 256, rotary_dim even and at most head_dim")
        pairs = rotary_dim // 2
        f = [float(x) for x in frequencies] if frequencies is not None else [float(base) ** (-2.0 * i / rotary_dim) for i in range(pairs)]
        if len(f) != pairs or not all(np.isfinite(f)):
            raise ValueError(f"{pairs} finite frequencies are needed")
        if sections is not None and pair_axis is not None:
            raise ValueError("sections or pair_axis, not both")
        if sections is not None:
            if any(int(n) < 0 for n in sections):
                raise ValueError("sections are numbers of pairs")
            pair_axis = [a for a, n in enumerate(sections) for _ in range(int(n))]
        axes = 1 if pair_axis is None else len(sections) if sections is not None else max(pair_axis, default=-1) + 1
        if pair_axis is not None and (len(pair_axis) != pairs or not 1 <= axes <= 255 or not all(0 <= int(a) < axes for a in pair_axis)):
            raise ValueError(f"an axis for each of the {pairs} pairs is needed, 255 axes at most")
        self.head_dim, self.rotary_dim, self.interleaved, self.axes = int(head_dim), rotary_dim, bool(interleaved), int(axes)
        # turns a place, in units of 2^-64: the quotient's 53 bits, of which whole turns are left out
        turns = [int(np.ldexp(abs(x) / (2 * np.pi) % 1.0, 64)) * (1 if x >= 0 else -1) % (1 << 64) for x in f]
        self.turns = torch.from_numpy(np.array(turns, dtype=np.uint64).view(np.int64)).to(device)
        self.pair_axis = torch.tensor([int(a) for a in pair_axis], dtype=torch.uint8).to(device) if self.axes > 1 else None
        if self.turns.is_cuda:
            torch.cuda.synchronize(self.turns.device)
        self._struct = us_rotary(self.turns.data_ptr(), self.pair_axis.data_ptr() if self.axes > 1 else None, rotary_dim, self.axes, self.interleaved)
        self._address = ctypes.addressof(self._struct)


def qk_norm_rope(q, k, positions, rotary: Rotary, q_weight=None, k_weight=None, eps: float = 1e-6, q_out=None, k_out=None, stream=None):
    """(q, k) with every head normed (x / sqrt(mean x^2 + eps) * weight; a part without a weight is not) and turned to its position, in one pass. q (N, n_heads,
    head_dim), k (N, n_kv_heads, head_dim) or None: float16, bfloat16 or float32, any token and head strides: columns of a stacked projection's output
    need no copy. positions: int32 (N,), or (axes, N) for a rotary of several axes; any value. Weights: (head_dim,) of any of the types. q_out and k_out
    may be q and k themselves."""
    return (_ext or _native()).qk_norm_rope(q, k, positions, rotary._address, rotary.turns, rotary.head_dim, q_weight, k_weight, eps, q_out, k_out, stream)


# ---- the cache of keys and values in 8 bits ----

def us_kv_create(k_codes_ptr: int, v_codes_ptr: int, k_steps_ptr: int, v_steps_ptr: int, n_blocks: int, n_kv_heads: int, block_tokens: int,
                 head_dim: int) -> int:
    """Raw call: device pointers as integers. Returns the handle; the memory stays the caller's."""
    h = _vp()
    _check(_lib.us_kv_create(k_codes_ptr, v_codes_ptr, k_steps_ptr, v_steps_ptr, int(n_blocks), int(n_kv_heads), int(block_tokens), int(head_dim),
                             ctypes.byref(h)), "us_kv_create")
    return h.value


class KVCache:
    """Keys and values of a pool of token blocks as int8 codes with a float32 step for each (block, head): value = code * step.

    Device tensors, contiguous: codes (n_blocks, n_kv_heads, block_tokens, head_dim), steps (n_blocks, n_kv_heads). block_tokens 16, 32,
    64, 128 or 256; head_dim 64 or 128. The tensors are the caller's to copy, move between blocks or save.

    The calls take a batch of sequences: block_table (S, width) int32, the sequence's blocks in order; lengths (S,) int32, this call's new
    tokens included; cu_tokens (S + 1,) int32, where each sequence's rows begin among the call's, or None for one row each."""

    def __init__(self, k_codes, v_codes, k_steps, v_steps):
        import torch
        self.handle = None
        _native()
        for c in (k_codes, v_codes):
            if c.dtype != torch.int8 or c.dim() != 4 or not c.is_contiguous() or not c.is_cuda or c.shape != k_codes.shape or c.device != k_codes.device:
                raise ValueError("codes must be two contiguous int8 (n_blocks, n_kv_heads, block_tokens, head_dim) tensors on one CUDA device")
        for s in (k_steps, v_steps):
            if s.dtype != torch.float32 or tuple(s.shape) != tuple(k_codes.shape[:2]) or not s.is_contiguous() or s.device != k_codes.device:
                raise ValueError("steps must be two contiguous float32 (n_blocks, n_kv_heads) tensors on the codes' device")
        self.k_codes, self.v_codes, self.k_steps, self.v_steps = k_codes, v_codes, k_steps, v_steps
        self.n_blocks, self.n_kv_heads, self.block_tokens, self.head_dim = k_codes.shape
        self.handle = us_kv_create(k_codes.data_ptr(), v_codes.data_ptr(), k_steps.data_ptr(), v_steps.data_ptr(), self.n_blocks, self.n_kv_heads,
                                   self.block_tokens, self.head_dim)

    @classmethod
    def new(cls, n_blocks: int, n_kv_heads: int, head_dim: int, block_tokens: int = 64, device="cuda"):
        """A pool of its own memory, all zero."""
        import torch
        codes = [torch.zeros((n_blocks, n_kv_heads, block_tokens, head_dim), dtype=torch.int8, device=device) for _ in range(2)]
        steps = [torch.zeros((n_blocks, n_kv_heads), dtype=torch.float32, device=device) for _ in range(2)]
        return cls(*codes, *steps)

    def append(self, k, v, block_table, lengths, cu_tokens=None, stream=None, granted=None):
        """Writes new tokens, the last ones of their sequences: k, v (N, n_kv_heads, head_dim) float16, bfloat16 or float32 (any token and
        head strides). Finite values are expected; others do not count for a step. granted: what `KVPages.extend` wrote there: sequences that it had no room
        for are left out."""
        _ext.kv_append(self.handle, self.k_codes, k, v, block_table, lengths, cu_tokens, stream, granted)

    def read(self, block_table, lengths, tokens: int, dtype=None, stream=None):
        """(K, V): values of the first `tokens` places of each sequence, (S, tokens, n_kv_heads, head_dim), float32 unless another type is
        asked for; zero behind a sequence's end."""
        return _ext.kv_read(self.handle, self.k_codes, block_table, lengths, int(tokens), dtype, stream)

    def attention(self, q, block_table, lengths, cu_tokens=None, scale=None, causal=True, window=0, out=None, lse=None, stream=None):
        """Attention of q (N, n_heads, head_dim), float16 or bfloat16, over the sequences' cached tokens, their new ones (appended before)
        included. scale: head_dim ** -0.5 unless given. causal: a token sees itself and those before it, else its whole sequence;
        window > 0: none further back than window - 1. out: like q; lse: float32 (N, n_heads), gets the logarithm of the softmax's sum.

        The softmax's weights have 11 bits in the product with V; what is left is multiplied, too, for float16 and up to 32 rows (tokens x
        query heads) a sequence and cache head."""
        return _ext.kv_attention(self.handle, self.k_codes, q, block_table, lengths, cu_tokens, self.head_dim ** -0.5 if scale is None else scale,
                                 causal, window, out, lse, stream)

    def shared_attention(self, q, prefix_table, prefix_lengths, cu_seqs, block_table, lengths, cu_tokens=None, scale=None, causal=True, out=None, lse=None,
                         stream=None):
        """Attention of sequences behind prefixes that groups of them share: a prefix's keys and values are read once for its group. prefix_table (groups, width)
        and prefix_lengths (groups,) describe the prefixes, cu_seqs int32 (groups + 1,) says whose sequences are whose: [cu_seqs[g], cu_seqs[g + 1]). block_table, lengths
        and cu_tokens are of the sequences' own tokens, the new ones included; the rest is as for `attention`, but that what the softmax's weights have
        beyond 11 bits is multiplied for float16 and any number of rows.

        After `KVPages.fork` of a prompt of p whole blocks: prefix_table = table[:1, :p], block_table = table[:, p:], lengths - p * block_tokens. The tables' widths, not
        the lengths on the device, say which kernels run: columns that no sequence needs (table[:, p:p + n] has n) make a call slower where own contexts are short."""
        return _ext.kv_shared_attention(self.handle, self.k_codes, q, block_table, lengths, cu_tokens, self.head_dim ** -0.5 if scale is None else scale,
                                        causal, 0, out, lse, stream, prefix_table, prefix_lengths, cu_seqs)

    def copy_blocks(self, src, dst, stream=None):
        """Copies block src[i], its codes and steps, to block dst[i] (int32 tensors; dst[i] = -1: nothing). No block is twice in dst, or in dst and src."""
        _ext.kv_copy_blocks(self.handle, self.k_codes, src, dst, stream)

    def check(self):
        """Waits for the device and raises if a call on it met a block number, length or token count out of range."""
        import torch
        with torch.cuda.device(self.k_codes.device):
            _check(_lib.us_kv_last_error(), "us_kv_last_error")

    def close(self):
        if self.handle:
            _lib.us_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KVPages:
    """Which blocks of a cache are in use: `refs`, int32 (n_blocks,) on the cache's device, how many table entries hold each. Sequences may share blocks; a
    block that nobody holds is free. Calls that need free blocks take the lowest ones, sequence by sequence. Nothing waits for the host, and every call can
    be captured into a graph; calls on one KVPages follow one another on the device.

    A batch starts with a table of zeros and lengths of 0; `extend` makes room for new tokens, `KVCache.append` then writes them. Both take `granted` (int32 (S,)):
    `extend` leaves there by how many tokens each sequence has grown, and `append` passes over those that the pool had no room for. Without it the last
    tokens of such a sequence, which are old ones and may lie in blocks of others, would be written over."""

    def __init__(self, cache: KVCache, refs=None):
        import torch
        if refs is None:
            refs = torch.zeros(cache.n_blocks, dtype=torch.int32, device=cache.k_codes.device)
        elif refs.dtype != torch.int32 or tuple(refs.shape) != (cache.n_blocks,) or not refs.is_contiguous() or refs.device != cache.k_codes.device or refs.data_ptr() % 16:
            raise ValueError("refs must be a contiguous int32 (n_blocks,) tensor on the cache's device, 16-byte aligned")
        self.cache, self.refs = cache, refs

    def extend(self, block_table, lengths, tokens=1, stream=None, granted=None):
        """Room for `tokens` (a number, or int32 (S,)) more tokens of each sequence: block_table and lengths are written. A last block that would be written into
        and that others hold, too, is replaced by a copy. Sequences for which the pool has no blocks left stay as they are (see `check`). granted, an int32 (S,)
        tensor, gets how many tokens each has grown by: tokens - granted are still to come once blocks are free."""
        _ext.kv_extend(self.cache.handle, self.cache.k_codes, self.refs, block_table, lengths, tokens, stream, granted)

    def fork(self, block_table, lengths, parents, keep=False, stream=None):
        """(block_table, lengths) of a new batch: row i continues sequence parents[i] (int32; -1: an empty one) and shares its blocks. The old batch is given up
        unless `keep`. Beams are reordered, samples of a prompt begun, and finished sequences dropped this way."""
        return _ext.kv_fork(self.cache.handle, self.cache.k_codes, self.refs, block_table, lengths, parents, keep, stream)

    def release(self, block_table, lengths, stream=None):
        """Gives the sequences' blocks up; those that nobody else holds are free from then on. The tensors are left as they are."""
        _ext.kv_release(self.cache.handle, self.cache.k_codes, self.refs, block_table, lengths, stream)

    def compact(self, tables, stream=None):
        """Moves the blocks in use to the front of the pool. tables: (block_table, lengths) pairs, every table that is in use: their entries are rewritten. Returns how
        many blocks are in use, an int32 scalar on the device."""
        return _ext.kv_compact(self.cache.handle, self.cache.k_codes, self.refs, tuple((t, n) for t, n in tables), stream)

    def check(self):
        """Waits for the device and raises if the pool had too few free blocks, or a call met an entry, length or count out of range."""
        self.cache.check()
