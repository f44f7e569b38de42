"""ctypes binding of libiv.so: the same entry points as include/iv.h.

Argument marshalling only.  Tensors are torch CUDA tensors (torch supplies
device memory and streams); every step of the path runs inside the library's
kernels.  There is no fallback: if the shared library is missing, loading
raises with the build command.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libiv.so")

IV_OK = 0
IV_ERR_INVALID_ARG = -1
IV_ERR_NOMEM = -2
IV_ERR_CUDA = -3
IV_ERR_NO_DEVICE = -4
IV_ERR_TOO_LARGE = -5
NOALLOC_MAX_LEAVES = 512 * 512

EXPORTS = (
    "iv_create", "iv_destroy", "iv_strerror", "iv_last_cuda_error", "iv_kernel_launches",
    "iv_hash_chunks", "iv_merkle_root", "iv_verify_manifest", "iv_ctx_digests",
    "iv_verify_streamed", "iv_hash_ragged", "iv_set_timing", "iv_phase_times", "iv_probe_alu", "iv_device_status",
    "iv_merkle_root_noalloc", "iv_last_leaf_kernel", "iv_last_leaf_instance", "iv_selftest_wait_timeout", "iv_merkle_levels",
    "iv_tree_records", "iv_tree_build", "iv_tree_update",
    "iv_hash_chunks_two_level", "iv_verify_manifest_two_level", "iv_hash_ragged_update", "iv_verify_manifest_batch",
    "iv_hash_chunks_sha384", "iv_merkle_root_sha384", "iv_verify_manifest_sha384",
    "iv_hash_chunks_sha512", "iv_merkle_root_sha512", "iv_verify_manifest_sha512",
    "iv_hash_chunks_rfc6962", "iv_merkle_root_rfc6962", "iv_verify_manifest_rfc6962",
    "iv_embedding", "iv_embedding_grad", "iv_embedding_grad_rows", "iv_grad_norm", "iv_grad_clip", "iv_grad_scale",
    "iv_layer_norm", "iv_layer_norm_grad", "iv_adamw_step",
)

ADAMW_BLOCK = 256          # IV_ADAMW_BLOCK

# iv_dtype of the training-step operators
DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


class IvError(RuntimeError):
    def __init__(self, code: int, what: str, cuda_error: int = 0):
        self.code = code
        self.cuda_error = cuda_error
        extra = f" (cudaError {cuda_error})" if cuda_error else ""
        super().__init__(f"{what}: {_strerror(code)}{extra}")


class Manifest(ctypes.Structure):
    """iv_manifest: host struct, digest array on the device."""
    _fields_ = [("total_bytes", ctypes.c_uint64), ("chunk_bytes", ctypes.c_uint64),
                ("n_chunks", ctypes.c_uint64), ("d_digests", ctypes.c_void_p),
                ("root", ctypes.c_uint8 * 32)]


class Manifest384(ctypes.Structure):
    """iv_manifest_sha384: host struct, 48-byte digest records on the device."""
    _fields_ = [("total_bytes", ctypes.c_uint64), ("chunk_bytes", ctypes.c_uint64),
                ("n_chunks", ctypes.c_uint64), ("d_digests", ctypes.c_void_p),
                ("root", ctypes.c_uint8 * 48)]


class VerifyResult384(ctypes.Structure):
    """iv_verify_result_sha384 as laid out in device memory (64 bytes)."""
    _fields_ = [("status", ctypes.c_uint32), ("root_ok", ctypes.c_uint32),
                ("n_mismatch", ctypes.c_uint64), ("root", ctypes.c_uint8 * 48)]


class Manifest512(ctypes.Structure):
    """iv_manifest_sha512: host struct, 64-byte digest records on the device."""
    _fields_ = [("total_bytes", ctypes.c_uint64), ("chunk_bytes", ctypes.c_uint64),
                ("n_chunks", ctypes.c_uint64), ("d_digests", ctypes.c_void_p),
                ("root", ctypes.c_uint8 * 64)]


class VerifyResult512(ctypes.Structure):
    """iv_verify_result_sha512 as laid out in device memory (80 bytes)."""
    _fields_ = [("status", ctypes.c_uint32), ("root_ok", ctypes.c_uint32),
                ("n_mismatch", ctypes.c_uint64), ("root", ctypes.c_uint8 * 64)]


class VerifyResult(ctypes.Structure):
    """iv_verify_result as laid out in device memory (48 bytes)."""
    _fields_ = [("status", ctypes.c_uint32), ("root_ok", ctypes.c_uint32),
                ("n_mismatch", ctypes.c_uint64), ("root", ctypes.c_uint8 * 32)]


class NormResult(ctypes.Structure):
    """iv_norm_result as laid out in device memory (32 bytes)."""
    _fields_ = [("status", ctypes.c_uint32), ("n_nonfinite", ctypes.c_uint32), ("norm", ctypes.c_float),
                ("scale", ctypes.c_float), ("sum_squares", ctypes.c_double), ("n_elements", ctypes.c_uint64)]


class AdamwOptions(ctypes.Structure):
    """iv_adamw_options: host struct."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("max_norm", ctypes.c_float), ("stochastic", ctypes.c_uint32),
                ("seed", ctypes.c_uint64)]


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads libiv.so from the package directory; raises if it was not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2510_23938_b200.build` "
            "(needs nvcc; there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, u64, i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int
    lib.iv_create.argtypes = [ctypes.POINTER(vp), i32]
    lib.iv_create.restype = i32
    lib.iv_destroy.argtypes = [vp]
    lib.iv_destroy.restype = i32
    lib.iv_strerror.argtypes = [i32]
    lib.iv_strerror.restype = ctypes.c_char_p
    lib.iv_last_cuda_error.argtypes = [vp]
    lib.iv_last_cuda_error.restype = i32
    lib.iv_kernel_launches.argtypes = [vp]
    lib.iv_kernel_launches.restype = u64
    lib.iv_hash_chunks.argtypes = [vp, vp, u64, u64, vp, u64, ctypes.POINTER(u64), vp]
    lib.iv_hash_chunks.restype = i32
    lib.iv_merkle_root.argtypes = [vp, vp, u64, vp, vp]
    lib.iv_merkle_root.restype = i32
    lib.iv_merkle_levels.argtypes = [vp, vp, u64, ctypes.c_uint32, vp, u64, ctypes.POINTER(u64), vp]
    lib.iv_merkle_levels.restype = i32
    lib.iv_tree_records.argtypes = [u64]
    lib.iv_tree_records.restype = u64
    lib.iv_tree_build.argtypes = [vp, vp, u64, vp, u64, vp]
    lib.iv_tree_build.restype = i32
    lib.iv_tree_update.argtypes = [vp, vp, u64, u64, vp, u64, vp, u64, vp]
    lib.iv_tree_update.restype = i32
    lib.iv_hash_chunks_two_level.argtypes = [vp, vp, u64, u64, u64, vp, u64, ctypes.POINTER(u64), vp]
    lib.iv_hash_chunks_two_level.restype = i32
    lib.iv_verify_manifest_two_level.argtypes = [vp, vp, u64, ctypes.POINTER(Manifest), u64, vp, vp, u64, vp]
    lib.iv_verify_manifest_two_level.restype = i32
    lib.iv_hash_ragged_update.argtypes = [vp, vp, vp, vp, u64, vp, i32, vp, vp]
    lib.iv_hash_ragged_update.restype = i32
    lib.iv_verify_manifest_batch.argtypes = [vp, ctypes.POINTER(vp), u64, u64, ctypes.POINTER(Manifest), vp, vp, u64, vp]
    lib.iv_verify_manifest_batch.restype = i32
    lib.iv_hash_chunks_sha384.argtypes = [vp, vp, u64, u64, vp, u64, ctypes.POINTER(u64), vp]
    lib.iv_hash_chunks_sha384.restype = i32
    lib.iv_merkle_root_sha384.argtypes = [vp, vp, u64, vp, vp]
    lib.iv_merkle_root_sha384.restype = i32
    lib.iv_hash_chunks_sha512.argtypes = [vp, vp, u64, u64, vp, u64, ctypes.POINTER(u64), vp]
    lib.iv_hash_chunks_sha512.restype = i32
    lib.iv_merkle_root_sha512.argtypes = [vp, vp, u64, vp, vp]
    lib.iv_merkle_root_sha512.restype = i32
    lib.iv_verify_manifest_sha512.argtypes = [vp, vp, u64, ctypes.POINTER(Manifest512), vp, vp, u64, vp]
    lib.iv_verify_manifest_sha512.restype = i32
    lib.iv_verify_manifest_rfc6962.argtypes = [vp, vp, u64, ctypes.POINTER(Manifest), vp, vp, u64, vp]
    lib.iv_verify_manifest_rfc6962.restype = i32
    lib.iv_verify_manifest_sha384.argtypes = [vp, vp, u64, ctypes.POINTER(Manifest384), vp, vp, u64, vp]
    lib.iv_verify_manifest_sha384.restype = i32
    lib.iv_hash_chunks_rfc6962.argtypes = [vp, vp, u64, u64, vp, u64, ctypes.POINTER(u64), vp]
    lib.iv_hash_chunks_rfc6962.restype = i32
    lib.iv_merkle_root_rfc6962.argtypes = [vp, vp, u64, vp, vp]
    lib.iv_merkle_root_rfc6962.restype = i32
    lib.iv_verify_manifest.argtypes = [vp, vp, u64, ctypes.POINTER(Manifest), vp, vp, u64, vp]
    lib.iv_verify_manifest.restype = i32
    lib.iv_ctx_digests.argtypes = [vp]
    lib.iv_ctx_digests.restype = vp
    lib.iv_verify_streamed.argtypes = [vp, ctypes.POINTER(vp), u64, u64, u64, ctypes.POINTER(Manifest),
                                       vp, vp, u64, vp]
    lib.iv_verify_streamed.restype = i32
    lib.iv_set_timing.argtypes = [vp, i32]
    lib.iv_set_timing.restype = i32
    lib.iv_phase_times.argtypes = [vp, ctypes.c_uint32, ctypes.POINTER(ctypes.c_float)]
    lib.iv_phase_times.restype = i32
    lib.iv_hash_ragged.argtypes = [vp, vp, vp, vp, u64, vp, vp]
    lib.iv_hash_ragged.restype = i32
    lib.iv_merkle_root_noalloc.argtypes = [vp, u64, vp, vp]
    lib.iv_merkle_root_noalloc.restype = i32
    lib.iv_last_leaf_kernel.argtypes = [vp]
    lib.iv_last_leaf_kernel.restype = ctypes.c_char_p
    lib.iv_last_leaf_instance.argtypes = [vp]
    lib.iv_last_leaf_instance.restype = ctypes.c_char_p
    lib.iv_selftest_wait_timeout.argtypes = [vp, u64, ctypes.POINTER(u64), vp]
    lib.iv_selftest_wait_timeout.restype = i32
    lib.iv_device_status.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32)]
    lib.iv_device_status.restype = i32
    lib.iv_probe_alu.argtypes = [vp, i32, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint32,
                                 ctypes.POINTER(ctypes.c_double)]
    lib.iv_probe_alu.restype = i32
    i64, f32 = ctypes.c_int64, ctypes.c_float
    lib.iv_embedding.argtypes = [vp, vp, i32, u64, u64, u64, vp, i32, u64, f32, vp, i32, u64, vp]
    lib.iv_embedding.restype = i32
    lib.iv_embedding_grad.argtypes = [vp, vp, i32, u64, u64, vp, i32, u64, u64, i64, f32, i32, vp, i32, u64, vp]
    lib.iv_embedding_grad.restype = i32
    lib.iv_embedding_grad_rows.argtypes = [vp, vp, i32, u64, u64, vp, i32, u64, u64, i64, f32, vp, vp, i32, u64, u64, vp, vp]
    lib.iv_embedding_grad_rows.restype = i32
    lib.iv_grad_norm.argtypes = [vp, vp, vp, vp, vp, i32, u64, vp, vp, vp]
    lib.iv_grad_norm.restype = i32
    lib.iv_grad_clip.argtypes = [vp, vp, vp, vp, vp, i32, u64, f32, vp, vp, i32, vp, vp, vp]
    lib.iv_grad_clip.restype = i32
    lib.iv_grad_scale.argtypes = [vp, vp, vp, vp, vp, i32, u64, vp, vp, vp, i32, vp]
    lib.iv_grad_scale.restype = i32
    lib.iv_layer_norm.argtypes = [vp, vp, i32, u64, u64, u64, vp, vp, i32, f32, i32, vp, i32, u64, vp, vp, vp]
    lib.iv_layer_norm.restype = i32
    lib.iv_layer_norm_grad.argtypes = [vp, vp, i32, u64, vp, i32, u64, u64, u64, vp, i32, vp, vp, i32, vp, u64, vp, vp, i32,
                                       i32, vp]
    lib.iv_layer_norm_grad.restype = i32
    lib.iv_adamw_step.argtypes = [vp, vp, vp, vp, i32, u64, vp, vp, i32, vp, u64, i32, vp, vp, vp, vp, vp,
                                  ctypes.POINTER(AdamwOptions), vp, vp, vp, vp]
    lib.iv_adamw_step.restype = i32
    _lib = lib
    return lib


def _strerror(code: int) -> str:
    try:
        return load_library().iv_strerror(code).decode()
    except Exception:  # pragma: no cover
        return f"status {code}"


def n_chunks(nbytes: int, chunk_bytes: int) -> int:
    return 0 if nbytes == 0 else (nbytes - 1) // chunk_bytes + 1


# A device's current stream's handle without a Stream object around it (0.3 us a call against 3.2); no public
# interface, so a torch without it takes the other way.
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _current_raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _current_raw_stream(torch.cuda.current_device())


def _dev_ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None or t.numel() == 0:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return t.data_ptr()


def _nbytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def _ptr(t: torch.Tensor) -> int:
    assert t.is_cuda, "device tensors must be CUDA tensors"
    return t.data_ptr()


def _matrix(t: torch.Tensor) -> tuple:
    """(device pointer, rows, columns, elements from one row to the next) of a tensor whose rows are contiguous."""
    assert t.is_cuda, "device tensors must be CUDA tensors"
    rows, dim = t.shape
    stride, unit = t.stride()
    assert unit == 1 or dim <= 1, "rows must be contiguous"
    return t.data_ptr(), rows, dim, stride if rows > 1 else dim


def _rows_of(t: torch.Tensor, n: int, dim: int) -> tuple:
    """(device pointer, elements from one row to the next) of n rows of `dim` elements."""
    assert t.is_cuda, "device tensors must be CUDA tensors"
    if t.dim() == 2:
        rows, columns = t.shape
        assert rows == n and columns == dim, "wrong number of rows or columns"
        stride, unit = t.stride()
        assert unit == 1 or dim <= 1, "rows must be contiguous"
        return t.data_ptr(), stride if n > 1 else dim
    assert t.is_contiguous() and t.numel() == n * dim and t.shape[-1] == dim, "wrong number of rows or columns"
    return t.data_ptr(), dim


def _vector_ptr(t: Optional[torch.Tensor], n: int, dtype: Optional[torch.dtype] = None) -> Optional[int]:
    """Device pointer of n contiguous elements (of `dtype`), None for no tensor."""
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous() and t.numel() == n, "must be a contiguous CUDA tensor of one element per place"
    assert dtype is None or t.dtype is dtype, "wrong type of elements"
    return t.data_ptr()


def _int64_ptr(t: torch.Tensor, n: int) -> Optional[int]:
    """Device pointer of n int64 numbers, None if n is 0."""
    assert t.dtype is torch.int64 and t.numel() == n, "offsets, lengths and places: one int64 per tensor"
    if n == 0:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return t.data_ptr()


def _token_bytes(tokens: torch.Tensor) -> int:
    assert tokens.dtype in (torch.int32, torch.int64), "tokens are int32 or int64"
    return tokens.element_size()


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _result_ptr(result: torch.Tensor) -> int:
    assert result.is_cuda and result.is_contiguous() and _nbytes(result) >= ctypes.sizeof(NormResult)
    return result.data_ptr()


def _out_args(out, out_offsets, out_dtype, types, n):
    """(d_out, d_out_offsets, out_type) of iv_grad_clip and iv_grad_scale."""
    if out is None:
        assert out_offsets is None and out_dtype is None, "in place needs no output arguments"
        return None, None, -1
    assert out_offsets is not None and out_offsets.dtype == torch.int64 and out_offsets.numel() == n, \
        "out needs out_offsets: one int64 byte offset per tensor"
    code = DTYPES[out_dtype] if out_dtype is not None else (DTYPES[out.dtype] if types is None else -1)
    return _ptr(out), _dev_ptr(out_offsets), code


class Context:
    """iv_ctx: scratch memory and streams of one verifier on one device."""

    def __init__(self, device: int | None = None):
        lib = load_library()
        if device is None:
            device = torch.cuda.current_device() if torch.cuda.is_available() else 0
        self.device = int(device)
        handle = ctypes.c_void_p()
        rc = lib.iv_create(ctypes.byref(handle), self.device)
        if rc != IV_OK:
            raise IvError(rc, "iv_create")
        self._h = handle
        self._lib = lib

    # -- plumbing ---------------------------------------------------------------------------
    def close(self):
        if getattr(self, "_h", None):
            self._lib.iv_destroy(self._h)
            self._h = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _check(self, rc: int, what: str):
        if rc != IV_OK:
            raise IvError(rc, what, self._lib.iv_last_cuda_error(self._h))

    @property
    def kernel_launches(self) -> int:
        return int(self._lib.iv_kernel_launches(self._h))

    # -- entry points -----------------------------------------------------------------------
    def hash_chunks(self, data: torch.Tensor, chunk_bytes: int, out: torch.Tensor | None = None,
                    nbytes: int | None = None, stream=None) -> torch.Tensor:
        """iv_hash_chunks: (n, 32) uint8 digests of the chunks of `data` (any dtype, read as bytes)."""
        nb = _nbytes(data) if nbytes is None else int(nbytes)
        n = n_chunks(nb, chunk_bytes) if chunk_bytes > 0 else 0
        if out is None:
            out = torch.empty((n, 32), dtype=torch.uint8, device=data.device)
        got = ctypes.c_uint64(0)
        rc = self._lib.iv_hash_chunks(self._h, _dev_ptr(data), nb, chunk_bytes, _dev_ptr(out),
                                      out.numel() // 32, ctypes.byref(got), _stream_ptr(stream))
        self._check(rc, "iv_hash_chunks")
        return out[:got.value]

    def hash_chunks_two_level(self, data: torch.Tensor, chunk_bytes: int, sub_bytes: int, stream=None,
                              out: torch.Tensor | None = None) -> torch.Tensor:
        """iv_hash_chunks_two_level: digest i = Merkle root over the SHA-256 digests of chunk i's sub_bytes pieces."""
        nb = _nbytes(data)
        n = n_chunks(nb, chunk_bytes) if chunk_bytes > 0 else 0
        if out is None:
            out = torch.empty((n, 32), dtype=torch.uint8, device=data.device)
        got = ctypes.c_uint64(0)
        rc = self._lib.iv_hash_chunks_two_level(self._h, _dev_ptr(data), nb, chunk_bytes, sub_bytes, _dev_ptr(out), n,
                                                ctypes.byref(got), _stream_ptr(stream))
        self._check(rc, "iv_hash_chunks_two_level")
        return out[:got.value]

    def verify_manifest_two_level(self, data: torch.Tensor, manifest: Manifest, sub_bytes: int, result: torch.Tensor,
                                  mismatch_idx: torch.Tensor | None, stream=None) -> None:
        """iv_verify_manifest_two_level (asynchronous); the manifest must hold two-level digests."""
        cap = 0 if mismatch_idx is None else mismatch_idx.numel()
        rc = self._lib.iv_verify_manifest_two_level(self._h, _dev_ptr(data), _nbytes(data), ctypes.byref(manifest),
                                                    sub_bytes, _dev_ptr(result), _dev_ptr(mismatch_idx), cap,
                                                    _stream_ptr(stream))
        self._check(rc, "iv_verify_manifest_two_level")

    def merkle_root(self, leaves: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """iv_merkle_root: 32-byte root (uint8 tensor on the device) of (n, 32) leaf digests."""
        n = leaves.numel() // 32
        if out is None:
            out = torch.empty(32, dtype=torch.uint8, device=leaves.device)
        rc = self._lib.iv_merkle_root(self._h, _dev_ptr(leaves), n, _dev_ptr(out), _stream_ptr(stream))
        self._check(rc, "iv_merkle_root")
        return out

    def hash_chunks_sha384(self, data: torch.Tensor, chunk_bytes: int, stream=None,
                           out: torch.Tensor | None = None) -> torch.Tensor:
        """iv_hash_chunks_sha384: (n, 48) uint8 SHA-384 digests of the chunks of `data`."""
        nb = _nbytes(data)
        n = n_chunks(nb, chunk_bytes) if chunk_bytes > 0 else 0
        if out is None:
            out = torch.empty((n, 48), dtype=torch.uint8, device=data.device)
        got = ctypes.c_uint64(0)
        rc = self._lib.iv_hash_chunks_sha384(self._h, _dev_ptr(data), nb, chunk_bytes, _dev_ptr(out), n,
                                             ctypes.byref(got), _stream_ptr(stream))
        self._check(rc, "iv_hash_chunks_sha384")
        return out[:got.value]

    def merkle_root_sha384(self, leaves: torch.Tensor, stream=None, out: torch.Tensor | None = None) -> torch.Tensor:
        """iv_merkle_root_sha384: 48-byte root of (n, 48) leaf digests."""
        n = leaves.numel() // 48
        if out is None:
            out = torch.empty(48, dtype=torch.uint8, device=leaves.device)
        rc = self._lib.iv_merkle_root_sha384(self._h, _dev_ptr(leaves), n, _dev_ptr(out), _stream_ptr(stream))
        self._check(rc, "iv_merkle_root_sha384")
        return out

    def hash_chunks_sha512(self, data: torch.Tensor, chunk_bytes: int, stream=None,
                           out: torch.Tensor | None = None) -> torch.Tensor:
        """iv_hash_chunks_sha512: (n, 64) uint8 SHA-512 digests of the chunks of `data`."""
        nb = _nbytes(data)
        n = n_chunks(nb, chunk_bytes) if chunk_bytes > 0 else 0
        if out is None:
            out = torch.empty((n, 64), dtype=torch.uint8, device=data.device)
        got = ctypes.c_uint64(0)
        rc = self._lib.iv_hash_chunks_sha512(self._h, _dev_ptr(data), nb, chunk_bytes, _dev_ptr(out), n,
                                             ctypes.byref(got), _stream_ptr(stream))
        self._check(rc, "iv_hash_chunks_sha512")
        return out[:got.value]

    def merkle_root_sha512(self, leaves: torch.Tensor, stream=None, out: torch.Tensor | None = None) -> torch.Tensor:
        """iv_merkle_root_sha512: 64-byte root of (n, 64) leaf digests."""
        n = leaves.numel() // 64
        if out is None:
            out = torch.empty(64, dtype=torch.uint8, device=leaves.device)
        rc = self._lib.iv_merkle_root_sha512(self._h, _dev_ptr(leaves), n, _dev_ptr(out), _stream_ptr(stream))
        self._check(rc, "iv_merkle_root_sha512")
        return out

    def verify_manifest_sha384(self, data: torch.Tensor, total_bytes: int, chunk_bytes: int, digests: torch.Tensor,
                               root: bytes, mismatch_idx: torch.Tensor | None = None, stream=None) -> dict:
        """iv_verify_manifest_sha384: verifies `data` against SHA-384 chunk digests (an (n, 48) device tensor) and
        the 48-byte root; waits for the result and returns it as a dict (status, root_ok, n_mismatch, root)."""
        m = Manifest384()
        m.total_bytes, m.chunk_bytes, m.n_chunks = total_bytes, chunk_bytes, digests.numel() // 48
        m.d_digests = _dev_ptr(digests)
        m.root = (ctypes.c_uint8 * 48).from_buffer_copy(root)
        result = torch.zeros(ctypes.sizeof(VerifyResult384), dtype=torch.uint8, device=data.device)
        cap = 0 if mismatch_idx is None else mismatch_idx.numel()
        rc = self._lib.iv_verify_manifest_sha384(self._h, _dev_ptr(data), _nbytes(data), ctypes.byref(m), _dev_ptr(result),
                                                 _dev_ptr(mismatch_idx), cap, _stream_ptr(stream))
        self._check(rc, "iv_verify_manifest_sha384")
        r = VerifyResult384.from_buffer_copy(bytes(result.cpu().numpy().tobytes()))
        return {"status": int(r.status), "root_ok": bool(r.root_ok), "n_mismatch": int(r.n_mismatch), "root": bytes(r.root)}

    def verify_manifest_sha512(self, data: torch.Tensor, total_bytes: int, chunk_bytes: int, digests: torch.Tensor,
                               root: bytes, mismatch_idx: torch.Tensor | None = None, stream=None) -> dict:
        """iv_verify_manifest_sha512: as verify_manifest_sha384 with (n, 64) digests and a 64-byte root."""
        m = Manifest512()
        m.total_bytes, m.chunk_bytes, m.n_chunks = total_bytes, chunk_bytes, digests.numel() // 64
        m.d_digests = _dev_ptr(digests)
        m.root = (ctypes.c_uint8 * 64).from_buffer_copy(root)
        result = torch.zeros(ctypes.sizeof(VerifyResult512), dtype=torch.uint8, device=data.device)
        cap = 0 if mismatch_idx is None else mismatch_idx.numel()
        rc = self._lib.iv_verify_manifest_sha512(self._h, _dev_ptr(data), _nbytes(data), ctypes.byref(m), _dev_ptr(result),
                                                 _dev_ptr(mismatch_idx), cap, _stream_ptr(stream))
        self._check(rc, "iv_verify_manifest_sha512")
        r = VerifyResult512.from_buffer_copy(bytes(result.cpu().numpy().tobytes()))
        return {"status": int(r.status), "root_ok": bool(r.root_ok), "n_mismatch": int(r.n_mismatch), "root": bytes(r.root)}

    def hash_chunks_rfc6962(self, data: torch.Tensor, chunk_bytes: int, stream=None,
                            out: torch.Tensor | None = None) -> torch.Tensor:
        """iv_hash_chunks_rfc6962: (n, 32) uint8 leaf hashes SHA-256(0x00 || chunk)."""
        nb = _nbytes(data)
        n = n_chunks(nb, chunk_bytes) if chunk_bytes > 0 else 0
        if out is None:
            out = torch.empty((n, 32), dtype=torch.uint8, device=data.device)
        got = ctypes.c_uint64(0)
        rc = self._lib.iv_hash_chunks_rfc6962(self._h, _dev_ptr(data), nb, chunk_bytes, _dev_ptr(out), n,
                                              ctypes.byref(got), _stream_ptr(stream))
        self._check(rc, "iv_hash_chunks_rfc6962")
        return out[:got.value]

    def merkle_root_rfc6962(self, leaves: torch.Tensor, stream=None, out: torch.Tensor | None = None) -> torch.Tensor:
        """iv_merkle_root_rfc6962: 32-byte root with 0x01-prefixed nodes over (n, 32) leaf hashes."""
        n = leaves.numel() // 32
        if out is None:
            out = torch.empty(32, dtype=torch.uint8, device=leaves.device)
        rc = self._lib.iv_merkle_root_rfc6962(self._h, _dev_ptr(leaves), n, _dev_ptr(out), _stream_ptr(stream))
        self._check(rc, "iv_merkle_root_rfc6962")
        return out

    def merkle_levels(self, nodes: torch.Tensor, levels: int, stream=None, out: torch.Tensor | None = None) -> torch.Tensor:
        """iv_merkle_levels: the (ceil(n / 2^levels), 32) nodes `levels` levels above `nodes`."""
        n = nodes.numel() // 32
        n_out = n
        for _ in range(levels):
            if n_out <= 1:
                break
            n_out = (n_out + 1) // 2
        if out is None:
            out = torch.empty((n_out, 32), dtype=torch.uint8, device=nodes.device)
        got = ctypes.c_uint64(0)
        rc = self._lib.iv_merkle_levels(self._h, _dev_ptr(nodes), n, levels, _dev_ptr(out), n_out,
                                        ctypes.byref(got), _stream_ptr(stream))
        self._check(rc, "iv_merkle_levels")
        assert got.value == n_out
        return out

    def tree_records(self, n_leaves: int) -> int:
        return int(self._lib.iv_tree_records(n_leaves))

    def tree_build(self, leaves: torch.Tensor, stream=None, out: torch.Tensor | None = None) -> torch.Tensor:
        """iv_tree_build: the retained tree (iv_tree_records(n), 32) of the (n, 32) leaf digests; root = tree[-1]."""
        n = leaves.numel() // 32
        records = int(self._lib.iv_tree_records(n))
        tree = torch.empty((records, 32), dtype=torch.uint8, device=leaves.device) if out is None else out
        rc = self._lib.iv_tree_build(self._h, _dev_ptr(leaves), n, _dev_ptr(tree), records, _stream_ptr(stream))
        self._check(rc, "iv_tree_build")
        return tree

    def tree_update(self, data: torch.Tensor, chunk_bytes: int, dirty: torch.Tensor, tree: torch.Tensor,
                    stream=None) -> None:
        """iv_tree_update: re-hash the chunks whose indices are in the int64 device tensor `dirty`."""
        assert dirty.dtype == torch.int64
        rc = self._lib.iv_tree_update(self._h, _dev_ptr(data), _nbytes(data), chunk_bytes, _dev_ptr(dirty),
                                      dirty.numel(), _dev_ptr(tree), tree.numel() // 32, _stream_ptr(stream))
        self._check(rc, "iv_tree_update")

    def make_manifest(self, total_bytes: int, chunk_bytes: int, digests: torch.Tensor, root: bytes) -> Manifest:
        m = Manifest()
        m.total_bytes = total_bytes
        m.chunk_bytes = chunk_bytes
        m.n_chunks = digests.numel() // 32
        m.d_digests = _dev_ptr(digests)
        m.root = (ctypes.c_uint8 * 32).from_buffer_copy(root)
        m._keepalive = digests
        return m

    def verify_manifest(self, data: torch.Tensor, manifest: Manifest, result: torch.Tensor,
                        mismatch_idx: torch.Tensor | None, nbytes: int | None = None, stream=None) -> None:
        """iv_verify_manifest (asynchronous): `result` is a 48-byte uint8 device tensor,
        `mismatch_idx` an int64 device tensor whose length is the index capacity."""
        nb = _nbytes(data) if nbytes is None else int(nbytes)
        cap = 0 if mismatch_idx is None else mismatch_idx.numel()
        rc = self._lib.iv_verify_manifest(self._h, _dev_ptr(data), nb, ctypes.byref(manifest),
                                          _dev_ptr(result), _dev_ptr(mismatch_idx), cap, _stream_ptr(stream))
        self._check(rc, "iv_verify_manifest")

    def verify_manifest_rfc6962(self, data: torch.Tensor, manifest: Manifest, result: torch.Tensor,
                                mismatch_idx: torch.Tensor | None, stream=None) -> None:
        """iv_verify_manifest_rfc6962 (asynchronous); the manifest holds prefixed leaf hashes and their root."""
        cap = 0 if mismatch_idx is None else mismatch_idx.numel()
        rc = self._lib.iv_verify_manifest_rfc6962(self._h, _dev_ptr(data), _nbytes(data), ctypes.byref(manifest),
                                                  _dev_ptr(result), _dev_ptr(mismatch_idx), cap, _stream_ptr(stream))
        self._check(rc, "iv_verify_manifest_rfc6962")

    def verify_manifest_batch(self, blobs: list, manifest: Manifest, results: torch.Tensor,
                              mismatch_idx: torch.Tensor | None, stream=None) -> None:
        """iv_verify_manifest_batch (asynchronous): `blobs` are equally sized device tensors, `results` a
        (len(blobs), 48) uint8 device tensor, `mismatch_idx` a (len(blobs), cap) int64 device tensor."""
        nb = _nbytes(blobs[0])
        assert all(_nbytes(b) == nb and b.is_cuda and b.is_contiguous() for b in blobs)
        ptrs = (ctypes.c_void_p * len(blobs))(*[b.data_ptr() for b in blobs])
        cap = 0 if mismatch_idx is None else mismatch_idx.shape[1]
        rc = self._lib.iv_verify_manifest_batch(self._h, ptrs, len(blobs), nb, ctypes.byref(manifest), _dev_ptr(results),
                                                _dev_ptr(mismatch_idx), cap, _stream_ptr(stream))
        self._check(rc, "iv_verify_manifest_batch")

    def verify_streamed(self, host_windows, window_bytes: int, nbytes: int, manifest: Manifest,
                        result: torch.Tensor, mismatch_idx: torch.Tensor | None, stream=None) -> None:
        """iv_verify_streamed (asynchronous).  `host_windows` is a CPU uint8 tensor holding the whole
        blob, or a list of CPU tensors, one per window (pinned for overlap; entries may repeat)."""
        if isinstance(host_windows, torch.Tensor):
            flat = host_windows.view(torch.uint8).reshape(-1)
            assert not flat.is_cuda and flat.is_contiguous() and flat.numel() >= nbytes
            host_windows = [flat[o:o + window_bytes] for o in range(0, nbytes, window_bytes)] if window_bytes > 0 else []
        n_win = len(host_windows)
        ptrs = (ctypes.c_void_p * max(n_win, 1))()
        for w, t in enumerate(host_windows):
            assert not t.is_cuda and t.is_contiguous()
            ptrs[w] = t.data_ptr()
        cap = 0 if mismatch_idx is None else mismatch_idx.numel()
        rc = self._lib.iv_verify_streamed(self._h, ptrs, n_win, window_bytes, nbytes, ctypes.byref(manifest),
                                          _dev_ptr(result), _dev_ptr(mismatch_idx), cap, _stream_ptr(stream))
        self._check(rc, "iv_verify_streamed")

    def set_timing(self, enabled: bool) -> None:
        self._check(self._lib.iv_set_timing(self._h, int(enabled)), "iv_set_timing")

    def phase_times(self, calls_back: int = 0) -> tuple[float, float, float]:
        """iv_phase_times: (hash, tree, compare) milliseconds of a recent verification call."""
        ms = (ctypes.c_float * 3)()
        self._check(self._lib.iv_phase_times(self._h, calls_back, ms), "iv_phase_times")
        return float(ms[0]), float(ms[1]), float(ms[2])

    def hash_ragged(self, base: torch.Tensor, offsets: torch.Tensor, lengths: torch.Tensor,
                    out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """iv_hash_ragged: (n, 32) digests of base[offset_k : offset_k + length_k) (offsets/lengths int64 on device)."""
        n = offsets.numel()
        assert lengths.numel() == n and offsets.dtype == torch.int64 and lengths.dtype == torch.int64
        if out is None:
            out = torch.empty((n, 32), dtype=torch.uint8, device=base.device)
        rc = self._lib.iv_hash_ragged(self._h, _dev_ptr(base), _dev_ptr(offsets), _dev_ptr(lengths), n,
                                      _dev_ptr(out), _stream_ptr(stream))
        self._check(rc, "iv_hash_ragged")
        return out

    @property
    def last_leaf_kernel(self) -> str:
        return self._lib.iv_last_leaf_kernel(self._h).decode()

    @property
    def last_leaf_instance(self) -> str:
        return self._lib.iv_last_leaf_instance(self._h).decode()

    def selftest_wait_timeout(self, limit_cycles: int, stream=None) -> int:
        """iv_selftest_wait_timeout: a warp waits `limit_cycles` SM clocks on a barrier nobody arrives at, gives
        up and sets the device status to 1; returns the clocks it waited (synchronises the stream)."""
        waited = ctypes.c_uint64(0)
        rc = self._lib.iv_selftest_wait_timeout(self._h, int(limit_cycles), ctypes.byref(waited), _stream_ptr(stream))
        self._check(rc, "iv_selftest_wait_timeout")
        return int(waited.value)

    def device_status(self) -> int:
        """iv_device_status: waits for the device, returns and clears the device-side status word."""
        st = ctypes.c_uint32(0)
        self._check(self._lib.iv_device_status(self._h, ctypes.byref(st)), "iv_device_status")
        return int(st.value)

    PROBE_KINDS = {"iadd3": 0, "lop3": 1, "shf": 2, "prmt": 3, "imad": 4, "mixed": 5, "sha256": 6, "sha256_sched_fma": 7,
                   "lat_iadd3": 8, "lat_lop3": 9, "lat_shf": 10, "lat_imad": 11, "lat_cross": 12,
                   "rounds": 13, "schedule": 14}

    def probe_alu(self, kind: str, warps_per_block: int = 4, blocks_per_sm: int = 1, active_lanes: int = 32,
                  iters: int = 2000) -> tuple[float, float]:
        """iv_probe_alu: (lane-ops or bytes per clock per SM, mean cycles per block)."""
        out = (ctypes.c_double * 2)()
        rc = self._lib.iv_probe_alu(self._h, self.PROBE_KINDS[kind], warps_per_block, blocks_per_sm,
                                    active_lanes, iters, out)
        self._check(rc, "iv_probe_alu")
        return float(out[0]), float(out[1])

    SHA_STATE_BYTES = 48

    def new_sha_states(self, n: int) -> torch.Tensor:
        """Zero-filled iv_sha_state records for n tensors (an (n, 48) uint8 device tensor)."""
        return torch.zeros((n, self.SHA_STATE_BYTES), dtype=torch.uint8, device=f"cuda:{self.device}")

    def hash_ragged_update(self, base: torch.Tensor, offsets: torch.Tensor, lengths: torch.Tensor,
                           states: torch.Tensor, finish: bool, out: torch.Tensor | None = None, stream=None):
        """iv_hash_ragged_update: hash the next part of every tensor; returns the (n, 32) digests when finishing."""
        n = offsets.numel()
        assert lengths.numel() == n and states.numel() == n * self.SHA_STATE_BYTES
        if finish and out is None:
            out = torch.empty((n, 32), dtype=torch.uint8, device=base.device)
        rc = self._lib.iv_hash_ragged_update(self._h, _dev_ptr(base) or base.data_ptr(), _dev_ptr(offsets),
                                             _dev_ptr(lengths), n, _dev_ptr(states), int(finish),
                                             _dev_ptr(out) if out is not None else None, _stream_ptr(stream))
        self._check(rc, "iv_hash_ragged_update")
        return out if finish else None

    # -- training-step operators --------------------------------------------------------------
    # Tensors the calls allocate come from the stream the work runs on; a caller that passes `stream` keeps its other
    # tensors alive until that stream has reached the work, as everywhere in this binding.

    def embedding(self, table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, out: torch.Tensor | None = None,
                  out_dtype: torch.dtype | None = None, stream=None) -> torch.Tensor:
        """iv_embedding: scale * table[tokens] (tokens int32 or int64, any shape), rounded once to `out_dtype`
        (default: the table's).  `table` is (rows, dim) with contiguous rows, at any element alignment."""
        table_ptr, rows, dim, row_stride = _matrix(table)
        if out is None:
            out = _empty((*tokens.shape, dim), out_dtype or table.dtype, table.device, stream)
        n = tokens.numel()
        out_ptr, out_stride = _rows_of(out, n, dim)
        rc = self._lib.iv_embedding(self._h, table_ptr, DTYPES[table.dtype], rows, dim, row_stride, _dev_ptr(tokens),
                                    _token_bytes(tokens), n, scale, out_ptr, DTYPES[out.dtype], out_stride,
                                    _stream_ptr(stream))
        if rc:
            self._check(rc, "iv_embedding")
        return out

    def embedding_grad(self, grad_out: torch.Tensor, tokens: torch.Tensor, n_rows: int, scale: float = 1.0,
                       padding_row: int | None = None, out: torch.Tensor | None = None,
                       out_dtype: torch.dtype | None = None, accumulate: bool = False, stream=None) -> torch.Tensor:
        """iv_embedding_grad: the (n_rows, dim) gradient of `embedding`'s table, `grad_out` (..., dim) being the
        gradient of its result; with `accumulate`, added to `out`."""
        dim, n = grad_out.shape[-1], tokens.numel()
        grad_ptr, grad_stride = _rows_of(grad_out, n, dim)
        if out is None:
            assert not accumulate, "accumulate needs the gradient to add to"
            out = _empty((n_rows, dim), out_dtype or grad_out.dtype, grad_out.device, stream)
        out_ptr, out_rows, out_dim, out_stride = _matrix(out)
        assert (out_rows, out_dim) == (n_rows, dim), "out must be (n_rows, dim)"
        rc = self._lib.iv_embedding_grad(self._h, grad_ptr, DTYPES[grad_out.dtype], grad_stride, dim,
                                         _dev_ptr(tokens), _token_bytes(tokens), n, n_rows,
                                         -1 if padding_row is None else padding_row, scale, accumulate, out_ptr,
                                         DTYPES[out.dtype], out_stride, _stream_ptr(stream))
        if rc:
            self._check(rc, "iv_embedding_grad")
        return out

    def embedding_grad_rows(self, grad_out: torch.Tensor, tokens: torch.Tensor, n_rows: int, scale: float = 1.0,
                            padding_row: int | None = None, rows: torch.Tensor | None = None,
                            out: torch.Tensor | None = None, count: torch.Tensor | None = None,
                            out_dtype: torch.dtype | None = None, stream=None):
        """iv_embedding_grad_rows: (rows, grad, count) -- the distinct rows ascending (int64, -1 behind them), their
        gradients (zero rows behind them) and their number (int64, on the device).  min(tokens, n_rows) rows in all."""
        dim, n = grad_out.shape[-1], tokens.numel()
        grad_ptr, grad_stride = _rows_of(grad_out, n, dim)
        cap = min(n, n_rows) if out is None else out.shape[0]
        if out is None:
            out = _empty((cap, dim), out_dtype or grad_out.dtype, grad_out.device, stream)
        if rows is None:
            rows = _empty((cap,), torch.int64, grad_out.device, stream)
        if count is None:
            count = _empty((1,), torch.int64, grad_out.device, stream)
        out_ptr, _, out_dim, out_stride = _matrix(out)
        assert out_dim == dim and rows.numel() == cap and rows.dtype == count.dtype == torch.int64 and count.numel() == 1
        assert rows.is_cuda and rows.is_contiguous() and count.is_cuda
        count_ptr = count.data_ptr()
        rc = self._lib.iv_embedding_grad_rows(self._h, grad_ptr, DTYPES[grad_out.dtype], grad_stride, dim,
                                              _dev_ptr(tokens), _token_bytes(tokens), n, n_rows,
                                              -1 if padding_row is None else padding_row, scale,
                                              rows.data_ptr() or count_ptr, out_ptr, DTYPES[out.dtype], out_stride, cap,
                                              count_ptr, _stream_ptr(stream))
        if rc:
            self._check(rc, "iv_embedding_grad_rows")
        return rows, out, count

    def _set_args(self, base, offsets, lengths, dtype, types):
        n = offsets.numel()
        assert lengths.numel() == n and offsets.dtype == lengths.dtype == torch.int64
        if types is not None:
            assert types.dtype == torch.uint8 and types.numel() == n
        return (_ptr(base), _dev_ptr(offsets), _dev_ptr(lengths), _dev_ptr(types),
                DTYPES[base.dtype if dtype is None else dtype] if types is None else 0, n)

    def grad_norm(self, base: torch.Tensor, offsets: torch.Tensor, lengths: torch.Tensor, result: torch.Tensor,
                  norms: torch.Tensor | None = None, dtype: torch.dtype | None = None,
                  types: torch.Tensor | None = None, stream=None) -> None:
        """iv_grad_norm (asynchronous): `offsets`, `lengths` in bytes as for hash_ragged (see tensor_ranges for tensors
        of their own); `result` is a 32-byte uint8 device tensor (new_norm_result, read_norm_result), `norms` an
        optional float32 tensor for the tensors' own norms; element type `dtype` (default: base's) or `types`, one
        DTYPES code per tensor (uint8)."""
        args = self._set_args(base, offsets, lengths, dtype, types)
        assert norms is None or (norms.dtype == torch.float32 and norms.numel() == args[-1])
        rc = self._lib.iv_grad_norm(self._h, *args, _dev_ptr(norms), _result_ptr(result), _stream_ptr(stream))
        self._check(rc, "iv_grad_norm")

    def grad_clip(self, base: torch.Tensor, offsets: torch.Tensor, lengths: torch.Tensor, max_norm: float,
                  result: torch.Tensor, norms: torch.Tensor | None = None, out: torch.Tensor | None = None,
                  out_offsets: torch.Tensor | None = None, dtype: torch.dtype | None = None,
                  types: torch.Tensor | None = None, out_dtype: torch.dtype | None = None, stream=None) -> None:
        """iv_grad_clip (asynchronous): grad_norm, then every tensor times min(1, max_norm / norm), in place or to
        `out` + `out_offsets` (bytes) as `out_dtype` (default: out's type, or with `types` each tensor's own)."""
        args = self._set_args(base, offsets, lengths, dtype, types)
        assert norms is None or (norms.dtype == torch.float32 and norms.numel() == args[-1])
        rc = self._lib.iv_grad_clip(self._h, *args, max_norm, *_out_args(out, out_offsets, out_dtype, types, args[-1]),
                                    _dev_ptr(norms), _result_ptr(result), _stream_ptr(stream))
        self._check(rc, "iv_grad_clip")

    def grad_scale(self, base: torch.Tensor, offsets: torch.Tensor, lengths: torch.Tensor, scale: torch.Tensor,
                   out: torch.Tensor | None = None, out_offsets: torch.Tensor | None = None,
                   dtype: torch.dtype | None = None, types: torch.Tensor | None = None,
                   out_dtype: torch.dtype | None = None, stream=None) -> None:
        """iv_grad_scale (asynchronous): every tensor times the float32 device scalar `scale`; output as grad_clip."""
        args = self._set_args(base, offsets, lengths, dtype, types)
        assert scale.is_cuda and scale.dtype == torch.float32 and scale.numel() == 1
        rc = self._lib.iv_grad_scale(self._h, *args, scale.data_ptr(),
                                     *_out_args(out, out_offsets, out_dtype, types, args[-1]), _stream_ptr(stream))
        self._check(rc, "iv_grad_scale")

    def layer_norm(self, x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
                   eps: float = 1e-5, rms: bool = False, out: torch.Tensor | None = None,
                   out_dtype: torch.dtype | None = None, mean: torch.Tensor | None = None,
                   rstd: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """iv_layer_norm over the last dimension of `x` (a matrix with contiguous rows, or a contiguous tensor of more
        dimensions): (x - mean) * rstd * weight + bias, rounded once to `out_dtype` (default: x's); `rms`: without the
        mean.  `mean` and `rstd` (float32, one per row) receive what `layer_norm_grad` wants."""
        dim = x.shape[-1]
        n = x.numel() // dim if dim else math.prod(x.shape[:-1])
        x_ptr, x_stride = _rows_of(x, n, dim)
        if out is None:
            out = _empty(x.shape, out_dtype or x.dtype, x.device, stream)
        out_ptr, out_stride = _rows_of(out, n, dim)
        param, weight_ptr, bias_ptr = 0, None, None
        if bias is not None:
            assert weight is None or weight.dtype is bias.dtype, "weight and bias are of one type"
            param, bias_ptr = DTYPES[bias.dtype], _vector_ptr(bias, dim)
        if weight is not None:
            param, weight_ptr = DTYPES[weight.dtype], _vector_ptr(weight, dim)
        rc = self._lib.iv_layer_norm(self._h, x_ptr, DTYPES[x.dtype], x_stride, n, dim, weight_ptr, bias_ptr, param, eps, rms, out_ptr,
                                     DTYPES[out.dtype], out_stride,
                                     None if mean is None else _vector_ptr(mean, n, torch.float32),
                                     None if rstd is None else _vector_ptr(rstd, n, torch.float32), _stream_ptr(stream))
        if rc:
            self._check(rc, "iv_layer_norm")
        return out

    def layer_norm_grad(self, grad_out: torch.Tensor, x: torch.Tensor, mean: torch.Tensor | None, rstd: torch.Tensor,
                        weight: torch.Tensor | None = None, rms: bool = False, out: torch.Tensor | None = None,
                        weight_grad: torch.Tensor | None = None, bias_grad: torch.Tensor | None = None,
                        accumulate: bool = False, stream=None) -> torch.Tensor:
        """iv_layer_norm_grad: the gradient of `layer_norm`'s x (of x's type), `grad_out` being that of its result;
        `weight_grad` and `bias_grad` (of one type), where given, receive the sums over the rows, or with `accumulate`
        have them added.  `mean` is not read with `rms` and may then be None."""
        dim = x.shape[-1]
        n = x.numel() // dim if dim else math.prod(x.shape[:-1])
        x_ptr, x_stride = _rows_of(x, n, dim)
        grad_ptr, grad_stride = _rows_of(grad_out, n, dim)
        if out is None:
            out = _empty(x.shape, x.dtype, x.device, stream)
        assert out.dtype == x.dtype, "the gradient is of x's type"
        out_ptr, out_stride = _rows_of(out, n, dim)
        sums, weight_grad_ptr, bias_grad_ptr = 0, None, None
        if bias_grad is not None:
            assert weight_grad is None or weight_grad.dtype is bias_grad.dtype, "sums are of one type"
            sums, bias_grad_ptr = DTYPES[bias_grad.dtype], _vector_ptr(bias_grad, dim)
        if weight_grad is not None:
            sums, weight_grad_ptr = DTYPES[weight_grad.dtype], _vector_ptr(weight_grad, dim)
        rc = self._lib.iv_layer_norm_grad(self._h, grad_ptr, DTYPES[grad_out.dtype], grad_stride, x_ptr, DTYPES[x.dtype], x_stride,
                                          n, dim, _vector_ptr(weight, dim), 0 if weight is None else DTYPES[weight.dtype],
                                          None if rms else _vector_ptr(mean, n, torch.float32),
                                          _vector_ptr(rstd, n, torch.float32), rms, out_ptr, out_stride, weight_grad_ptr,
                                          bias_grad_ptr, sums, accumulate, _stream_ptr(stream))
        if rc:
            self._check(rc, "iv_layer_norm_grad")
        return out

    def adamw_step(self, base: torch.Tensor, offsets: torch.Tensor, lengths: torch.Tensor, grads: torch.Tensor,
                   grad_offsets: torch.Tensor, state_offsets: torch.Tensor, m: torch.Tensor, v: torch.Tensor,
                   step: torch.Tensor, m_scales: torch.Tensor | None = None, v_scales: torch.Tensor | None = None,
                   master: torch.Tensor | None = None, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                   weight_decay: float = 1e-2, norm: torch.Tensor | None = None, max_norm: float | None = None,
                   stochastic: bool = False, seed: int = 0, dtype: torch.dtype | None = None,
                   grad_dtype: torch.dtype | None = None, stream=None) -> None:
        """iv_adamw_step (asynchronous), in place: `base`, `offsets`, `lengths` (bytes) give the weights as for grad_norm,
        `grads`, `grad_offsets` (bytes) the gradients; `state_offsets` to `master` are the state as adamw_state makes it
        (`**state`), its moments float32 or float8_e4m3fn.  `lr` is a number or a one-element float32 device tensor, read
        when the step runs.  `norm` is the record of grad_norm over the gradients: they are clipped to `max_norm` on the
        way (None: not clipped), and where one is not finite nothing changes.  `seed` sets the random words that round
        8-bit moments and, with `stochastic`, 16-bit weights.  Types default to those of `base` and `grads`."""
        n, size, kind = offsets.numel(), m.numel(), m.dtype
        tensors = (_int64_ptr(offsets, n), _int64_ptr(lengths, n), _int64_ptr(grad_offsets, n), _int64_ptr(state_offsets, n))
        if kind is torch.float32:
            bits, m_scales_ptr, v_scales_ptr = 32, None, None
        else:
            assert kind is torch.float8_e4m3fn, "moments are float32 or float8_e4m3fn"
            assert m_scales is not None and v_scales is not None, "8-bit moments need their scales"
            bits, blocks = 8, size // ADAMW_BLOCK
            m_scales_ptr = _vector_ptr(m_scales, blocks, torch.float32)
            v_scales_ptr = _vector_ptr(v_scales, blocks, torch.float32)
        assert step.is_cuda and step.dtype is torch.int64 and step.numel() == 1, "step: one int64 on the device"
        assert max_norm is None or norm is not None, "clipping needs the record of the gradients' norm"
        lr_ptr = None
        if isinstance(lr, torch.Tensor):
            assert lr.is_cuda and lr.dtype is torch.float32 and lr.numel() == 1, "lr: a number or one float32 on the device"
            lr_ptr, lr = lr.data_ptr(), 0.0
        assert base.is_cuda and grads.is_cuda, "device tensors must be CUDA tensors"
        options = AdamwOptions(lr, betas[0], betas[1], eps, weight_decay, math.inf if max_norm is None else max_norm, stochastic,
                               seed & 0xffffffffffffffff)
        rc = self._lib.iv_adamw_step(
            self._h, base.data_ptr(), tensors[0], tensors[1], DTYPES[dtype or base.dtype], n, grads.data_ptr(), tensors[2],
            DTYPES[grad_dtype or grads.dtype], tensors[3], size, bits, _vector_ptr(m, size), _vector_ptr(v, size, kind),
            m_scales_ptr, v_scales_ptr, None if master is None else _vector_ptr(master, size, torch.float32), options, lr_ptr,
            None if norm is None else _result_ptr(norm), step.data_ptr(), _stream_ptr(stream))
        if rc:
            self._check(rc, "iv_adamw_step")

    def last_digests(self, n: int) -> torch.Tensor:
        """Copy of the chunk digests the last verification on this context computed."""
        ptr = self._lib.iv_ctx_digests(self._h)
        if not ptr:
            raise RuntimeError("no verification has run on this context")
        if n == 0:
            return torch.empty((0, 32), dtype=torch.uint8, device=f"cuda:{self.device}")
        view = torch.as_tensor(_DeviceBytes(ptr, 32 * n), device=f"cuda:{self.device}")
        return view.clone().view(n, 32)


class _DeviceBytes:
    """Exposes a raw device pointer to torch through the CUDA array interface (no ownership)."""

    def __init__(self, ptr: int, nbytes: int):
        self.__cuda_array_interface__ = {"shape": (nbytes,), "typestr": "|u1", "data": (int(ptr), False),
                                         "version": 2}


def merkle_root_noalloc(leaves: torch.Tensor, out: torch.Tensor, n_leaves: int | None = None, stream=None) -> torch.Tensor:
    """iv_merkle_root_noalloc: Merkle root into the caller's 32-byte device tensor `out`.

    For callers that cannot allocate on the device (a pool owns the GPU, or the allocator must not
    be touched): no context, no allocation in the library, and none here -- both tensors are the
    caller's.  At most NOALLOC_MAX_LEAVES leaves; calls must not overlap on the GPU."""
    lib = load_library()
    n = leaves.numel() // 32 if n_leaves is None else int(n_leaves)
    assert out.is_cuda and out.is_contiguous() and out.numel() >= 32
    rc = lib.iv_merkle_root_noalloc(_dev_ptr(leaves), n, out.data_ptr(), _stream_ptr(stream))
    if rc != IV_OK:
        raise IvError(rc, "iv_merkle_root_noalloc")
    return out


def read_result(result: torch.Tensor) -> dict:
    """Decodes a 48-byte iv_verify_result tensor (synchronises on the copy to the host)."""
    raw = bytes(result.cpu().numpy().tobytes())
    r = VerifyResult.from_buffer_copy(raw)
    return {"status": int(r.status), "root_ok": bool(r.root_ok), "n_mismatch": int(r.n_mismatch),
            "root": bytes(r.root)}


def new_norm_result(device) -> torch.Tensor:
    return torch.zeros(ctypes.sizeof(NormResult), dtype=torch.uint8, device=device)


def read_norm_result(result: torch.Tensor) -> dict:
    """Decodes a 32-byte iv_norm_result tensor (synchronises on the copy to the host)."""
    r = NormResult.from_buffer_copy(bytes(result.cpu().numpy().tobytes()))
    return {name: getattr(r, name) for name, _ in NormResult._fields_}


def tensor_ranges(tensors) -> tuple:
    """(base, offsets, lengths, types) of tensors of their own, as grad_norm, grad_clip and grad_scale take a set: a
    tensor and, per tensor, the bytes from it (modulo 2^64), the length in bytes (int64 device tensors) and the
    DTYPES code.  The arrays hold addresses: they are for these tensors, not for others of the same shapes.  Tensors
    without elements may stand anywhere; they have no address, so the base is the first one that has (or, for a set of
    nothing, an element of its own)."""
    tensors = list(tensors)
    assert all(t.is_cuda and t.is_contiguous() for t in tensors), "device tensors must be contiguous CUDA tensors"
    device = tensors[0].device if tensors else "cuda"
    base = next((t for t in tensors if t.numel()), None)
    if base is None:
        base = torch.zeros(1, device=device)
    signed = [(t.data_ptr() - base.data_ptr() + (1 << 63)) % (1 << 64) - (1 << 63) if t.numel() else 0 for t in tensors]
    return (base, torch.tensor(signed, dtype=torch.int64, device=device),
            torch.tensor([_nbytes(t) for t in tensors], dtype=torch.int64, device=device),
            torch.tensor([DTYPES[t.dtype] for t in tensors], dtype=torch.uint8, device=device))


def adamw_state(elements, device, bits: int = 32, master=False) -> dict:
    """The state of adamw_step for tensors of `elements` elements each (a list of numbers), before the first step: places
    (multiples of ADAMW_BLOCK), moments in 32 or 8 bits, the number of steps and, with `master`, the weights in 32 bits: `master` is
    the list of the weight tensors, which are copied, or True for room that the caller fills before the first step (zeros until
    then, from which a step would set the weights; grad_scale by 1 into `master` at 4 * state_offsets fills it)."""
    assert bits in (8, 32), "moments are held in 8 or 32 bits"
    places, size = [], 0
    for n in elements:
        places.append(size)
        size += -(-int(n) // ADAMW_BLOCK) * ADAMW_BLOCK
    state = {"state_offsets": torch.tensor(places, dtype=torch.int64, device=device),
             "step": torch.zeros(1, dtype=torch.int64, device=device)}
    for name in ("m", "v"):
        if bits == 32:
            state[name] = torch.zeros(size, device=device)
        else:
            state[name] = torch.zeros(size, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
            state[name + "_scales"] = torch.zeros(size // ADAMW_BLOCK, device=device)
    if master is not False:
        state["master"] = torch.zeros(size, device=device)
        if master is not True:
            assert [w.numel() for w in master] == [int(n) for n in elements], "master: one tensor of weights per place"
            for place, w in zip(places, master):
                state["master"][place:place + w.numel()].copy_(w.reshape(-1))
    return state


def read_results(results: torch.Tensor) -> list:
    """Decodes an (n, 48) tensor of iv_verify_result records."""
    raw = results.cpu().numpy().tobytes()
    size = ctypes.sizeof(VerifyResult)
    out = []
    for o in range(0, len(raw), size):
        r = VerifyResult.from_buffer_copy(raw[o:o + size])
        out.append({"status": int(r.status), "root_ok": bool(r.root_ok), "n_mismatch": int(r.n_mismatch),
                    "root": bytes(r.root)})
    return out


def new_result(device) -> torch.Tensor:
    return torch.zeros(ctypes.sizeof(VerifyResult), dtype=torch.uint8, device=device)
