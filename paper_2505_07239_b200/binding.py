"""Thin binding of libcomet_b200.so (the C ABI of include/comet.h): ctypes, and for the calls of every pass the
CPython module _marshal (csrc/marshal.cpp).

Argument marshalling only: every step of the path runs in the library's CUDA
kernels.  Tensors are torch uint64/int64 CUDA tensors or numpy/torch host
arrays; torch is used for device memory and streams and for nothing else.
There is no CPU fallback: if a shared object is missing or fails to load,
importing this module raises.
"""
from __future__ import annotations

import ctypes
import os
import subprocess
from typing import Any, NamedTuple, Optional

import numpy as np
import torch

from .build import LIB_PATH, build_library, is_current

OK = 0
DEVICE, HOST = 0, 1
PATH_AUTO, PATH_SIMT, PATH_LIMB = 0, 1, 2
KERNEL_SIMT, KERNEL_STREAM, KERNEL_LIMB, KERNEL_GROUPED, KERNEL_RESIDUE = 1, 2, 3, 4, 5

(X, W1, WG, W2, A_UP, B_UP, C_UP, H, A_DN, B_DN, C_DN,
 E_UP, F_UP, Z_UP, E_DN, F_DN, Y, W3) = range(18)
NUM_TENSORS = 18

EXPORTS = (
    "comet_init", "comet_destroy", "comet_load_shares", "comet_set_mask", "comet_ffn_up", "comet_ffn_down",
    "comet_truncate", "comet_get", "comet_get_index", "comet_stats", "comet_strerror", "comet_last_cuda_error",
    "comet_set_profiling", "comet_beaver_matmul_static", "comet_shuffle", "comet_invert_permutation",
    "comet_beaver_mul", "comet_set_token_mask", "comet_get_components", "comet_kv_plan",
    "comet_add_bias", "comet_bind_shares", "comet_truncate_pair", "comet_synchronize", "comet_inject_timeout",
    "comet_pipe_probe", "comet_device_pointer", "comet_static_status", "comet_static_inject_timeout",
    "comet_linear", "comet_linear_workspace", "comet_norm_rotate", "comet_linear_attention",
    "comet_linear_attention_workspace", "comet_linear_attention_step", "comet_group_norm", "comet_group_norm_workspace",
)
STATIC_SCRATCH_WORDS = 1 << 20
ERR_SHAPE = -2
ERR_SCRATCH_LIMIT = -7
ERR_TIMEOUT = -6
NUM_PHASES = 5
PHASE_NAMES = ("compact", "open", "prep", "combine", "truncate")


class CometConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "max_tokens", "d_model", "d_ff", "block", "frac_bits", "gated", "device", "max_active", "matmul_path")]


class CometStats(ctypes.Structure):
    _fields_ = [("message_bytes", ctypes.c_int64), ("ring_macs", ctypes.c_int64), ("n_active", ctypes.c_int32),
                ("n_active_blocks", ctypes.c_int32), ("tokens", ctypes.c_int32), ("matmul_path", ctypes.c_int32),
                ("kernel_launches", ctypes.c_int64), ("phase_ms", ctypes.c_double * 5),
                ("phase_launches", ctypes.c_int64 * 5), ("n_components", ctypes.c_int32),
                ("product_kernel", ctypes.c_int32), ("tensor_tile_macs", ctypes.c_int64)]


class CometLinearArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tokens", "inner", "cols", "frac_bits", "quadratic")] + [
        ("k", ctypes.c_uint64 * 3)] + [(n, ctypes.c_void_p * 2) for n in (
            "X", "A", "W", "B", "C", "bias", "residual", "R", "Q", "E", "F", "M", "Y")] + [
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_int64)]


class CometNormRotateArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tokens", "heads", "q_heads", "dim")] + [("x_stride", ctypes.c_int64)] + [
        (n, ctypes.c_int32) for n in ("frac_bits", "steps")] + [(n, ctypes.c_uint64) for n in ("guess", "eps")] + [
        (n, ctypes.c_int32) for n in ("rot_dim", "interleaved", "table_rows")] + [(n, ctypes.c_void_p * 2) for n in (
            "X", "U", "row_words", "UV", "gain", "gain_mask", "A", "C")] + [
        (n, ctypes.c_void_p) for n in ("cos", "sin", "positions")] + [(n, ctypes.c_void_p * 2) for n in ("M", "S", "D", "G", "Z")] + [
        ("bad_index_flag", ctypes.c_void_p)]


class CometLinearAttentionArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tokens", "sequences", "q_heads", "kv_heads", "k_dim", "v_dim", "chunk", "chunks")] + [
        (n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride")] + [("frac_bits", ctypes.c_int32)] + [
        (n, ctypes.c_void_p) for n in ("starts", "decay")] + [(n, ctypes.c_void_p * 2) for n in (
            "Q", "K", "V", "mq", "mk", "mv", "md", "mp", "ms", "qk", "pv", "qs", "dv", "state", "Eq", "Ek", "Ev", "Ed", "Ep", "Es", "O",
            "state_out")] + [("bad_starts_flag", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_int64),
        ("zero_unwritten", ctypes.c_int32)]


class CometLinearAttentionStepArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "q_heads", "kv_heads", "k_dim", "v_dim")] + [
        (n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride")] + [("frac_bits", ctypes.c_int32), ("decay", ctypes.c_void_p)] + [
        (n, ctypes.c_void_p * 2) for n in ("Q", "K", "V", "mq", "mk", "mv", "ms", "kv", "qs", "state", "Eq", "Ek", "Ev", "Es", "O", "state_out")]


class CometGroupNormArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("samples", "positions", "channels", "groups")] + [("x_stride", ctypes.c_int64)] + [
        (n, ctypes.c_int32) for n in ("frac_bits", "steps")] + [(n, ctypes.c_uint64) for n in ("guess", "eps")] + [
        ("quadratic", ctypes.c_int32), ("k", ctypes.c_uint64 * 3)] + [(n, ctypes.c_void_p * 2) for n in (
            "X", "U", "words", "UT", "gain", "gain_mask", "T", "VW", "bias", "R", "Q", "M", "S", "D", "G", "N", "Z")] + [
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_int64)]


class CometError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {_lib.comet_strerror(code).decode()} ({code})")
        self.code = code


def _load():
    if not is_current():
        # missing, or built from other sources than the ones in the tree: rebuild rather than run stale kernels
        try:
            build_library()
        except (OSError, subprocess.CalledProcessError) as exc:
            raise ImportError(
                f"{LIB_PATH} is missing or stale and could not be rebuilt ({exc}); build it with "
                "`python -m paper_2505_07239_b200.build` (there is no CPU fallback)") from exc
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.comet_init.argtypes = [ctypes.POINTER(CometConfig), vp, ctypes.POINTER(vp)]
    lib.comet_destroy.argtypes = [vp]
    lib.comet_destroy.restype = None
    lib.comet_load_shares.argtypes = [vp, ctypes.c_int, ctypes.c_int, vp, ctypes.c_int, i64, i64]
    lib.comet_bind_shares.argtypes = [vp, ctypes.c_int, ctypes.c_int, vp, i64, i64]
    lib.comet_set_mask.argtypes = [vp, vp, ctypes.c_int, i32, ctypes.POINTER(i32)]
    lib.comet_set_token_mask.argtypes = [vp, vp, ctypes.c_int, i32, i32, ctypes.POINTER(i64)]
    lib.comet_get_components.argtypes = [vp, vp, vp, ctypes.c_int, ctypes.POINTER(i32)]
    lib.comet_ffn_up.argtypes = [vp, i32]
    lib.comet_ffn_down.argtypes = [vp, i32]
    lib.comet_truncate.argtypes = [vp, ctypes.c_int]
    lib.comet_get.argtypes = [vp, ctypes.c_int, ctypes.c_int, vp, ctypes.c_int, i64, ctypes.POINTER(i64)]
    lib.comet_get_index.argtypes = [vp, vp, ctypes.c_int, i32, ctypes.POINTER(i32)]
    lib.comet_stats.argtypes = [vp, ctypes.POINTER(CometStats)]
    lib.comet_strerror.argtypes = [ctypes.c_int]
    lib.comet_strerror.restype = ctypes.c_char_p
    lib.comet_last_cuda_error.argtypes = [vp]
    lib.comet_set_profiling.argtypes = [vp, ctypes.c_int]
    lib.comet_synchronize.argtypes = [vp]
    lib.comet_inject_timeout.argtypes = [vp]
    lib.comet_device_pointer.argtypes = [vp, ctypes.c_int, ctypes.c_int, ctypes.POINTER(vp)]
    lib.comet_pipe_probe.argtypes = [vp, ctypes.c_int, i32, i32, ctypes.POINTER(ctypes.c_float),
                                     ctypes.POINTER(ctypes.c_double)]
    pair = ctypes.c_void_p * 2
    lib.comet_beaver_matmul_static.argtypes = [vp, pair, pair, pair, pair, pair, pair, i32, i32, i32]
    lib.comet_static_status.argtypes = [vp]
    lib.comet_static_inject_timeout.argtypes = [vp]
    lib.comet_shuffle.argtypes = [vp, pair, pair, pair, pair, pair, pair, pair, i64, i64, vp]
    lib.comet_invert_permutation.argtypes = [vp, vp, vp, i64, vp]
    lib.comet_add_bias.argtypes = [vp, pair, pair, i64, i64]
    lib.comet_truncate_pair.argtypes = [vp, pair, pair, pair, pair, i64, i32]
    lib.comet_kv_plan.argtypes = [vp, vp, i32, i32, i64, i64, vp, vp, ctypes.POINTER(i32)]
    lib.comet_beaver_mul.argtypes = [vp, pair, pair, pair, pair, pair, pair, pair, pair, i64]
    lib.comet_linear.argtypes = [vp, ctypes.POINTER(CometLinearArgs)]
    lib.comet_linear_workspace.argtypes = [i32, i32, i32, ctypes.POINTER(i64)]
    lib.comet_norm_rotate.argtypes = [vp, ctypes.POINTER(CometNormRotateArgs)]
    lib.comet_linear_attention.argtypes = [vp, ctypes.POINTER(CometLinearAttentionArgs)]
    lib.comet_linear_attention_workspace.argtypes = [i32] * 7 + [ctypes.POINTER(i64)]
    lib.comet_linear_attention_step.argtypes = [vp, ctypes.POINTER(CometLinearAttentionStepArgs)]
    lib.comet_group_norm.argtypes = [vp, ctypes.POINTER(CometGroupNormArgs)]
    lib.comet_group_norm_workspace.argtypes = [i32, i32, i32, i32, ctypes.POINTER(i64)]
    return lib


_lib = _load()
from . import _marshal as _native  # noqa: E402  (built together with the library)


def library():
    """The loaded ctypes library (for tests that poke the raw ABI)."""
    return _lib


def _ptr_loc(t):
    """(address, location, element count) of a torch tensor or numpy array of 8-byte words."""
    if isinstance(t, np.ndarray):
        assert t.flags["C_CONTIGUOUS"] and t.dtype.itemsize == 8
        return t.ctypes.data, HOST, t.size
    assert t.is_contiguous() and t.element_size() == 8
    return t.data_ptr(), (DEVICE if t.is_cuda else HOST), t.numel()


class Comet:
    """One secret-shared FFN layer on one GPU (both parties), over the C ABI."""

    def __init__(self, max_tokens: int, d_model: int, d_ff: int, block: int, frac_bits: int, gated: bool = False,
                 device: int = 0, max_active: int = 0, matmul_path: int = PATH_AUTO,
                 stream: Optional[torch.cuda.Stream] = None):
        self.cfg = CometConfig(max_tokens, d_model, d_ff, block, frac_bits, int(gated), device, max_active,
                               matmul_path)
        self.device = torch.device("cuda", device)
        self.stream = stream
        self._h = ctypes.c_void_p()
        sp = ctypes.c_void_p(stream.cuda_stream if stream is not None else 0)
        self._address = None               # of the context, for the marshalling module
        self._check(_lib.comet_init(ctypes.byref(self.cfg), sp, ctypes.byref(self._h)), "comet_init")
        self._address = self._h.value
        self.groups = int(gated) + 1
        self.n_active = 0

    # ------------------------------------------------------------------ plumbing
    def _check(self, code: int, what: str):
        if code != OK:
            raise CometError(code, what)

    def close(self):
        if self._h:
            _lib.comet_destroy(self._h)
            self._h = ctypes.c_void_p()
            self._address = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def synchronize(self):
        """Wait for the context's work; raises if one of its kernels gave up on a bounded wait."""
        self._check(_lib.comet_synchronize(self._h), "comet_synchronize")

    # ------------------------------------------------------------------ the six calls
    def load_shares(self, party: int, tensor_id: int, t):
        if isinstance(t, torch.Tensor):
            code = _native.load_shares(self._address, party, tensor_id, t)
        else:
            ptr, loc, _ = _ptr_loc(t)
            rows, cols = t.shape
            code = _lib.comet_load_shares(self._h, party, tensor_id, ptr, loc, rows, cols)
        if code:
            raise CometError(code, "comet_load_shares")

    def bind_shares(self, party: int, tensor_id: int, t):
        """Use a CUDA tensor of 8-byte words in place (no copy); the caller keeps it alive and unchanged."""
        code = _native.bind_shares(self._address, party, tensor_id, t)
        if code:
            raise CometError(code, "comet_bind_shares")

    def set_mask(self, mask) -> int:
        if isinstance(mask, np.ndarray):
            code, active = _native.set_mask(self._address, mask)
        else:
            assert mask.dtype == torch.uint8 and mask.is_contiguous()
            n = ctypes.c_int32(0)
            code = _lib.comet_set_mask(self._h, mask.data_ptr(), DEVICE if mask.is_cuda else HOST, mask.numel(),
                                       ctypes.byref(n))
            active = n.value
        if code:
            raise CometError(code, "comet_set_mask")
        self.n_active = active
        return active

    def set_token_mask(self, mask) -> int:
        """Per-token mask over the active blocks, [tokens, n_active_blocks] uint8 (numpy or torch), or None to
        clear it.  Returns the number of non-zero entries of the hidden state under it."""
        masked = ctypes.c_int64(0)
        if mask is None:
            self._check(_lib.comet_set_token_mask(self._h, None, DEVICE, 0, 0, ctypes.byref(masked)),
                        "comet_set_token_mask")
            return 0
        if isinstance(mask, np.ndarray):
            assert mask.dtype == np.uint8 and mask.flags["C_CONTIGUOUS"] and mask.ndim == 2
            ptr, loc = mask.ctypes.data, HOST
        else:
            assert mask.dtype == torch.uint8 and mask.is_contiguous() and mask.dim() == 2
            ptr, loc = mask.data_ptr(), (DEVICE if mask.is_cuda else HOST)
        self._check(_lib.comet_set_token_mask(self._h, ptr, loc, mask.shape[0], mask.shape[1], ctypes.byref(masked)),
                    "comet_set_token_mask")
        return masked.value

    def get_components(self, tokens: int, n_active_blocks: int):
        """(row_label [tokens], blk_label [n_active_blocks], number of components) under the current token mask."""
        rl = torch.empty(tokens, dtype=torch.int32, device=self.device)
        bl = torch.empty(n_active_blocks, dtype=torch.int32, device=self.device)
        cnt = ctypes.c_int32(0)
        self._check(_lib.comet_get_components(self._h, rl.data_ptr(), bl.data_ptr(), DEVICE, ctypes.byref(cnt)),
                    "comet_get_components")
        self.synchronize()
        return rl.cpu().numpy(), bl.cpu().numpy(), cnt.value

    def ffn_up(self, tokens: int):
        code = _native.ffn_up(self._address, tokens)
        if code:
            raise CometError(code, "comet_ffn_up")

    def ffn_down(self, tokens: int):
        code = _native.ffn_down(self._address, tokens)
        if code:
            raise CometError(code, "comet_ffn_down")

    def truncate(self, tensor_id: int):
        code = _native.truncate(self._address, tensor_id)
        if code:
            raise CometError(code, "comet_truncate")

    # ------------------------------------------------------------------ read-back
    def get_into(self, party: int, tensor_id: int, out) -> int:
        """Copy a tensor into caller memory (device tensor, or pinned/pageable host array)."""
        ptr, loc, cap = _ptr_loc(out)
        written = ctypes.c_int64(0)
        self._check(_lib.comet_get(self._h, party, tensor_id, ptr, loc, cap, ctypes.byref(written)), "comet_get")
        return written.value

    def get(self, party: int, tensor_id: int, shape) -> np.ndarray:
        """Read a tensor back to a numpy uint64 array of the given stored shape."""
        out = torch.empty(int(np.prod(shape)), dtype=torch.int64, device=self.device)
        n = self.get_into(party, tensor_id, out)
        self.synchronize()
        assert n == out.numel(), (n, shape)
        return out.cpu().numpy().view(np.uint64).reshape(shape)

    def result_view(self, party: int, tensor_id: int, shape) -> torch.Tensor:
        """The library's own buffer of a result tensor (Z_UP or Y) as a torch int64 tensor of the given stored
        shape, sharing memory with the library (no copy): for in-place collectives between two calls of the path."""
        addr = ctypes.c_void_p()
        self._check(_lib.comet_device_pointer(self._h, party, tensor_id, ctypes.byref(addr)), "comet_device_pointer")

        class _View:                             # the CUDA array interface: address, shape and element type
            __cuda_array_interface__ = {"shape": tuple(int(v) for v in shape), "typestr": "<i8",
                                        "data": (addr.value, False), "version": 2, "strides": None}

        return torch.as_tensor(_View(), device=self.device)

    def get_index(self) -> np.ndarray:
        nb = self.cfg.d_ff // self.cfg.block
        out = torch.empty(nb, dtype=torch.int32, device=self.device)
        cnt = ctypes.c_int32(0)
        self._check(_lib.comet_get_index(self._h, out.data_ptr(), DEVICE, nb, ctypes.byref(cnt)), "comet_get_index")
        self.synchronize()
        return out[:cnt.value].cpu().numpy()

    def set_profiling(self, on: bool):
        self._check(_lib.comet_set_profiling(self._h, int(on)), "comet_set_profiling")

    def stats(self) -> CometStats:
        s = CometStats()
        self._check(_lib.comet_stats(self._h, ctypes.byref(s)), "comet_stats")
        return s


def to_device(a: np.ndarray, device="cuda:0") -> torch.Tensor:
    """numpy uint64 -> torch int64 CUDA tensor holding the same words."""
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int64)).to(device)


def beaver_matmul_static(X, A, Y, B, C, Z, stream: Optional[torch.cuda.Stream] = None) -> int:
    """Allocation-free dense Beaver product for both parties (comet_beaver_matmul_static).

    For callers that cannot allocate device memory when they need the product
    (all memory already owned by a framework's pool, or a serving loop that must
    not stall on cudaMalloc): the message buffers live in an 8 MiB array inside
    the library.  Each argument is a pair (party 0, party 1) of CUDA tensors of
    8-byte words on the current device: X, A [T, K]; Y, B [N, K]; C, Z [T, N].
    Returns the library's status code (0 = ok) instead of raising, so that the
    size-limit refusal can be observed.  Calls that overlap on the GPU race on
    the shared array: keep them on one stream.
    """
    return _native.beaver_matmul_static(stream, X, A, Y, B, C, Z)


def static_status(stream: Optional[torch.cuda.Stream] = None) -> int:
    """Waits for the stream; ERR_TIMEOUT if a beaver_matmul_static, linear or linear_attention call on the current device gave up on a
    bounded wait since this was last asked (comet_static_status), else 0 = ok."""
    return _lib.comet_static_status(ctypes.c_void_p(stream.cuda_stream if stream is not None else 0))


PIPE_TENSOR_I8, PIPE_ALU_U64 = 0, 1


def pipe_probe(pipe: int, launches: int, work: int, stream: Optional[torch.cuda.Stream] = None):
    """Measured rate of a multiply pipe (comet_pipe_probe): returns (ms per launch [launches], multiply-adds per
    launch): 8-bit ones for PIPE_TENSOR_I8, 64-bit ones for PIPE_ALU_U64."""
    ms = (ctypes.c_float * launches)()
    macs = ctypes.c_double(0.0)
    sp = ctypes.c_void_p(stream.cuda_stream if stream is not None else 0)
    code = _lib.comet_pipe_probe(sp, pipe, launches, work, ms, ctypes.byref(macs))
    if code != OK:
        raise CometError(code, "comet_pipe_probe")
    return [float(v) for v in ms], macs.value


def shuffle(X, tau, rho, a, b, stream: Optional[torch.cuda.Stream] = None, bad_index_flag=None):
    """Oblivious shuffle of the rows of a shared matrix (comet_shuffle), both parties.

    Each argument is a pair (party 0, party 1) of CUDA tensors: X, a, b of 8-byte
    words with the same shape [rows, ...]; tau, rho int32 of length rows.
    Returns (Y, Z): the two messages and the two shares of pi(x).  Only the
    output tensors are allocated here (torch); the arithmetic is the library's.
    """
    code, Y, Z = _native.shuffle(stream, X, tau, rho, a, b, bad_index_flag)
    if code:
        raise CometError(code, "comet_shuffle")
    return Y, Z


def invert_permutation(perm, stream: Optional[torch.cuda.Stream] = None, bad_index_flag=None):
    """inverse[perm[j]] = j on the device (comet_invert_permutation)."""
    code, out = _native.invert_permutation(stream, perm, bad_index_flag)
    if code:
        raise CometError(code, "comet_invert_permutation")
    return out


def beaver_mul(X, Y, A, B, C, stream: Optional[torch.cuda.Stream] = None):
    """Element-wise Beaver product of two shared tensors (comet_beaver_mul), both parties.
    Every argument is a pair of equally shaped CUDA tensors of 8-byte words.
    Returns (D, E, Z): the messages x - a and y - b, and the shares of x * y."""
    code, D, E, Z = _native.beaver_mul(stream, X, Y, A, B, C)
    if code:
        raise CometError(code, "comet_beaver_mul")
    return D, E, Z


def truncate_pair(Z, R, RP, frac_bits: int, stream: Optional[torch.cuda.Stream] = None):
    """Truncation with a dealer's pair (comet_truncate_pair), both parties: Z is replaced by shares of
    floor(z / 2^frac_bits) (or one less).  Z, R, RP are pairs of equally shaped CUDA tensors of 8-byte words.
    Returns the messages M = Z - R (a pair)."""
    code, M = _native.truncate_pair(stream, Z, R, RP, frac_bits)
    if code:
        raise CometError(code, "comet_truncate_pair")
    return M


def kv_plan(present: np.ndarray, active: np.ndarray, x: int, w: int):
    """KV-cache manager's request planning (comet_kv_plan, host logic): returns (request [tokens, heads] uint8,
    prefetch [heads] uint8, L1).  `request` is the per-token head mask of the merged refill + prefetch batch."""
    present = np.ascontiguousarray(present, dtype=np.uint8)
    active = np.ascontiguousarray(active, dtype=np.uint8)
    tokens, heads = present.shape
    request = np.empty((tokens, heads), np.uint8)
    prefetch = np.empty(heads, np.uint8)
    l1 = ctypes.c_int32(0)
    code = _lib.comet_kv_plan(present.ctypes.data, active.ctypes.data, tokens, heads, x, w, request.ctypes.data,
                              prefetch.ctypes.data, ctypes.byref(l1))
    if code != OK:
        raise CometError(code, "comet_kv_plan")
    return request, prefetch, l1.value


def add_bias(Z, bias, stream: Optional[torch.cuda.Stream] = None):
    """Z[i][r, :] += bias[i] in place for both parties (comet_add_bias)."""
    code = _native.add_bias(stream, Z, bias)
    if code:
        raise CometError(code, "comet_add_bias")


def linear_workspace(tokens: int, inner: int, cols: int) -> int:
    """Bytes that `linear` takes for the length of a call on the current device (comet_linear_workspace)."""
    out = ctypes.c_int64(0)
    held = all(0 <= n < 1 << 31 for n in (tokens, inner, cols))          # ctypes would cut a larger one to 32 bits
    code = _lib.comet_linear_workspace(tokens, inner, cols, ctypes.byref(out)) if held else ERR_SHAPE
    if code != OK:
        raise CometError(code, "comet_linear_workspace")
    return out.value


def linear(X, A, W, B, C, frac_bits: int, bias=None, act=None, residual=None, stream: Optional[torch.cuda.Stream] = None):
    """Shared linear layer (comet_linear), both parties: Y = act(trunc(X W^T + bias)) + residual.

    Every tensor argument is a pair (party 0, party 1) of contiguous CUDA tensors of 64-bit integers: X, A [T, K]; W, B [N, K];
    C [T, N] with the dealer's C = A B^T; bias [N]; residual [T, N].  K is a multiple of 8, N of 4.  `act`: None, or
    ((k0, k1, k2), R, Q) for k2 y^2 + k1 y + k0 with coefficients at scale f and the dealer's Q = R * R, [T, N].
    Returns (E, F, M, Y): the messages (M is None without an activation) and the result's shares, new tensors.  A share of the
    result has memory of its own; a party's messages may lie together in one piece, none of the other party's words in it.  The
    operand planes of more than a few rows live in a tensor of linear_workspace(T, K, N) bytes for the length of the call.
    A captured call is replayed on the memory that it was captured with.
    """
    code, E, F, M, Y = _native.linear(stream, X, A, W, B, C, frac_bits, bias, act, residual)
    if code:
        raise CometError(code, "comet_linear")
    return E, F, M, Y


class Norm(NamedTuple):
    """Dealer's material and public numbers of a norm (comet_norm_rotate): pairs U [T, H, D] (masks of x), words
    [T, H, 6 steps - 3] (a row's own), UV [T, H, D]; Newton's steps, its first guess and eps, both at scale f."""
    U: Any
    words: Any
    UV: Any
    steps: int
    guess: int
    eps: int = 0


class Gain(NamedTuple):
    """Shared gain and its triple: pairs weight, mask [gains, D], A, C [T, H, D] with C = A * mask."""
    weight: Any
    mask: Any
    A: Any
    C: Any


class Rotation(NamedTuple):
    """Public angles at scale f, 64-bit integers [rows, rotated / 2], and every token's row of them, int32 [T]."""
    cos: torch.Tensor
    sin: torch.Tensor
    positions: torch.Tensor
    interleaved: bool = False


class NormMessages(NamedTuple):
    """What a party sends: M = x - U, S (a row's openings), D and G (the gain's); pairs, or None where the part is absent."""
    M: Any
    S: Any
    D: Any
    G: Any


def norm_rotate(X, frac_bits: int, norm: Optional[Norm] = None, gain: Optional[Gain] = None,
                rotation: Optional[Rotation] = None, q_heads: Optional[int] = None,
                stream: Optional[torch.cuda.Stream] = None, bad_index_flag=None):
    """Root-mean-square norm of every head, gain and rotation by position (comet_norm_rotate), both parties, in one pass.

    X: a pair of CUDA tensors of 64-bit integers [T, H, D], D even and at most 8192; a token's heads lie together, tokens may
    lie further apart (a view of a stacked projection's result).  Heads below `q_heads` take the gain's first row, the others
    its second; without `q_heads` there is one row.  A rotation may come alone.
    Returns (NormMessages, Z): Z a pair of new tensors [T, H, D], each in memory of its own; a party's messages may lie together in
    one piece, none of the other party's words in it.
    """
    code, M, S, D, G, Z = _native.norm_rotate(stream, X, frac_bits, norm, gain, rotation, q_heads, bad_index_flag)
    if code:
        raise CometError(code, "comet_norm_rotate")
    return NormMessages(M, S, D, G), Z


class PromptDealer(NamedTuple):
    """Dealer's material of a prompt (comet_linear_attention), pairs: the masks q [T, Hq, Dk], k [T, Hk, Dk], v [T, Hk, Dv], d (of the decayed
    keys) [T, Hk, Dk], p (of the weights) [T, Hq, C], s (of the states) [chunks, Hk, Dk, Dv], and the products of masks qk [T, Hq, C], pv, qs
    [T, Hq, Dv], dv [chunks, Hk, Dk, Dv]."""
    q: Any
    k: Any
    v: Any
    d: Any
    p: Any
    s: Any
    qk: Any
    pv: Any
    qs: Any
    dv: Any


class PromptMessages(NamedTuple):
    """What a party sends: its shares of q, k, v, of the decayed keys d, the weights p and the states s, minus their masks; pairs."""
    q: Any
    k: Any
    v: Any
    d: Any
    p: Any
    s: Any


def linear_attention(Q, K, V, starts, decay, dealer: PromptDealer, frac_bits: int, state=None, stream: Optional[torch.cuda.Stream] = None,
                     bad_starts_flag=None):
    """Linear attention with a decay for every head over packed prompts (comet_linear_attention), both parties.

    Q [T, Hq, Dk], K [T, Hk, Dk], V [T, Hk, Dv]: pairs of CUDA tensors of 64-bit integers, a token's heads together, tokens may lie further
    apart (views of a stacked projection's result); Hk divides Hq; Dk and Dv are even, at most 256.  starts: int32 [sequences + 1] on the
    GPU, sequence j the tokens from starts[j] to before starts[j + 1].  decay: public powers [Hk, C + 1] at scale f, of exponents 0 to C; C, at most 64,
    is the length of a chunk.  state: None (zero) or a pair [sequences, Hk, Dk, Dv].
    Returns (PromptMessages, O, state behind the last tokens): new tensors, each share of a result in memory of its own; a party's messages
    may lie together in one piece, none of the other party's words in it.  Rows of tokens in no sequence, and messages of states that no chunk finds, are zero.
    """
    code, *m, O, S = _native.linear_attention(stream, Q, K, V, starts, decay, dealer, frac_bits, state, bad_starts_flag)
    if code:
        raise CometError(code, "comet_linear_attention")
    return PromptMessages(*m), O, S


class StepDealer(NamedTuple):
    """Dealer's material of a token for every sequence (comet_linear_attention_step), pairs: the masks q [B, Hq, Dk], k [B, Hk, Dk],
    v [B, Hk, Dv], s (of the new state) [B, Hk, Dk, Dv], and the products of masks kv [B, Hk, Dk, Dv], qs [B, Hq, Dv]."""
    q: Any
    k: Any
    v: Any
    s: Any
    kv: Any
    qs: Any


class StepMessages(NamedTuple):
    """What a party sends: its shares of q, k, v and the new state s, minus their masks; pairs."""
    q: Any
    k: Any
    v: Any
    s: Any


def linear_attention_step(Q, K, V, decay, state, dealer: StepDealer, frac_bits: int, stream: Optional[torch.cuda.Stream] = None):
    """One token for every sequence of a batch (comet_linear_attention_step), both parties: S <- decay S + k v^T, o = q S.

    Q [B, Hq, Dk], K [B, Hk, Dk], V [B, Hk, Dv] as for linear_attention, a row per sequence; decay: public, [Hk] at scale f; state: a pair
    [B, Hk, Dk, Dv], or None for zero.  Returns (StepMessages, O, new state), new tensors as linear_attention's.
    """
    code, *m, O, S = _native.linear_attention_step(stream, Q, K, V, decay, state, dealer, frac_bits)
    if code:
        raise CometError(code, "comet_linear_attention_step")
    return StepMessages(*m), O, S


class GroupNorm(NamedTuple):
    """Dealer's material and public numbers of a norm of channel groups (comet_group_norm): pairs U [S, P, C] (masks), words [S, groups,
    6 steps - 3] (a group's own), UT [S, P, C] (U times the mask of what it meets); Newton's steps, its first guess and eps, both at scale f."""
    U: Any
    words: Any
    UT: Any
    steps: int
    guess: int
    eps: int = 0


class GroupGain(NamedTuple):
    """Shared gain and bias of every channel with the gain's material: pairs weight, mask, bias [C]; T (masks of gain times root), VW (mask of the
    root times mask of the gain) [S, C]."""
    weight: Any
    mask: Any
    T: Any
    VW: Any
    bias: Any


class GroupNormMessages(NamedTuple):
    """What a party sends: M (the words without their mean), S (a group's openings), D and G (the gain's), N (the activation's); pairs, or None
    where the part is absent."""
    M: Any
    S: Any
    D: Any
    G: Any
    N: Any


def group_norm(X, groups: int, frac_bits: int, norm: GroupNorm, gain: Optional[GroupGain] = None, act=None,
               stream: Optional[torch.cuda.Stream] = None):
    """Norm of groups of neighbouring channels over all positions of a sample, gain, bias and quadratic activation (comet_group_norm).

    X: a pair of CUDA tensors of 64-bit integers [samples, positions, channels], positions may lie further apart; positions = 1 norms
    groups of a token's channels, heads for instance.  act: None, or ((k0, k1, k2), R, Q) for k2 z^2 + k1 z + k0 with coefficients at scale f
    and the dealer's Q = R * R.  Returns (GroupNormMessages, Z): new tensors as norm_rotate's.
    """
    code, *m, Z = _native.group_norm(stream, X, groups, frac_bits, norm, gain, act)
    if code:
        raise CometError(code, "comet_group_norm")
    return GroupNormMessages(*m), Z
