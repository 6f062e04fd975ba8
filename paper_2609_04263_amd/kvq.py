"""Thin ctypes binding of libkvq.so (the C ABI in include/kvq.h).

Argument marshalling only: torch tensors provide device memory and the HIP
stream; every step of the path runs in the library's HIP kernels.  Importing
this module loads ``libkvq.so`` and raises if it is missing or cannot load
(there is no CPU fallback).  Names follow the C ABI without the ``kvq_``
prefix.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from array import array

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvq.so")

FORMAT_FIELDS = ("k_bits", "v_bits", "k_mode", "v_mode", "k_axis", "v_axis",
                 "k_group", "v_group", "residual", "flush", "rotate", "meta_fp16", "sink")

OK, ERR_ARG, ERR_FORMAT, ERR_CAPACITY, ERR_WORKSPACE, ERR_DEVICE, ERR_SCRATCH = range(7)
SCRATCH_BYTES = 4 << 20  # KVQ_SCRATCH_BYTES


class KvqError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {_lib.kvq_strerror(status).decode()} (status {status})")
        self.status = status


class _Rope(C.Structure):  # kvq_rope
    _fields_ = [("rot", C.c_int32), ("layout", C.c_int32), ("scale", C.c_float), ("eps", C.c_float),
                ("turns", C.c_double * 128)]


class Format(C.Structure):
    _fields_ = [(name, C.c_int32) for name in FORMAT_FIELDS]

    @classmethod
    def of(cls, fmt) -> "Format":
        if isinstance(fmt, Format):
            return fmt
        return cls(*[int(fmt.get(name, 0)) for name in FORMAT_FIELDS])


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                          "(the HIP library is required, there is no fallback)")
    L = C.CDLL(LIB_PATH)
    P, I, S = C.c_void_p, C.c_int, C.c_size_t
    Fp = C.POINTER(Format)
    L.kvq_strerror.argtypes = [I]
    L.kvq_strerror.restype = C.c_char_p
    L.kvq_cache_bytes.argtypes = [Fp, I, I, I, I, C.POINTER(S)]
    L.kvq_cache_init.argtypes = [Fp, I, I, I, I, P, S, C.POINTER(P)]
    L.kvq_cache_section.argtypes = [P, I, C.POINTER(S), C.POINTER(S)]
    L.kvq_cache_reset.argtypes = [P]
    L.kvq_cache_len.argtypes = [P, C.POINTER(I), C.POINTER(I)]
    L.kvq_cache_rewind.argtypes = [P, I]
    L.kvq_cache_restore.argtypes = [P, I]
    L.kvq_cache_destroy.argtypes = [P]
    L.kvq_cache_destroy.restype = None
    L.kvq_project_workspace_bytes.argtypes = [I, I, C.POINTER(S)]
    L.kvq_project_qkv.argtypes = [P, I, I, P, I, I, P, P, I, C.c_float, P, P, P, P, S, P]
    L.kvq_merge_adapter.argtypes = [P, I, I, I, P, P, I, C.c_float, P, P]
    L.kvq_project_append.argtypes = [P, I, I, P, I, I, P, P, I, C.c_float, P, P, I, P, S, P]
    L.kvq_append.argtypes = [P, P, P, I, Fp, P]
    Rp = C.POINTER(_Rope)
    L.kvq_rope_init.argtypes = [Rp, I, I] + [C.c_double, I] + [C.c_double] * 4
    L.kvq_rope_qk.argtypes = [Rp, P, P, I, I, I, I, I, P, P, P, I, P, P, P]
    L.kvq_append_rope.argtypes = [P, Rp, P, P, I, P, I, P, I, P, P, P, I, P, Fp, P]
    L.kvq_cache_gather.argtypes = [P, P, C.POINTER(C.c_int32), I, P]
    L.kvq_decode_workspace_bytes.argtypes = [P, I, C.POINTER(S)]
    L.kvq_decode_attn.argtypes = [P, P, I, C.c_float, P, P, S, P]
    L.kvq_decode_attn_noalloc.argtypes = [P, P, I, C.c_float, P, P]
    L.kvq_prefill_attn.argtypes = [P, P, I, I, C.c_float, P, P, S, P]
    L.kvq_prefill_workspace_bytes.argtypes = [P, C.POINTER(S)]
    Ip = C.POINTER(C.c_int32)
    L.kvq_shared_workspace_bytes.argtypes = [P, P, I, I, C.POINTER(S)]
    L.kvq_decode_attn_shared.argtypes = [P, P, Ip, P, I, C.c_float, P, P, S, P]
    L.kvq_prefill_attn_shared.argtypes = [P, P, Ip, P, I, I, C.c_float, P, P, S, P]
    L.kvq_tree_attn_shared.argtypes = [P, P, Ip, P, I, I, C.c_float, P, P, P, S, P]
    L.kvq_time_launches.argtypes = [P, P]
    for name in ("kvq_cache_bytes", "kvq_cache_init", "kvq_cache_section", "kvq_cache_reset",
                 "kvq_cache_len", "kvq_cache_rewind", "kvq_cache_restore", "kvq_project_workspace_bytes",
                 "kvq_project_qkv", "kvq_project_append", "kvq_merge_adapter", "kvq_append",
                 "kvq_rope_init", "kvq_rope_qk", "kvq_append_rope",
                 "kvq_cache_gather", "kvq_decode_workspace_bytes", "kvq_decode_attn", "kvq_decode_attn_noalloc",
                 "kvq_prefill_attn", "kvq_prefill_workspace_bytes", "kvq_shared_workspace_bytes", "kvq_decode_attn_shared",
                 "kvq_prefill_attn_shared", "kvq_tree_attn_shared", "kvq_time_launches"):
        getattr(L, name).restype = I
    return L


_lib = _load()
EXPORTED = ("kvq_strerror", "kvq_cache_bytes", "kvq_cache_init", "kvq_cache_section",
            "kvq_cache_reset", "kvq_cache_len", "kvq_cache_rewind", "kvq_cache_restore", "kvq_cache_destroy",
            "kvq_project_workspace_bytes", "kvq_project_qkv", "kvq_project_append", "kvq_merge_adapter", "kvq_append",
            "kvq_rope_init", "kvq_rope_qk", "kvq_append_rope", "kvq_cache_gather", "kvq_decode_workspace_bytes", "kvq_decode_attn", "kvq_decode_attn_noalloc",
            "kvq_prefill_attn", "kvq_prefill_workspace_bytes", "kvq_shared_workspace_bytes", "kvq_decode_attn_shared",
            "kvq_prefill_attn_shared", "kvq_tree_attn_shared", "kvq_time_launches")


# Calls whose arguments come as 64-bit numbers, in their order: packing them takes a third of ctypes' conversions (1.0 of
# 1.4 us of 16), which is what checking the tensors costs.
_rope_qk, _append_rope = _lib.kvq_internal_rope_qk, _lib.kvq_internal_append_rope
for _f in (_rope_qk, _append_rope):
    _f.argtypes, _f.restype = [C.c_char_p], C.c_int
_pack_qk, _pack_append = struct.Struct("15q").pack, struct.Struct("16q").pack


def lib() -> C.CDLL:
    return _lib


def _check(status: int, what: str) -> None:
    if status != OK:
        raise KvqError(status, what)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


try:  # raw handle of torch's current stream without building a Stream object, of the current device
    _raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
except AttributeError:  # pragma: no cover - older torch
    _raw_stream = None


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(_current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _ints(values, count: int, what: str):
    """Host int32 array of `count` entries from a list, an array or a CPU tensor: (its owner, pointer)."""
    try:
        if not isinstance(values, (list, tuple)):
            values = np.ascontiguousarray(values)
            if not np.issubdtype(values.dtype, np.integer) or values.ndim != 1:
                raise TypeError
            values = values.tolist()
        a = array("i", values)
    except TypeError:
        raise ValueError(f"{what}: {count} integers expected") from None
    except OverflowError:
        raise KvqError(ERR_ARG, what) from None
    if len(a) != count:
        raise ValueError(f"{what}: {count} integers expected, got {len(a)}")
    return a, C.cast(a.buffer_info()[0], C.POINTER(C.c_int32))


# ------------------------------------------------------------- positions

ROPE_SCALINGS = ("plain", "linear", "base", "bands", "yarn")


def _positions(t, count: int, what: str, beside) -> None:
    """Refuses what is not `count` int32 numbers in one piece on the device of `beside` (the library sees an address
    alone)."""
    if t.dtype != torch.int32 or t.numel() != count or not t.is_contiguous():
        raise ValueError(f"{what}: {count} contiguous int32 numbers expected")
    if t.get_device() != beside.get_device():
        raise ValueError(f"{what}: on another device than the tensors beside it")


_bf16, _Tensor = torch.bfloat16, torch.Tensor


def _rows(x, y, count: int, what: str, device: int | None = None) -> int:
    """The device of x and y, refused if they are not `count` bf16 numbers in one piece each (x by its shape) on one
    device, or not on that given: the library sees addresses alone.  (What is no tensor is taken at its word.)"""
    at = x.get_device()
    if isinstance(x, _Tensor):
        if x.dtype is not _bf16 or not x.is_contiguous() or (
                y is not x and (y.dtype is not _bf16 or y.numel() != count or not y.is_contiguous())):
            raise ValueError(f"{what}: {count} contiguous bf16 numbers each expected")
        if y is not x and y.get_device() != at or device is not None and device != at:
            raise ValueError(f"{what}: on another device than the tensors beside it")
    return at


def _weights(w, D: int, what: str, device: int) -> int:
    """The address of a norm's weights."""
    if isinstance(w, _Tensor):
        if w.dtype is not _bf16 or w.numel() != D or not w.is_contiguous():
            raise ValueError(f"{what}: {D} contiguous bf16 numbers expected")
        if w.get_device() != device:
            raise ValueError(f"{what}: on another device than the tensors beside it")
    return w.data_ptr()


class Rope:
    """Rotary positions of `rot` channels of a head (kvq_rope): frequencies base^(-2 i / rot), scaled for contexts
    `factor` times `original` (low, high: the waves in it between which "bands" and "yarn" go over; 32 is yarn's usual
    high, bands' is 4), or `turns`, turns per position of each of the rot / 2 pairs; and the norms' eps."""

    def __init__(self, rot: int, base: float = 10000.0, interleaved: bool = False, scaling: str = "plain",
                 factor: float = 1.0, original: float = 0.0, low: float = 1.0, high: float = 32.0, scale=None,
                 eps: float = 1e-6, turns=None):
        self.c = _Rope()
        self._ref, self._at = C.byref(self.c), C.addressof(self.c)
        if scaling not in ROPE_SCALINGS:
            raise ValueError(f"scaling: one of {', '.join(ROPE_SCALINGS)} expected")
        _check(_lib.kvq_rope_init(self._ref, rot, int(bool(interleaved)), base, ROPE_SCALINGS.index(scaling),
                                  factor, original, low, high), "rope_init")
        if turns is not None:
            if len(turns) != rot // 2:
                raise ValueError(f"turns: {rot // 2} numbers expected, got {len(turns)}")
            self.c.turns[:rot // 2] = [float(x) for x in turns]
        if scale is not None:
            self.c.scale = scale
        self.c.eps = eps

    def qk(self, Q, K, Qo=None, Ko=None, q_norm=None, k_norm=None, pos=None, pos0: int = 0, stream=None) -> None:
        """Qo, Ko (Q and K themselves where not given) <- bf16 Q [B, n, H_q, D] and K [B, n, H_kv, D] (either may be
        None), normed by bf16 weights [D] where given and rotated to positions pos (device int32 [B, n], or None for
        pos0, pos0 + 1, ..)."""
        q = k = qo = ko = H_q = H = 0
        if Q is not None:
            B, n, H_q, D = Q.shape
            if Qo is None:
                Qo = Q
            device = _rows(Q, Qo, B * n * H_q * D, "Q, Qo")
            q, qo = Q.data_ptr(), Qo.data_ptr()
        if K is not None:
            b, m, H, d = K.shape
            if Q is None:
                B, n, D, device = b, m, d, None
            elif b != B or m != n or d != D:
                raise ValueError("Q and K are of different tokens or head sizes")
            if Ko is None:
                Ko = K
            device = _rows(K, Ko, B * n * H * D, "K, Ko", device)
            k, ko = K.data_ptr(), Ko.data_ptr()
        elif Q is None:
            raise ValueError("neither Q nor K")
        q_norm = 0 if q_norm is None else _weights(q_norm, D, "q_norm", device)
        k_norm = 0 if k_norm is None else _weights(k_norm, D, "k_norm", device)
        if pos is not None:
            _positions(pos, B * n, "pos", K if Q is None else Q)
        st = _rope_qk(_pack_qk(self._at, q, k, B, n, H_q, H, D, q_norm, k_norm, 0 if pos is None else pos.data_ptr(), pos0,
                               qo, ko, _stream(stream)))
        if st:
            _check(st, "rope_qk")


# ------------------------------------------------------------------ cache

def cache_bytes(fmt, B: int, H_kv: int, D: int, T_max: int) -> int:
    out = C.c_size_t()
    _check(_lib.kvq_cache_bytes(C.byref(Format.of(fmt)), B, H_kv, D, T_max, C.byref(out)), "cache_bytes")
    return out.value


class Cache:
    """A packed cache: caller-owned device storage (a zero-filled uint8 torch
    tensor) plus the library's host handle."""

    def __init__(self, fmt, B: int, H_kv: int, D: int, T_max: int, device="cuda", storage=None):
        self.fmt = Format.of(fmt)
        self.B, self.H, self.D, self.T_max = B, H_kv, D, T_max
        nbytes = cache_bytes(self.fmt, B, H_kv, D, T_max)
        if storage is None:
            storage = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        self.storage = storage
        h = C.c_void_p()
        _check(_lib.kvq_cache_init(C.byref(self.fmt), B, H_kv, D, T_max, C.c_void_p(_ptr(storage)),
                                   storage.numel() * storage.element_size(), C.byref(h)), "cache_init")
        self.handle, self._at = h, h.value
        self._fmt_ref, self._fmt_at = C.byref(self.fmt), C.addressof(self.fmt)

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and h.value and _lib is not None:
            _lib.kvq_cache_destroy(h)
            self.handle = None

    def section(self, index: int):
        off, ln = C.c_size_t(), C.c_size_t()
        _check(_lib.kvq_cache_section(self.handle, index, C.byref(off), C.byref(ln)), "cache_section")
        return off.value, ln.value

    def reset(self) -> None:
        _check(_lib.kvq_cache_reset(self.handle), "cache_reset")

    def rewind(self, n: int) -> None:
        _check(_lib.kvq_cache_rewind(self.handle, n), "cache_rewind")

    def restore(self, n: int) -> None:
        """Length n after the storage was restored from a snapshot taken at n."""
        _check(_lib.kvq_cache_restore(self.handle, n), "cache_restore")

    def length(self):
        n, nc = C.c_int(), C.c_int()
        _check(_lib.kvq_cache_len(self.handle, C.byref(n), C.byref(nc)), "cache_len")
        return n.value, nc.value

    @property
    def n(self) -> int:
        return self.length()[0]

    def append(self, K, V, n_new: int | None = None, fmt=None, stream=None) -> None:
        """Append bf16 K, V [B, n_new, H_kv, D] (device tensors)."""
        if n_new is None:
            n_new = K.shape[1] if K.dim() == 4 else 1
        f = self._fmt_ref if fmt is None else C.byref(Format.of(fmt))
        st = _lib.kvq_append(self.handle, K.data_ptr(), V.data_ptr(), n_new, f, _stream(stream))
        if st:
            _check(st, "append")

    def append_rope(self, rope: "Rope", K, V, n_new: int | None = None, rows=None, Q=None, Qo=None, q_norm=None,
                    k_norm=None, pos=None, pos0: int = 0, fmt=None, stream=None) -> None:
        """append of keys that `rope` norms and rotates on the way.  bf16 K, V [B, n_in, H_kv, D]; with rows (device
        int32 [B, n_new]) the tokens appended are those rows, else the first n_new (all by default; K, V [B, H_kv, D]
        or [B, H_kv D]: one token).  Q, Qo [B, n_new, H_q, D]: these tokens' queries, rotated too (not with rows; Qo may be Q and has to
        be given).  pos: device int32 [B, n_new], or None for pos0, pos0 + 1, .. (pos0 = self.n where the cache holds
        all tokens before these)."""
        shape = K.shape
        if len(shape) == 4:
            B, n_in, H, D = shape
            fits = B == self.B and H == self.H and D == self.D
        else:
            B, n_in, H, D = self.B, 1, self.H, self.D
            fits = not isinstance(K, _Tensor) or K.numel() == B * H * D
        if not fits:
            raise ValueError(f"K: rows of {self.B} sequences, {self.H} heads of {self.D} expected")
        device = _rows(K, V, B * n_in * H * D, "K, V")
        if n_new is None:
            n_new = n_in if rows is None else rows.shape[1]
        if rows is not None:
            _positions(rows, B * n_new, "rows", K)
        if pos is not None:
            _positions(pos, B * n_new, "pos", K)
        q = H_q = 0
        if Q is not None:
            shape = Q.shape
            if len(shape) == 4:
                b, m, H_q, d = shape
            else:
                (b, H_q, d), m = shape, 1
            if m != n_new:
                raise ValueError(f"Q: rows of {n_new} tokens expected")
            if b != B or d != D:
                raise ValueError(f"Q: rows of {B} sequences, heads of {D} expected")
            _rows(Q, Q if Qo is None else Qo, B * m * H_q * D, "Q, Qo", device)
            q = Q.data_ptr()
        if fmt is not None:
            fmt = Format.of(fmt)
        st = _append_rope(_pack_append(
            self._at, rope._at, K.data_ptr(), V.data_ptr(), n_in, 0 if rows is None else rows.data_ptr(), n_new, q, H_q,
            0 if q_norm is None else _weights(q_norm, D, "q_norm", device), 0 if k_norm is None else _weights(k_norm, D, "k_norm", device),
            0 if pos is None else pos.data_ptr(), pos0, 0 if Qo is None else Qo.data_ptr(),
            self._fmt_at if fmt is None else C.addressof(fmt), _stream(stream)))
        if st:
            _check(st, "append_rope")

    def gather(self, src: "Cache", rows, n: int | None = None, stream=None) -> None:
        """Sequence b becomes the first n tokens (all by default) of src's
        sequence rows[b]; -1 leaves b's bytes.  src may be this cache.  rows
        is host data: a list, an array or a CPU tensor of B integers."""
        keep, ptr = _ints(rows, self.B, "gather")
        st = _lib.kvq_cache_gather(self.handle, src.handle, ptr, src.n if n is None else n, _stream(stream))
        if st:
            _check(st, "gather")

    def decode_workspace_bytes(self, H_q: int) -> int:
        out = C.c_size_t()
        _check(_lib.kvq_decode_workspace_bytes(self.handle, H_q, C.byref(out)), "decode_workspace_bytes")
        return out.value

    def decode_workspace(self, H_q: int, device="cuda"):
        """A workspace of the required size (reuse it across calls)."""
        return torch.empty(self.decode_workspace_bytes(H_q), dtype=torch.uint8, device=device)

    def decode_attn(self, Q, H_q: int, sm_scale: float, O, workspace, stream=None) -> None:
        """O[B, H_q, D] (fp32) <- attention of bf16 Q[B, H_q, D] over the cache."""
        nbytes = workspace.numel() * workspace.element_size()
        st = _lib.kvq_decode_attn(self.handle, Q.data_ptr(), H_q, sm_scale, O.data_ptr(), workspace.data_ptr(),
                                  nbytes, _stream(stream))
        if st:
            _check(st, "decode_attn")

    def decode_attn_noalloc(self, Q, H_q: int, sm_scale: float, O, stream=None) -> None:
        """As decode_attn, with the split partials in the library's static
        scratch (no workspace, nothing allocated)."""
        st = _lib.kvq_decode_attn_noalloc(self.handle, Q.data_ptr(), H_q, sm_scale, O.data_ptr(), _stream(stream))
        if st:
            _check(st, "decode_attn_noalloc")

    def prefill_workspace_bytes(self) -> int:
        out = C.c_size_t()
        _check(_lib.kvq_prefill_workspace_bytes(self.handle, C.byref(out)), "prefill_workspace_bytes")
        return out.value

    def prefill_workspace(self, device="cuda"):
        """A workspace for prefill_attn at the cache's current length."""
        return torch.empty(self.prefill_workspace_bytes(), dtype=torch.uint8, device=device)

    def prefill_attn(self, Q, C_len: int, H_q: int, sm_scale: float, O, workspace, stream=None) -> None:
        """O[B, C, H_q, D] (fp32) <- causal attention of the newest C_len tokens'
        bf16 queries Q[B, C, H_q, D] over the cache."""
        nbytes = workspace.numel() * workspace.element_size()
        st = _lib.kvq_prefill_attn(self.handle, Q.data_ptr(), C_len, H_q, sm_scale, O.data_ptr(),
                                   workspace.data_ptr(), nbytes, _stream(stream))
        if st:
            _check(st, "prefill_attn")


    # This cache as the suffix of a shared one: `prefix` holds P sequences, and
    # sequences first[g] .. first[g + 1] - 1 of this cache come after prefix g
    # (first: P + 1 host integers, or None for equal groups).

    def shared_workspace_bytes(self, prefix: "Cache", H_q: int, C_len: int = 1) -> int:
        out = C.c_size_t()
        _check(_lib.kvq_shared_workspace_bytes(prefix.handle, self.handle, C_len, H_q, C.byref(out)),
               "shared_workspace_bytes")
        return out.value

    def shared_workspace(self, prefix: "Cache", H_q: int, C_len: int = 1, device="cuda"):
        """A workspace for calls of up to C_len queries per sequence (reuse it across calls)."""
        return torch.empty(self.shared_workspace_bytes(prefix, H_q, C_len), dtype=torch.uint8, device=device)

    def decode_attn_shared(self, prefix: "Cache", Q, H_q: int, sm_scale: float, O, workspace, first=None,
                           stream=None) -> None:
        """O[B, H_q, D] (fp32) <- attention of bf16 Q[B, H_q, D] over each
        sequence's prefix and its own tokens here."""
        keep, ptr = (None, None) if first is None else _ints(first, prefix.B + 1, "first")
        nbytes = workspace.numel() * workspace.element_size()
        st = _lib.kvq_decode_attn_shared(prefix.handle, self.handle, ptr, Q.data_ptr(), H_q, sm_scale, O.data_ptr(),
                                         workspace.data_ptr(), nbytes, _stream(stream))
        if st:
            _check(st, "decode_attn_shared")

    def prefill_attn_shared(self, prefix: "Cache", Q, C_len: int, H_q: int, sm_scale: float, O, workspace, first=None,
                            stream=None) -> None:
        """O[B, C, H_q, D] (fp32) <- attention of the newest C_len tokens' bf16
        queries Q[B, C, H_q, D] over each sequence's prefix and, causally, its
        own tokens here."""
        keep, ptr = (None, None) if first is None else _ints(first, prefix.B + 1, "first")
        nbytes = workspace.numel() * workspace.element_size()
        st = _lib.kvq_prefill_attn_shared(prefix.handle, self.handle, ptr, Q.data_ptr(), C_len, H_q, sm_scale,
                                          O.data_ptr(), workspace.data_ptr(), nbytes, _stream(stream))
        if st:
            _check(st, "prefill_attn_shared")

    def tree_attn_shared(self, prefix: "Cache", Q, C_len: int, H_q: int, sm_scale: float, tree, O, workspace,
                         first=None, stream=None) -> None:
        """O[B, C, H_q, D] (fp32) <- attention of the newest C_len tokens' bf16 queries over each sequence's prefix,
        the tokens here before those, and those of them whose bits are set in tree (device int32
        [B, C, ceil(C / 32)], see tree_words)."""
        keep, ptr = (None, None) if first is None else _ints(first, prefix.B + 1, "first")
        _positions(tree, self.B * C_len * (-(-C_len // 32)), "tree", Q)
        nbytes = workspace.numel() * workspace.element_size()
        st = _lib.kvq_tree_attn_shared(prefix.handle, self.handle, ptr, Q.data_ptr(), C_len, H_q, sm_scale,
                                       tree.data_ptr(), O.data_ptr(), workspace.data_ptr(), nbytes, _stream(stream))
        if st:
            _check(st, "tree_attn_shared")


def tree_words(parents):
    """The bits of drafted trees for tree_attn_shared, int32 [B, C, ceil(C / 32)] on the parents' device: parents
    [B, C] holds the index of every draft's parent among the drafts before it, -1 for one that follows the context
    itself, or anything below for a row that is no draft and sees none."""
    p = torch.as_tensor(parents)
    host = p.cpu().tolist()
    C_len = p.shape[1]
    words = -(-C_len // 32)
    flat = array("I")
    for row in host:
        seen = []
        for i, parent in enumerate(row):
            if parent >= i:
                raise ValueError(f"draft {i} comes before its parent {parent}")
            seen.append(0 if parent < -1 else (seen[parent] if parent >= 0 else 0) | 1 << i)
        for bits in seen:
            flat.extend(bits >> 32 * w & 0xFFFFFFFF for w in range(words))
    out = torch.from_numpy(np.frombuffer(flat, np.int32).copy()) if flat else torch.zeros(0, dtype=torch.int32)
    return out.view(len(host), C_len, words).to(p.device)


# ------------------------------------------------------------- projection

def project_workspace_bytes(M: int, rank: int) -> int:
    out = C.c_size_t()
    _check(_lib.kvq_project_workspace_bytes(M, rank, C.byref(out)), "project_workspace_bytes")
    return out.value


def project_qkv(H, W, A, Bm, rank: int, lora_scale: float, d_q: int, d_kv: int, Q, K, V, workspace,
                stream=None) -> None:
    """Q/K/V (bf16) <- H W^T + lora_scale * (H A_p^T) B_p^T per projection."""
    M, d_in = H.shape[0], H.shape[-1]
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib.kvq_project_qkv(_ptr(H), M, d_in, _ptr(W), d_q, d_kv, _ptr(A), _ptr(Bm), rank, lora_scale,
                              _ptr(Q), _ptr(K), _ptr(V), _ptr(workspace), nbytes, _stream(stream))
    if st:
        _check(st, "project_qkv")


def project_append(H, W, A, Bm, rank: int, lora_scale: float, d_q: int, d_kv: int, Q, cache: "Cache",
                   n_new: int, workspace, stream=None) -> None:
    """Q (bf16) as project_qkv; K and V coded straight into `cache` (n_new
    tokens of each sequence, rows of H sequence-major)."""
    M, d_in = H.shape[0], H.shape[-1]
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib.kvq_project_append(_ptr(H), M, d_in, _ptr(W), d_q, d_kv, _ptr(A), _ptr(Bm), rank, lora_scale,
                                 _ptr(Q), cache.handle, n_new, _ptr(workspace), nbytes, _stream(stream))
    if st:
        _check(st, "project_append")


def merge_adapter(W, A, Bm, rank: int, lora_scale: float, d_q: int, d_kv: int, Wout, stream=None) -> None:
    """Wout (bf16) <- W + lora_scale * B_p A_p per projection (dense merge; Wout may be W)."""
    d_in = W.shape[-1]
    st = _lib.kvq_merge_adapter(_ptr(W), d_in, d_q, d_kv, _ptr(A), _ptr(Bm), rank, lora_scale, _ptr(Wout),
                                _stream(stream))
    if st:
        _check(st, "merge_adapter")


def time_launches(start_event, stop_event) -> None:
    """Measurement hook: while set, the library's kernels record the two
    hipEvent_t handles (ints) from their own dispatches (see
    kvq_time_launches); time_launches(None, None) clears it."""
    st = _lib.kvq_time_launches(start_event, stop_event)
    if st:
        _check(st, "time_launches")
