"""GB300 (sm_103a) hot path of MemAttention's memory system (arXiv 2607.05708).

Thin Python binding of the C ABI in ``include/akashic_mem.h``
(``libakashic_mem.so``, built in-tree by ``_build.build()``).  It only
marshals arguments: every step of retrieval (score, relation propagation,
top-k, page resolve), of the relation update (cosine top-M, CSR insert) and of the
quantised key and value cache (write, read, rotation, attention) and the latent cache (append,
attention) runs in the library's CUDA kernels.  PyTorch is used for device memory and
streams.  There is no CPU fallback: without the built library every call
raises.
"""
from __future__ import annotations

import ctypes
import os

from ._build import LIB as LIB_PATH
from ._build import build

__all__ = ["MemStore", "KVCache", "LatentCache", "AkashicError", "load_library", "build", "EXPORTS", "STATUS", "PHASES",
           "softmax_scores_noalloc", "sort_pairs"]

STATUS = {0: "OK", 1: "EINVAL", 2: "ENOMEM", 3: "ECAPACITY", 4: "ECUDA", 5: "ETIMEOUT",
          6: "EDEVICE", 7: "ERANGE"}
PHASES = ("score", "propagate", "select", "relate", "graph", "relocate", "compact", "bound",
          "last_hop", "csr_insert", "transpose", "hub_plan")

# Every function declared in include/akashic_mem.h.
EXPORTS = (
    "akashic_mem_create", "akashic_mem_destroy", "akashic_mem_append_chunks",
    "akashic_mem_update_relations", "akashic_mem_retrieve", "akashic_mem_export_csr",
    "akashic_mem_size", "akashic_mem_sync", "akashic_mem_set_profiling",
    "akashic_mem_phase_times", "akashic_mem_last_error", "akashic_mem_softmax_scores_noalloc",
    "akashic_mem_set_namespace", "akashic_mem_retrieve_scoped", "akashic_mem_delete",
    "akashic_mem_relocate", "akashic_mem_compact_pages", "akashic_mem_page_stats",
    "akashic_mem_export_pages", "akashic_mem_check_wait_timeout", "akashic_mem_sort_pairs",
    "akashic_mem_kv_cache_bytes", "akashic_mem_kv_write", "akashic_mem_kv_read",
    "akashic_mem_kv_attend_scratch", "akashic_mem_kv_attend", "akashic_mem_kv_append",
    "akashic_mem_latent_cache_bytes", "akashic_mem_latent_append", "akashic_mem_latent_attend_scratch",
    "akashic_mem_latent_expanded_scratch", "akashic_mem_latent_attend", "akashic_mem_latent_attend_expanded",
)


class AkashicError(RuntimeError):
    def __init__(self, status: int, message: str):
        self.status = status
        self.code = STATUS.get(status, str(status))
        super().__init__(f"akashic_mem {self.code}: {message}")


class _Config(ctypes.Structure):
    _fields_ = [("dim", ctypes.c_int32), ("capacity", ctypes.c_int64),
                ("chunks_per_page", ctypes.c_int32), ("device", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("relation_scale", ctypes.c_float)]


class _KVConfig(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block_tokens", ctypes.c_int32), ("n_blocks", ctypes.c_int64),
                ("device", ctypes.c_int32)]


class _KVAttend(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("q_row_stride", ctypes.c_int64),
                ("q_head_stride", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("n_q", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("n_seq", ctypes.c_int32),
                ("q_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("blocks", ctypes.c_void_p), ("max_blocks", ctypes.c_int64),
                ("causal", ctypes.c_int32), ("prefix_len", ctypes.c_void_p),
                ("scale", ctypes.c_float), ("cap", ctypes.c_float), ("slopes", ctypes.c_void_p),
                ("tags", ctypes.c_void_p), ("q_tags", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("lse", ctypes.c_void_p)]


class _Rotation(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p),
                ("table_rows", ctypes.c_int64), ("rotary_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("q", ctypes.c_void_p),
                ("q_row_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("q_heads", ctypes.c_int32), ("q_out", ctypes.c_void_p),
                ("q_out_row_stride", ctypes.c_int64), ("q_out_head_stride", ctypes.c_int64)]


class _LatentConfig(ctypes.Structure):
    _fields_ = [("latent_dim", ctypes.c_int32), ("rope_dim", ctypes.c_int32),
                ("block_tokens", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("n_blocks", ctypes.c_int64), ("device", ctypes.c_int32)]


class _LatentAttend(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("q_row_stride", ctypes.c_int64),
                ("q_head_stride", ctypes.c_int64), ("n_q", ctypes.c_int32),
                ("q_heads", ctypes.c_int32), ("n_seq", ctypes.c_int32),
                ("q_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("blocks", ctypes.c_void_p), ("max_blocks", ctypes.c_int64),
                ("causal", ctypes.c_int32), ("prefix_len", ctypes.c_void_p),
                ("scale", ctypes.c_float), ("tags", ctypes.c_void_p), ("q_tags", ctypes.c_void_p),
                ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("w_k", ctypes.c_void_p),
                ("w_v", ctypes.c_void_p), ("w_k_head_stride", ctypes.c_int64),
                ("w_k_row_stride", ctypes.c_int64), ("w_v_head_stride", ctypes.c_int64),
                ("w_v_row_stride", ctypes.c_int64), ("nope_dim", ctypes.c_int32),
                ("value_dim", ctypes.c_int32)]


_lib = None


def load_library(path: str | None = None):
    """Load libakashic_mem.so (raises if it has not been built)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise ImportError(f"{p} is missing: build the CUDA library first "
                          "(python -c 'import __graft_entry__ as g; g.build()')")
    lib = ctypes.CDLL(p)
    V, I32, I64, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    P64 = ctypes.POINTER(ctypes.c_int64)
    sig = {
        "akashic_mem_create": ([ctypes.POINTER(_Config), ctypes.POINTER(V)], ctypes.c_int),
        "akashic_mem_destroy": ([V], None),
        "akashic_mem_append_chunks": ([V, V, I64, V, V, V, V, P64, V], ctypes.c_int),
        "akashic_mem_update_relations": ([V, I64, I64, I32, I32, V], ctypes.c_int),
        "akashic_mem_retrieve": ([V, V, I32, I32, F, I32, V, V, V, V, V], ctypes.c_int),
        "akashic_mem_retrieve_scoped": ([V, V, I32, I32, F, I32, V, I32, V, V, V, V, V],
                                        ctypes.c_int),
        "akashic_mem_set_namespace": ([V, I64, I64, V, V], ctypes.c_int),
        "akashic_mem_delete": ([V, V, I64, V], ctypes.c_int),
        "akashic_mem_relocate": ([V, V, I32, I32, F, V], ctypes.c_int),
        "akashic_mem_compact_pages": ([V, F, F, P64, V], ctypes.c_int),
        "akashic_mem_page_stats": ([V, P64], ctypes.c_int),
        "akashic_mem_export_pages": ([V, V, V], ctypes.c_int),
        "akashic_mem_export_csr": ([V, P64, P64, V, V, V, V, V], ctypes.c_int),
        "akashic_mem_size": ([V, P64, P64], ctypes.c_int),
        "akashic_mem_sync": ([V, V], ctypes.c_int),
        "akashic_mem_check_wait_timeout": ([V, ctypes.c_uint32, V], ctypes.c_int),
        "akashic_mem_sort_pairs": ([V, V, I64, I32, V], ctypes.c_int),
        "akashic_mem_set_profiling": ([V, I32], ctypes.c_int),
        "akashic_mem_phase_times": ([V, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(I32)],
                                    ctypes.c_int),
        "akashic_mem_last_error": ([], ctypes.c_char_p),
        "akashic_mem_softmax_scores_noalloc": ([V, I64, I32, V, I32, F, V, V, V, V, V],
                                               ctypes.c_int),
        "akashic_mem_kv_cache_bytes": ([ctypes.POINTER(_KVConfig), P64], ctypes.c_int),
        "akashic_mem_kv_write": ([ctypes.POINTER(_KVConfig), V, V, V, I64, I64, V, I64, I64, I32,
                                  I64, V, V, V, V], ctypes.c_int),
        "akashic_mem_kv_read": ([ctypes.POINTER(_KVConfig), V, V, I64, I32, V, V, V, V],
                                ctypes.c_int),
        "akashic_mem_kv_attend_scratch": ([ctypes.POINTER(_KVConfig), ctypes.POINTER(_KVAttend),
                                           P64], ctypes.c_int),
        "akashic_mem_kv_attend": ([ctypes.POINTER(_KVConfig), V, ctypes.POINTER(_KVAttend), V, I64,
                                   V, V], ctypes.c_int),
        "akashic_mem_kv_append": ([ctypes.POINTER(_KVConfig), V, V, V, I64, I64, V, I64, I64, I32,
                                   I64, V, V, ctypes.POINTER(_Rotation), V, V], ctypes.c_int),
        "akashic_mem_latent_cache_bytes": ([ctypes.POINTER(_LatentConfig), P64], ctypes.c_int),
        "akashic_mem_latent_append": ([ctypes.POINTER(_LatentConfig), V, V, V, I64, V, I64, I32, I64, V, V,
                                       ctypes.POINTER(_Rotation), V, V], ctypes.c_int),
    }
    latent = [ctypes.POINTER(_LatentConfig), V, ctypes.POINTER(_LatentAttend), V, I64, V, V]
    for name in ("attend", "attend_expanded"):
        sig[f"akashic_mem_latent_{name}"] = (latent, ctypes.c_int)
    for name in ("attend", "expanded"):
        sig[f"akashic_mem_latent_{name}_scratch"] = ([latent[0], latent[2], P64], ctypes.c_int)
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    if path is None:
        _lib = lib
    return lib


def _check(rc: int):
    if rc != 0:
        msg = load_library().akashic_mem_last_error().decode(errors="replace")
        raise AkashicError(rc, msg)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(torch, stream, device):
    s = stream if stream is not None else torch.cuda.current_stream(device)
    return ctypes.c_void_p(s.cuda_stream)


def softmax_scores_noalloc(emb, q, u, z, temperature=0.0, shift=None, status=None, stream=None):
    """Scores for callers that cannot allocate: fills the caller's u [n, B]
    and z [B] (softmax = u[:, b] / z[b]) through
    akashic_mem_softmax_scores_noalloc, which uses a fixed scratch array and
    allocates nothing.  emb: int16 [n, dim], q: int16 [B, dim] with B in
    {32, 64, 128, 256}, all CUDA tensors on the current device."""
    import torch
    for t, name in ((emb, "emb"), (q, "q"), (u, "u"), (z, "z")):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous CUDA tensor")
    s = stream if stream is not None else torch.cuda.current_stream(emb.device)
    _check(load_library().akashic_mem_softmax_scores_noalloc(
        _ptr(emb), emb.shape[0], emb.shape[1], _ptr(q), q.shape[0], float(temperature), _ptr(u),
        _ptr(z), _ptr(shift), _ptr(status), ctypes.c_void_p(s.cuda_stream)))


def sort_pairs(keys, vals, bits=32, stream=None):
    """Stable in-place sort of (keys, vals), int32 CUDA tensors of equal
    length, by the low `bits` bits of the keys, through akashic_mem_sort_pairs
    (the library's own sort primitive)."""
    import torch
    for t, name in ((keys, "keys"), (vals, "vals")):
        if not t.is_cuda or not t.is_contiguous() or t.dtype != torch.int32:
            raise ValueError(f"{name} must be a contiguous int32 CUDA tensor")
    if keys.numel() != vals.numel():
        raise ValueError("keys and vals differ in length")
    s = stream if stream is not None else torch.cuda.current_stream(keys.device)
    _check(load_library().akashic_mem_sort_pairs(_ptr(keys), _ptr(vals), keys.numel(), int(bits),
                                                 ctypes.c_void_p(s.cuda_stream)))


class MemStore:
    """A chunk store on one GPU; methods mirror the C ABI one to one."""

    def __init__(self, dim: int, capacity: int, chunks_per_page: int = 64, device: int = 0,
                 temperature: float = 0.0, relation_scale: float = 0.0):
        import torch
        self._torch = torch
        self.device = device
        self.dim = dim
        lib = load_library()
        cfg = _Config(dim, capacity, chunks_per_page, device, temperature, relation_scale)
        h = ctypes.c_void_p()
        _check(lib.akashic_mem_create(ctypes.byref(cfg), ctypes.byref(h)))
        self._h = h

    @classmethod
    def from_arrays(cls, emb, page_of=None, row_ptr=None, col=None, aff=None, *, dim=None,
                    capacity=None, chunks_per_page=64, device=0, temperature=0.0,
                    relation_scale=0.0, stream=None):
        """Create a store and append host (numpy) arrays: emb uint16 [n, dim] bf16 bits,
        page_of int32 [n], optional out-edge CSR row_ptr/col/aff of those rows."""
        import numpy as np
        import torch
        dev = torch.device("cuda", device)
        n, d = emb.shape
        st = cls(d if dim is None else dim, capacity or n, chunks_per_page, device, temperature,
                 relation_scale)

        def up(a, dt):
            if a is None:
                return None
            return torch.from_numpy(np.ascontiguousarray(a).view(dt)).to(dev)

        st.append_chunks(up(emb, np.int16), up(page_of, np.int32),
                         up(row_ptr, np.int64), up(col, np.int32), up(aff, np.float32),
                         stream=stream)
        return st

    # -- helpers
    def _dev(self, t, dtype, name, numel=None):
        torch = self._torch
        if t is None:
            return None
        if not t.is_cuda or t.device.index != self.device:
            raise ValueError(f"{name} must be a CUDA tensor on device {self.device}")
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if numel is not None and t.numel() < numel:
            raise ValueError(f"{name} needs {numel} elements")
        return t

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            load_library().akashic_mem_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- ABI
    def append_chunks(self, emb, page_of=None, row_ptr=None, col=None, aff=None, stream=None) -> int:
        """emb: int16 [n, dim] (bf16 bits); page_of int32 [n]; optional CSR of the new rows."""
        torch = self._torch
        self._dev(emb, torch.int16, "emb")
        n = emb.shape[0]
        self._dev(page_of, torch.int32, "page_of", n)
        self._dev(row_ptr, torch.int64, "row_ptr", n + 1)
        self._dev(col, torch.int32, "col")
        self._dev(aff, torch.float32, "aff")
        first = ctypes.c_int64(-1)
        _check(load_library().akashic_mem_append_chunks(
            self._h, _ptr(emb), n, _ptr(page_of), _ptr(row_ptr), _ptr(col), _ptr(aff),
            ctypes.byref(first), _stream(torch, stream, self.device)))
        return first.value

    def update_relations(self, first: int, n: int, M: int, reciprocal: bool = True, stream=None):
        _check(load_library().akashic_mem_update_relations(
            self._h, first, n, M, int(bool(reciprocal)), _stream(self._torch, stream, self.device)))

    def relocate(self, S, tau_assoc: float = 0.7, stream=None):
        """Relocation of co-retrieved chunks (S: int64 [n_req, s_len] device tensor)."""
        torch = self._torch
        self._dev(S, torch.int64, "S")
        n_req, s_len = (S.shape[0], S.shape[1]) if S.dim() == 2 else (1, S.shape[0])
        _check(load_library().akashic_mem_relocate(self._h, _ptr(S), n_req, s_len,
                                                   float(tau_assoc),
                                                   _stream(torch, stream, self.device)))

    def compact_pages(self, theta: float = 0.75, tau_assoc: float = 0.7, stream=None) -> int:
        rel = ctypes.c_int64()
        _check(load_library().akashic_mem_compact_pages(
            self._h, float(theta), float(tau_assoc), ctypes.byref(rel),
            _stream(self._torch, stream, self.device)))
        return rel.value

    def page_stats(self) -> dict:
        out = (ctypes.c_int64 * 5)()
        _check(load_library().akashic_mem_page_stats(self._h, out))
        keys = ("pages_in_use", "slots_total", "slots_live", "chunk_writes", "appended")
        return dict(zip(keys, list(out)))

    def export_pages(self, stream=None):
        torch = self._torch
        n, _ = self.size()
        out = torch.empty(max(n, 1), dtype=torch.int32, device=torch.device("cuda", self.device))
        _check(load_library().akashic_mem_export_pages(self._h, _ptr(out),
                                                       _stream(torch, stream, self.device)))
        return out[:n]

    def delete(self, ids, stream=None):
        """Delete chunks (int64 device tensor of chunk IDs)."""
        torch = self._torch
        self._dev(ids, torch.int64, "ids")
        _check(load_library().akashic_mem_delete(self._h, _ptr(ids), ids.numel(),
                                                 _stream(torch, stream, self.device)))

    def set_namespace(self, first: int, ns, stream=None):
        """Tags of chunk IDs [first, first+len(ns)) (int32 device tensor)."""
        torch = self._torch
        self._dev(ns, torch.int32, "ns")
        _check(load_library().akashic_mem_set_namespace(
            self._h, first, ns.numel(), _ptr(ns), _stream(torch, stream, self.device)))

    def retrieve(self, q, k: int, alpha: float, hops: int, ids=None, scores=None, page_ids=None,
                 n_pages=None, stream=None, q_ns=None, sort_by_time: bool = False):
        """q: int16 [B, dim] bf16 bits.  Returns (ids int64 [B,k], scores f32 [B,k],
        page_ids int32 [B,k], n_pages int32 [B]); outputs are allocated unless given.
        q_ns (int32 [B] device tensor) scopes each query to its namespace;
        sort_by_time returns the winners in ascending chunk ID."""
        torch = self._torch
        self._dev(q, torch.int16, "q")
        B = q.shape[0]
        dev = q.device
        if ids is None:
            ids = torch.empty((B, k), dtype=torch.int64, device=dev)
        if scores is None:
            scores = torch.empty((B, k), dtype=torch.float32, device=dev)
        if page_ids is None:
            page_ids = torch.empty((B, k), dtype=torch.int32, device=dev)
        if n_pages is None:
            n_pages = torch.empty((B,), dtype=torch.int32, device=dev)
        self._dev(ids, torch.int64, "ids", B * k)
        self._dev(scores, torch.float32, "scores", B * k)
        self._dev(page_ids, torch.int32, "page_ids", B * k)
        self._dev(n_pages, torch.int32, "n_pages", B)
        if q_ns is None and not sort_by_time:
            _check(load_library().akashic_mem_retrieve(
                self._h, _ptr(q), B, k, float(alpha), hops, _ptr(ids), _ptr(scores),
                _ptr(page_ids), _ptr(n_pages), _stream(torch, stream, self.device)))
        else:
            if q_ns is not None:
                self._dev(q_ns, torch.int32, "q_ns", B)
            _check(load_library().akashic_mem_retrieve_scoped(
                self._h, _ptr(q), B, k, float(alpha), hops,
                None if q_ns is None else _ptr(q_ns), int(bool(sort_by_time)), _ptr(ids),
                _ptr(scores), _ptr(page_ids), _ptr(n_pages), _stream(torch, stream, self.device)))
        return ids, scores, page_ids, n_pages

    def size(self):
        n, e = ctypes.c_int64(), ctypes.c_int64()
        _check(load_library().akashic_mem_size(self._h, ctypes.byref(n), ctypes.byref(e)))
        return n.value, e.value

    def export_csr(self, stream=None):
        torch = self._torch
        n, e = ctypes.c_int64(), ctypes.c_int64()
        lib = load_library()
        st = _stream(torch, stream, self.device)
        _check(lib.akashic_mem_export_csr(self._h, ctypes.byref(n), ctypes.byref(e), None, None,
                                          None, None, st))
        dev = torch.device("cuda", self.device)
        rp = torch.empty(n.value + 1, dtype=torch.int64, device=dev)
        col = torch.empty(max(e.value, 1), dtype=torch.int32, device=dev)
        aff = torch.empty(max(e.value, 1), dtype=torch.float32, device=dev)
        w = torch.empty(max(e.value, 1), dtype=torch.float32, device=dev)
        _check(lib.akashic_mem_export_csr(self._h, ctypes.byref(n), ctypes.byref(e), _ptr(rp),
                                          _ptr(col), _ptr(aff), _ptr(w), st))
        return rp, col[:e.value], aff[:e.value], w[:e.value]

    def sync(self, stream=None):
        _check(load_library().akashic_mem_sync(self._h, _stream(self._torch, stream, self.device)))

    def check_wait_timeout(self, polls: int, stream=None):
        """Queue the bounded-wait self-check: the next sync() raises ETIMEOUT."""
        _check(load_library().akashic_mem_check_wait_timeout(
            self._h, int(polls), _stream(self._torch, stream, self.device)))

    def set_profiling(self, on: bool):
        _check(load_library().akashic_mem_set_profiling(self._h, int(bool(on))))

    def phase_times(self):
        ms = (ctypes.c_float * len(PHASES))()
        ln = (ctypes.c_int32 * len(PHASES))()
        _check(load_library().akashic_mem_phase_times(self._h, ms, ln))
        return {p: (ms[i], ln[i]) for i, p in enumerate(PHASES)}


class _BlockCache:
    """What the caches share: device, streams, checks of tensors, the status word."""

    def _open(self, n_blocks, block_tokens, device, tagged):
        import torch
        self._torch = torch
        self._lib = load_library()
        self.n_blocks, self.block_tokens, self.device = n_blocks, block_tokens, device
        self._dtypes = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
        self._scratch = {}
        self._tagged = tagged

    def _fill(self, data):
        """The cache's memory, and what every call needs, looked up once."""
        torch = self._torch
        self.data, self._dev = data, data.device
        self.tags = (torch.full((self.n_blocks * self.block_tokens,), -1, dtype=torch.int32, device=self._dev)
                     if self._tagged else None)
        self.status = torch.zeros(1, dtype=torch.int32, device=self._dev)
        # the first call may be on another stream than the one that filled these
        torch.cuda.current_stream(self._dev).synchronize()
        # the current stream's handle without a Stream object (4 us a call)
        self._current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
        self._data_ptr, self._status_ptr = self.data.data_ptr(), self.status.data_ptr()
        self._tags_ptr = None if self.tags is None else self.tags.data_ptr()

    def _vec(self, t, dtype, name, numel):
        """The pointer of a contiguous tensor of that type and length (None: NULL)."""
        if t is None:
            return None
        if t.dtype is not dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if t.get_device() != self.device:
            raise ValueError(f"{name} must be a CUDA tensor on device {self.device}")
        if not t.is_contiguous() or t.numel() != numel:
            raise ValueError(f"{name} must be contiguous, of {numel} elements")
        return t.data_ptr()

    def _rows(self, t, name, width, heads=None):
        """dtype code, shape and strides of rows [n, heads, width] whose last
        dimension is contiguous."""
        code = self._dtypes.get(t.dtype)
        if code is None:
            raise TypeError(f"{name} must be bfloat16, float16 or float32, got {t.dtype}")
        if t.get_device() != self.device:
            raise ValueError(f"{name} must be a CUDA tensor on device {self.device}")
        shape, strides = t.shape, t.stride()
        if len(shape) != 3 or shape[2] != width or (heads and shape[1] != heads):
            raise ValueError(f"{name} must be [n, {heads or 'heads'}, {width}]")
        if strides[2] != 1 and t.numel():
            raise ValueError(f"{name} must be contiguous in its last dimension")
        return code, shape, strides

    def _empty(self, shape, dtype, stream, zero=False):
        """A new tensor from the pool of the stream that the call runs on."""
        torch = self._torch
        make = torch.zeros if zero else torch.empty
        if stream is None:
            return make(shape, dtype=dtype, device=self._dev)
        with torch.cuda.stream(stream):
            return make(shape, dtype=dtype, device=self._dev)

    def _on(self, stream):
        return self._current(self.device) if stream is None else stream.cuda_stream

    def _rows2(self, t, name, width):
        """_rows of one head's rows [n, width]: dtype code, length, stride."""
        code = self._dtypes.get(t.dtype)
        if code is None:
            raise TypeError(f"{name} must be bfloat16, float16 or float32, got {t.dtype}")
        if t.get_device() != self.device:
            raise ValueError(f"{name} must be a CUDA tensor on device {self.device}")
        shape, strides = t.shape, t.stride()
        if len(shape) != 2 or shape[1] != width:
            raise ValueError(f"{name} must be [n, {width}]")
        if strides[1] != 1 and t.numel():
            raise ValueError(f"{name} must be contiguous in its last dimension")
        return code, shape[0], strides[0]

    def _rotation(self, n, width, dt, positions, cos, sin, q, q_out, interleaved, stream):
        """The rotation of n tokens as the ABI takes it, and q_out."""
        vec, f32 = self._vec, self._torch.float32
        if positions is None or cos is None or sin is None:
            raise ValueError("a rotation needs positions, cos and sin")
        if cos.dim() != 2 or sin.shape != cos.shape:
            raise ValueError("cos and sin must be [positions, rotary_dim / 2]")
        rows, half = cos.shape
        at = vec(positions, self._torch.int64, "positions", n)
        pc, ps = vec(cos, f32, "cos", rows * half), vec(sin, f32, "sin", rows * half)
        if q is None:
            if q_out is not None:
                raise ValueError("q_out needs q")
            return ctypes.byref(_Rotation(at, pc, ps, rows, 2 * half, 1 if interleaved else 0)), None
        code, shape, st = self._rows(q, "q", width)
        if code != dt or shape[0] != n:
            raise ValueError(f"q must be of the rows' type, {n} tokens")
        if q_out is None:
            q_out = self._empty(shape, q.dtype, stream)
            so = q_out.stride()
        else:
            code, other, so = self._rows(q_out, "q_out", width)
            if code != dt or other != shape:
                raise ValueError("q_out must be of q's type and shape")
        return ctypes.byref(_Rotation(at, pc, ps, rows, 2 * half, 1 if interleaved else 0, q.data_ptr(), st[0], st[1],
                                      shape[1], q_out.data_ptr(), so[0], so[1])), q_out

    def sync(self, stream=None):
        """Wait for the stream, then raise (and clear) what the kernels recorded: a slot,
        block ID, length or row range out of bounds (EDEVICE), an expired wait."""
        s = stream if stream is not None else self._torch.cuda.current_stream(self.device)
        s.synchronize()
        code = int(self.status.item())
        if code:
            self.status.zero_()
            self._torch.cuda.current_stream(self.device).synchronize()   # before any other stream's calls
            raise AkashicError(code, f"{self._name}: an index or length was out of bounds" if code == 6
                               else f"{self._name}: a kernel of the cache failed")


class KVCache(_BlockCache):
    """Keys and values of `heads` heads in 4 or 8 bits, in blocks of
    `block_tokens` tokens (akashic_mem_kv_*; the format is in the header).

    A block per stored chunk, block ID = chunk ID, makes what
    MemStore.retrieve returns the list of blocks to attend over.  With
    `tagged`, every slot has an int32 tag (-1 while it holds no token): a
    namespace or a document, which attention can be restricted to.  A slot keeps
    its token and tag until it is written again: set `tags` to -1 where a
    block is given to fewer tokens than it held.  No
    gradient is recorded through any of the calls.  The memory is `data`
    (uint8), `tags` (int32 [n_blocks * block_tokens] or None) and `status`
    (int32 [1], read and cleared by sync())."""

    _name = "kv"

    def __init__(self, n_blocks: int, heads: int, head_dim: int, block_tokens: int = 64,
                 bits: int = 4, device: int = 0, tagged: bool = False):
        self._open(n_blocks, block_tokens, device, tagged)
        torch = self._torch
        self.heads, self.head_dim, self.bits = heads, head_dim, bits
        self._cfg = ctypes.byref(_KVConfig(bits, heads, head_dim, block_tokens, n_blocks, device))
        size = ctypes.c_int64()
        _check(self._lib.akashic_mem_kv_cache_bytes(self._cfg, ctypes.byref(size)))
        self._fill(torch.empty(size.value, dtype=torch.uint8, device=torch.device("cuda", device)))
        self._write, self._read = self._lib.akashic_mem_kv_write, self._lib.akashic_mem_kv_read
        self._append, self._attend = self._lib.akashic_mem_kv_append, self._lib.akashic_mem_kv_attend

    def _kv(self, k, v, tags):
        """Checks of keys and values: dtype code, tokens, strides."""
        dt, shape, sk = self._rows(k, "k", self.head_dim, self.heads)
        dtv, shape_v, sv = self._rows(v, "v", self.head_dim, self.heads)
        if dtv != dt or shape_v != shape:
            raise ValueError("k and v must be of one type and shape")
        if tags is not None and self.tags is None:
            raise ValueError("tags need a tagged cache")
        return dt, shape[0], sk, sv

    # -- ABI
    def write(self, k, v, slots, tags=None, stream=None):
        """Quantise k, v [n, heads, head_dim] (bfloat16, float16 or float32; any strides
        of the first two dimensions) into slots (int64 [n]; block * block_tokens +
        place; -1 skips a row; a slot at most once).  tags (int32 [n], tagged caches
        only): the tags of the rows, 0 if not given."""
        torch = self._torch
        dt, n, sk, sv = self._kv(k, v, tags)
        rc = self._write(self._cfg, self._data_ptr, self._tags_ptr, k.data_ptr(), sk[0], sk[1],
                         v.data_ptr(), sv[0], sv[1], dt, n,
                         self._vec(slots, torch.int64, "slots", n),
                         self._vec(tags, torch.int32, "tags", n), self._status_ptr,
                         self._on(stream))
        if rc:
            _check(rc)

    def append(self, k, v, slots, positions, cos, sin, q=None, q_out=None, interleaved=False, tags=None,
               stream=None):
        """write() with the keys rotated to their positions (int64 [n]) on the way: of a head's
        first 2 * cos.shape[1] values (a multiple of 32) pair i, (x[i], x[i + half]) or, interleaved,
        (x[2i], x[2i + 1]), is turned by the angle whose cosine and sine the tables
        (float32 [positions, pairs]) hold.  q [n, q_heads, head_dim] of k's type: rotated too
        and returned, in q_out (q itself, or another tensor that does not overlap it; its
        rows apart from each other) if given; zero for tokens that are skipped."""
        dt, n, sk, sv = self._kv(k, v, tags)
        r, q_out = self._rotation(n, self.head_dim, dt, positions, cos, sin, q, q_out, interleaved, stream)
        rc = self._append(self._cfg, self._data_ptr, self._tags_ptr, k.data_ptr(), sk[0], sk[1], v.data_ptr(),
                          sv[0], sv[1], dt, n, self._vec(slots, self._torch.int64, "slots", n),
                          self._vec(tags, self._torch.int32, "tags", n), r, self._status_ptr,
                          self._on(stream))
        if rc:
            _check(rc)
        return q_out

    def read(self, slots, dtype=None, k=None, v=None, stream=None):
        """The values that slots (int64 [n], -1: zeros) stand for: k, v [n, heads,
        head_dim] of dtype (bfloat16 if not given), allocated unless given."""
        torch = self._torch
        dtype = dtype or (k.dtype if k is not None else torch.bfloat16)
        code = self._dtypes.get(dtype)
        if code is None:
            raise TypeError(f"dtype must be bfloat16, float16 or float32, got {dtype}")
        n = slots.numel()
        shape = (n, self.heads, self.head_dim)
        ps = self._vec(slots, torch.int64, "slots", n)
        numel = n * self.heads * self.head_dim
        if k is None:
            k = self._empty(shape, dtype, stream)
            pk = k.data_ptr()
        else:
            pk = self._vec(k, dtype, "k", numel)
        if v is None:
            v = self._empty(shape, dtype, stream)
            pv = v.data_ptr()
        else:
            pv = self._vec(v, dtype, "v", numel)
        rc = self._read(self._cfg, self._data_ptr, ps, n, code, pk, pv, self._status_ptr,
                        self._on(stream))
        if rc:
            _check(rc)
        return k, v

    def attend(self, q, blocks, kv_len=None, q_start=None, causal=True, prefix_len=None,
               scale=0.0, cap=0.0, slopes=None, q_tags=None, out=None, lse=None, stream=None):
        """Attention of q [n_q, q_heads, head_dim] (bfloat16 or float16) over the listed
        blocks (int64 [n_seq, max_blocks], -1: none).  Sequence s has the query rows
        q_start[s] to q_start[s + 1] (int32 [n_seq + 1]; not given: n_q / n_seq rows
        each) and the first kv_len[s] tokens (int32 [n_seq]; not given: all) of its
        blocks; its last query row stands at its last token.  causal, prefix_len
        (int32 [n_seq]: keys that all rows see), scale (0: 1 / sqrt(head_dim)), cap,
        slopes (float32 [q_heads]) and q_tags (int32 [n_q], tagged caches only) as in
        akashic_mem_kv_attend.  Returns (out [n_q, q_heads, head_dim] of q's type,
        lse float32 [n_q, q_heads]); rows behind the last sequence are left as they
        were (zero in tensors allocated here)."""
        torch = self._torch
        dt, (n_q, q_heads, _), sq = self._rows(q, "q", self.head_dim)
        if dt == 2:
            raise TypeError("q must be bfloat16 or float16, got torch.float32")
        if blocks.dim() != 2:
            raise ValueError("blocks must be [n_seq, max_blocks]")
        if q_tags is not None and self.tags is None:
            raise ValueError("q_tags need a tagged cache")
        n_seq, width = blocks.shape
        vec, i32, f32 = self._vec, torch.int32, torch.float32
        a = _KVAttend(
            q.data_ptr(), sq[0], sq[1], dt, n_q, q_heads, n_seq,
            vec(q_start, i32, "q_start", n_seq + 1), vec(kv_len, i32, "kv_len", n_seq),
            vec(blocks, torch.int64, "blocks", n_seq * width), width, 1 if causal else 0,
            vec(prefix_len, i32, "prefix_len", n_seq), scale, cap,
            vec(slopes, f32, "slopes", q_heads), None if q_tags is None else self._tags_ptr,
            vec(q_tags, i32, "q_tags", n_q))
        ref = ctypes.byref(a)
        behind = q_start is not None or n_seq == 0         # rows that no sequence has
        if out is None:
            out = self._empty(q.shape, q.dtype, stream, zero=behind)
            a.out = out.data_ptr()
        else:
            a.out = vec(out, q.dtype, "out", n_q * q_heads * self.head_dim)
        if lse is None:
            lse = self._empty((n_q, q_heads), f32, stream, zero=behind)
            a.lse = lse.data_ptr()
        else:
            a.lse = vec(lse, f32, "lse", n_q * q_heads)
        key = (n_q, q_heads, n_seq, width, q_start is None, q_tags is None)
        size = self._scratch.get(key)
        if size is None:
            need = ctypes.c_int64()
            _check(self._lib.akashic_mem_kv_attend_scratch(self._cfg, ref, ctypes.byref(need)))
            if len(self._scratch) > 4096:
                self._scratch.clear()
            size = self._scratch[key] = need.value
        scratch = self._empty((size,), torch.uint8, stream) if size else None
        rc = self._attend(self._cfg, self._data_ptr, ref, scratch.data_ptr() if size else None, size,
                          self._status_ptr, self._on(stream))
        if rc:
            _check(rc)
        return out, lse


class LatentCache(_BlockCache):
    """One latent vector and one rotated key a token, shared by all heads, in bfloat16 or
    float16, in blocks of `block_tokens` tokens (akashic_mem_latent_*).

    A block per stored chunk, block ID = chunk ID, makes what MemStore.retrieve returns the
    list of blocks to attend over; `tagged` as for KVCache.  No gradient is recorded
    through any of the calls.  The memory is `data` [n_blocks * block_tokens,
    latent_dim + rope_dim] (zero until it is written; it has to stay finite), `tags`
    and `status` as KVCache's."""

    _name = "latent"

    def __init__(self, n_blocks: int, latent_dim: int, rope_dim: int, block_tokens: int = 64,
                 dtype=None, device: int = 0, tagged: bool = False):
        self._open(n_blocks, block_tokens, device, tagged)
        torch = self._torch
        self.latent_dim, self.rope_dim, self.dtype = latent_dim, rope_dim, dtype or torch.bfloat16
        if self.dtype not in (torch.bfloat16, torch.float16):
            raise TypeError(f"dtype must be bfloat16 or float16, got {dtype}")
        self._cfg = ctypes.byref(_LatentConfig(latent_dim, rope_dim, block_tokens, self._dtypes[self.dtype],
                                               n_blocks, device))
        size = ctypes.c_int64()
        _check(self._lib.akashic_mem_latent_cache_bytes(self._cfg, ctypes.byref(size)))
        self._fill(torch.zeros(n_blocks * block_tokens, latent_dim + rope_dim, dtype=self.dtype,
                               device=torch.device("cuda", device)))
        self._append = self._lib.akashic_mem_latent_append
        self._calls = {False: (self._lib.akashic_mem_latent_attend, self._lib.akashic_mem_latent_attend_scratch),
                       True: (self._lib.akashic_mem_latent_attend_expanded,
                              self._lib.akashic_mem_latent_expanded_scratch)}

    def append(self, latent, k_rope, slots, positions=None, cos=None, sin=None, q=None, q_out=None,
               interleaved=False, tags=None, stream=None):
        """Round latent [n, latent_dim] and k_rope [n, rope_dim] (bfloat16, float16 or float32; any
        stride of the first dimension) into slots (as KVCache.write), k_rope rotated
        where positions, cos and sin (float32 [positions, rope_dim / 2]) are given, and with it
        q [n, q_heads, rope_dim] as in KVCache.append.  Returns q_out (None without q)."""
        dt, n, sl = self._rows2(latent, "latent", self.latent_dim)
        dtk, nk, sk = self._rows2(k_rope, "k_rope", self.rope_dim)
        if dtk != dt or nk != n:
            raise ValueError("latent and k_rope must be of one type and length")
        if tags is not None and self.tags is None:
            raise ValueError("tags need a tagged cache")
        ref = None
        if positions is not None or cos is not None or sin is not None or q is not None or q_out is not None:
            ref, q_out = self._rotation(n, self.rope_dim, dt, positions, cos, sin, q, q_out, interleaved, stream)
        rc = self._append(self._cfg, self._data_ptr, self._tags_ptr, latent.data_ptr(), sl, k_rope.data_ptr(),
                          sk, dt, n, self._vec(slots, self._torch.int64, "slots", n),
                          self._vec(tags, self._torch.int32, "tags", n), ref, self._status_ptr, self._on(stream))
        if rc:
            _check(rc)
        return q_out

    def _run(self, q, sq, blocks, scale, width, kv_len, q_start, causal, prefix_len, q_tags, out, lse, stream,
             weights=()):
        torch = self._torch
        vec, i32 = self._vec, torch.int32
        n_q, q_heads, _ = q.shape
        if blocks.dim() != 2:
            raise ValueError("blocks must be [n_seq, max_blocks]")
        if q_tags is not None and self.tags is None:
            raise ValueError("q_tags need a tagged cache")
        n_seq, listed = blocks.shape
        behind = q_start is not None or n_seq == 0         # rows that no sequence has
        if out is None:
            out = self._empty((n_q, q_heads, width), self.dtype, stream, zero=behind)
            po = out.data_ptr()
        else:
            po = vec(out, self.dtype, "out", n_q * q_heads * width)
        pl = None
        if not weights:
            if lse is None:
                lse = self._empty((n_q, q_heads), torch.float32, stream, zero=behind)
                pl = lse.data_ptr()
            else:
                pl = vec(lse, torch.float32, "lse", n_q * q_heads)
        ref = ctypes.byref(_LatentAttend(
            q.data_ptr(), sq[0], sq[1], n_q, q_heads, n_seq, vec(q_start, i32, "q_start", n_seq + 1),
            vec(kv_len, i32, "kv_len", n_seq), vec(blocks, torch.int64, "blocks", n_seq * listed), listed,
            1 if causal else 0, vec(prefix_len, i32, "prefix_len", n_seq), scale,
            None if q_tags is None else self._tags_ptr, vec(q_tags, i32, "q_tags", n_q), po, pl, *weights))
        call, scratch_of = self._calls[len(weights) > 0]
        key = (n_q, q_heads, n_seq, listed, q_start is None, q_tags is None, weights[-2:])
        size = self._scratch.get(key)
        if size is None:
            need = ctypes.c_int64()
            _check(scratch_of(self._cfg, ref, ctypes.byref(need)))
            if len(self._scratch) > 4096:
                self._scratch.clear()
            size = self._scratch[key] = need.value
        scratch = self._empty((size,), torch.uint8, stream) if size else None
        rc = call(self._cfg, self._data_ptr, ref, scratch.data_ptr() if size else None, size, self._status_ptr,
                  self._on(stream))
        if rc:
            _check(rc)
        return out, lse

    def attend(self, q, blocks, scale, kv_len=None, q_start=None, causal=True, prefix_len=None, q_tags=None,
               out=None, lse=None, stream=None):
        """Absorbed attention of q [n_q, q_heads, latent_dim + rope_dim] (the cache's type; a head's first
        latent_dim values its query times w_k) over the listed blocks; sequences, masks and
        tags as in KVCache.attend.  scale: of the scores (the width of a head before it was absorbed
        is not known here).  Returns (out [n_q, q_heads, latent_dim], to be multiplied by
        w_v, and lse float32 [n_q, q_heads]).  For single tokens and drafts; prompts
        take fewer products in attend_expanded."""
        _, _, sq = self._rows(q, "q", self.latent_dim + self.rope_dim)
        if q.dtype is not self.dtype:
            raise TypeError(f"q must be {self.dtype}, got {q.dtype}")
        return self._run(q, sq, blocks, scale, self.latent_dim, kv_len, q_start, causal, prefix_len, q_tags, out, lse,
                         stream)

    def attend_expanded(self, q, w_k, w_v, blocks, scale=None, kv_len=None, q_start=None, causal=True,
                        prefix_len=None, q_tags=None, out=None, stream=None):
        """Attention of q [n_q, q_heads, nope_dim + rope_dim] through per-head keys and values:
        w_k [q_heads, nope_dim, latent_dim] and w_v [q_heads, value_dim, latent_dim] (the
        cache's type, a head's rows evenly spaced: halves of one projection's rows do; nope_dim and
        value_dim 64 or 128).  scale: 1 / sqrt(nope_dim + rope_dim) if not given.  Returns out
        [n_q, q_heads, value_dim].  For prompts; other arguments as in attend."""
        for t, name in ((w_k, "w_k"), (w_v, "w_v")):
            if t.dtype is not self.dtype:
                raise TypeError(f"{name} must be {self.dtype}, got {t.dtype}")
            if t.dim() != 3 or t.shape[2] != self.latent_dim or t.stride(2) != 1:
                raise ValueError(f"{name} must be [q_heads, rows, {self.latent_dim}], contiguous in its last dimension")
            if t.get_device() != self.device:
                raise ValueError(f"{name} must be a CUDA tensor on device {self.device}")
        nope, value = w_k.shape[1], w_v.shape[1]
        _, shape, sq = self._rows(q, "q", nope + self.rope_dim)
        if q.dtype is not self.dtype:
            raise TypeError(f"q must be {self.dtype}, got {q.dtype}")
        if w_k.shape[0] != shape[1] or w_v.shape[0] != shape[1]:
            raise ValueError("w_k and w_v must have q's heads")
        scale = (nope + self.rope_dim) ** -0.5 if scale is None else scale
        return self._run(q, sq, blocks, scale, value, kv_len, q_start, causal, prefix_len, q_tags, out, None, stream,
                         (w_k.data_ptr(), w_v.data_ptr(), w_k.stride(0), w_k.stride(1), w_v.stride(0), w_v.stride(1),
                          nope, value))[0]
