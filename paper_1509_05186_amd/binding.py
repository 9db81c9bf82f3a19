"""ctypes binding of include/etf.h.  Method names are the C entry points without the prefix."""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

ETF_MAX_M = 16
ETF_MAX_TOPK = 1024
ETF_MODE_FLAT, ETF_MODE_TREE, ETF_MODE_FOREST = 0, 1, 2

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "lib", "libetf.so")
_lib = None

EXPORTS = [
    "etf_create", "etf_destroy", "etf_set_stream", "etf_strerror", "etf_last_error", "etf_set_option",
    "etf_pq_train", "etf_pq_set_codebooks", "etf_pq_get_codebooks", "etf_pq_encode",
    "etf_pq_set_rotation", "etf_pq_get_rotation", "etf_rotate", "etf_rotate_workspace_bytes", "etf_rotate_device", "etf_opq_train",
    "etf_index_build", "etf_index_set_leaf_term", "etf_index_set_leaf_bytes", "etf_index_set_chunk_order", "etf_suggest_chunk_order", "etf_suggest_partition", "etf_index_stats", "etf_index_device_bytes", "etf_index_upload",
    "etf_index_layout", "etf_index_export",
    "etf_encode_workspace_bytes", "etf_pq_encode_device",
    "etf_index_build_device_bytes", "etf_index_build_device", "etf_last_build_path",
    "etf_workspace_bytes", "etf_lut_build", "etf_adc", "etf_search", "etf_last_fallback_count", "etf_last_matrix_blocks", "etf_last_kept_encodings",
    "etf_static_scratch_bytes", "etf_search_static",
    "etf_profile_enable", "etf_profile_read", "etf_probe_bandwidth",
    "etf_ivf_set_coarse", "etf_ivf_assign_workspace_bytes", "etf_ivf_assign_device", "etf_ivf_build", "etf_ivf_stats",
    "etf_ivf_device_bytes", "etf_ivf_upload", "etf_ivf_workspace_bytes", "etf_ivf_search",
    "etf_kv_append", "etf_kv_attend_workspace_bytes", "etf_kv_attend", "etf_kv_select_workspace_bytes", "etf_kv_select", "etf_kv_evict", "etf_kv_evict_ahead",
    "etf_kv_append_packed", "etf_kv_take_workspace_bytes", "etf_kv_take", "etf_kv_fork_workspace_bytes", "etf_kv_fork", "etf_kv_free",
    "etf_kv_compact_workspace_bytes", "etf_kv_compact",
    "etf_prompt_attend_workspace_bytes", "etf_prompt_attend",
]
ETF_BUILD_NONE, ETF_BUILD_CHAIN, ETF_BUILD_GENERAL, ETF_BUILD_GENERAL_AFTER_CHAIN = 0, 1, 2, 3
ETF_PROBE_READ, ETF_PROBE_WRITE, ETF_PROBE_COPY, ETF_PROBE_ROWS, ETF_PROBE_LDS, ETF_PROBE_LDS_SCATTER = 0, 1, 2, 3, 4, 5
ETF_PROBE_VALU_F32, ETF_PROBE_VALU_ADD3, ETF_PROBE_VALU_PK16, ETF_PROBE_MFMA_F32 = 6, 7, 8, 9
KERNEL_CLASSES = ["lut", "level", "leaf", "flat", "reduce", "tau", "select", "exact", "sample", "lds", "encode",
                  "ivf_coarse", "ivf_scan", "lds16", "kv"]
ETF_KV_BLOCK, ETF_KV_MAX_LIST = 64, 4096
ETF_KV_BF16, ETF_KV_FP16 = 0, 1


class EtfStats(ctypes.Structure):
    _fields_ = [
        ("M", ctypes.c_int32), ("K", ctypes.c_int32), ("T", ctypes.c_int32),
        ("chunk_begin", ctypes.c_int32 * (ETF_MAX_M + 1)),
        ("N", ctypes.c_int64), ("n_distinct", ctypes.c_int64), ("max_dup", ctypes.c_int64),
        ("nI", (ctypes.c_int64 * ETF_MAX_M) * ETF_MAX_M),
        ("nL", (ctypes.c_int64 * ETF_MAX_M) * ETF_MAX_M),
        ("L1", ctypes.c_int64 * ETF_MAX_M), ("L2", ctypes.c_int64 * ETF_MAX_M),
        ("sumP", ctypes.c_int64 * ETF_MAX_M), ("lookups", ctypes.c_int64 * ETF_MAX_M),
        ("paper_bytes", ctypes.c_int64 * ETF_MAX_M),
        ("device_bytes", ctypes.c_int64),
        ("chunk_order", ctypes.c_int32 * ETF_MAX_M),
    ]

    def as_dict(self) -> dict:
        T = self.T
        cb = [int(self.chunk_begin[t]) for t in range(T + 1)]
        trees = []
        for t in range(T):
            D = cb[t + 1] - cb[t]
            trees.append({
                "chunks": (cb[t], cb[t + 1]), "D": D,
                "nI": [int(self.nI[t][l]) for l in range(D)], "nL": [int(self.nL[t][l]) for l in range(D)],
                "L1": int(self.L1[t]), "L2": int(self.L2[t]), "sumP": int(self.sumP[t]),
                "lookups": int(self.lookups[t]), "paper_bytes": int(self.paper_bytes[t]),
            })
        return {"M": self.M, "K": self.K, "T": T, "N": int(self.N), "n_distinct": int(self.n_distinct),
                "max_dup": int(self.max_dup), "device_bytes": int(self.device_bytes), "trees": trees,
                "chunk_order": [int(self.chunk_order[j]) for j in range(self.M)]}


class EtfIvfStats(ctypes.Structure):
    _fields_ = [("cells", ctypes.c_int32), ("N", ctypes.c_int64), ("entries", ctypes.c_int64), ("max_list", ctypes.c_int64),
                ("max_dup", ctypes.c_int64), ("tree_lookups", ctypes.c_int64), ("flat_lookups", ctypes.c_int64),
                ("device_bytes", ctypes.c_int64)]

    def as_dict(self) -> dict:
        return {name: int(getattr(self, name)) for name, _ in self._fields_}


_Grid64 = (ctypes.c_int64 * ETF_MAX_M) * ETF_MAX_M
_Grid32 = (ctypes.c_int32 * ETF_MAX_M) * ETF_MAX_M


class EtfLayout(ctypes.Structure):
    _fields_ = [
        ("total", ctypes.c_int64),
        ("codebooks", ctypes.c_int64), ("codes", ctypes.c_int64), ("ids_in", ctypes.c_int64),
        ("ids_sorted", ctypes.c_int64), ("ebegin", ctypes.c_int64), ("enc_of_pos", ctypes.c_int64),
        ("ecodes", ctypes.c_int64), ("sample_enc", ctypes.c_int64), ("sample_pos", ctypes.c_int64),
        ("n_sample_enc", ctypes.c_int64), ("n_sample_pos", ctypes.c_int64),
        ("leaf_of", ctypes.c_int64 * ETF_MAX_M),
        ("icode", _Grid64), ("iparent", _Grid64), ("lcodes", _Grid64), ("lparent", _Grid64), ("lrow", _Grid64),
        ("lstride", _Grid32),
        ("rec0", ctypes.c_int64), ("rec0_stride", ctypes.c_int32),
        ("trec", ctypes.c_int64 * ETF_MAX_M), ("trec_stride", ctypes.c_int32 * ETF_MAX_M),
        ("cb_centered", ctypes.c_int64), ("cb_norm", ctypes.c_int64), ("cb_mean", ctypes.c_int64),
        ("sample_enc_codes", ctypes.c_int64), ("sample_pos_codes", ctypes.c_int64),
        ("cb_row", ctypes.c_int32),
        ("eterm", ctypes.c_int64), ("pterm", ctypes.c_int64),
    ]


class EtfKvCache(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("pages", ctypes.c_int32)] + [
                    (name, ctypes.c_void_p) for name in ("k", "v", "bounds", "scales", "tail_k", "tail_v", "table", "lens", "evicted")]


class EtfError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__("etf error %d: %s" % (code, message))
        self.code = code


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads lib/libetf.so.  Raises if it has not been built: there is no other implementation."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError("HIP library %s is missing: run `python -m paper_1509_05186_amd.build`" % _LIB_PATH)
    try:
        # torch first: the library must bind to the HIP runtime torch brings along (whichever of the two is
        # loaded first decides), or its calls see no device in a process where torch holds the GPU
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = ctypes.CDLL(_LIB_PATH)
    P, I, L = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    sig = {
        "etf_create": (I, [ctypes.POINTER(P), I, P]),
        "etf_destroy": (None, [P]),
        "etf_set_stream": (I, [P, P]),
        "etf_strerror": (ctypes.c_char_p, [I]),
        "etf_last_error": (ctypes.c_char_p, [P]),
        "etf_set_option": (I, [P, ctypes.c_char_p, L]),
        "etf_pq_train": (I, [P, P, L, I, I, I, I, ctypes.c_uint64]),
        "etf_pq_set_codebooks": (I, [P, P, I, I, I]),
        "etf_pq_get_codebooks": (I, [P, P]),
        "etf_pq_encode": (I, [P, P, L, P]),
        "etf_pq_set_rotation": (I, [P, P, I]),
        "etf_pq_get_rotation": (I, [P, P]),
        "etf_rotate": (I, [P, P, L, P]),
        "etf_rotate_workspace_bytes": (L, [P]),
        "etf_rotate_device": (I, [P, P, L, P, P, L]),
        "etf_opq_train": (I, [P, P, L, I, I, I, I, I, ctypes.c_uint64]),
        "etf_index_build": (I, [P, P, L, P, I, P]),
        "etf_index_set_chunk_order": (I, [P, P]),
        "etf_index_set_leaf_term": (I, [P, P, L]),
        "etf_index_set_leaf_bytes": (I, [P, P, L, ctypes.c_float, ctypes.c_float]),
        "etf_suggest_chunk_order": (I, [P, P, L, I, P, P, ctypes.POINTER(L), ctypes.POINTER(L)]),
        "etf_suggest_partition": (I, [P, P, L, I, P, P, ctypes.POINTER(L), ctypes.POINTER(L)]),
        "etf_index_stats": (I, [P, ctypes.POINTER(EtfStats)]),
        "etf_index_device_bytes": (L, [P]),
        "etf_index_upload": (I, [P, P, L]),
        "etf_index_layout": (I, [P, ctypes.POINTER(EtfLayout)]),
        "etf_index_export": (I, [P, P, L]),
        "etf_encode_workspace_bytes": (L, [P]),
        "etf_pq_encode_device": (I, [P, P, L, P, P, L]),
        "etf_index_build_device_bytes": (I, [P, L, I, P, ctypes.POINTER(L), ctypes.POINTER(L)]),
        "etf_index_build_device": (I, [P, P, L, P, I, P, P, L, P, L]),
        "etf_workspace_bytes": (L, [P, L, I, I]),
        "etf_last_build_path": (I, [P, ctypes.POINTER(I)]),
        "etf_lut_build": (I, [P, P, L, P]),
        "etf_adc": (I, [P, P, L, I, P, P, L]),
        "etf_search": (I, [P, P, L, I, I, P, P, P, L]),
        "etf_last_fallback_count": (I, [P, ctypes.POINTER(L)]),
        "etf_last_matrix_blocks": (I, [P, ctypes.POINTER(L)]),
        "etf_last_kept_encodings": (I, [P, ctypes.POINTER(L)]),
        "etf_static_scratch_bytes": (L, []),
        "etf_search_static": (I, [P, P, L, I, I, P, P]),
        "etf_profile_enable": (I, [P, I]),
        "etf_profile_read": (I, [P, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(L)]),
        "etf_probe_bandwidth": (I, [P, I, P, P, L]),
        "etf_ivf_set_coarse": (I, [P, P, I]),
        "etf_ivf_assign_workspace_bytes": (L, [P, L]),
        "etf_ivf_assign_device": (I, [P, P, L, P, P, P, L]),
        "etf_ivf_build": (I, [P, P, P, L, P]),
        "etf_ivf_stats": (I, [P, ctypes.POINTER(EtfIvfStats)]),
        "etf_ivf_device_bytes": (L, [P]),
        "etf_ivf_upload": (I, [P, P, L]),
        "etf_ivf_workspace_bytes": (L, [P, L, I, I]),
        "etf_ivf_search": (I, [P, P, L, I, I, P, P, P, L]),
        "etf_kv_append": (I, [P, P, P, P, P, P, I, P]),
        "etf_kv_attend_workspace_bytes": (L, [P, P, I, I, I, I]),
        "etf_kv_attend": (I, [P, P, P, P, I, I, ctypes.c_float, P, P, I, P, P, P, P, P, L]),
        "etf_kv_select_workspace_bytes": (L, [P, P, I, I, I]),
        "etf_kv_select": (I, [P, P, P, P, I, I, P, I, I, I, P, P, L]),
        "etf_kv_evict": (I, [P, P, P, I, I, I, P, P, P, P, P]),
        "etf_kv_evict_ahead": (I, [P, P, P, I, I, I, P, P, P, P, P]),
        "etf_kv_append_packed": (I, [P, P, P, P, P, P, L, P]),
        "etf_kv_take_workspace_bytes": (L, [P, P, I]),
        "etf_kv_take": (I, [P, P, P, I, P, P, P, P, P, L]),
        "etf_kv_fork_workspace_bytes": (L, [P, P]),
        "etf_kv_fork": (I, [P, P, P, P, P, P, L]),
        "etf_kv_free": (I, [P, P, I, P, L]),
        "etf_kv_compact_workspace_bytes": (L, [P, P]),
        "etf_kv_compact": (I, [P, P, P, P, P, P, P, L]),
        "etf_prompt_attend_workspace_bytes": (L, [P, I, L, I, I, I]),
        "etf_prompt_attend": (I, [P, I, I, P, P, P, P, P, P, L, I, I, P, I, ctypes.c_float, P, P, P, L]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _lib = lib
    return lib


def _current_stream(gpu: int) -> int:
    """torch's current stream on that GPU, as a number; 0 for the CPU."""
    if gpu < 0:
        return 0
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # current_stream() without the object around it
    return raw(gpu) if raw is not None else torch.cuda.current_stream(gpu).cuda_stream


def _host(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def _dev(t) -> int:
    """Device pointer of a torch tensor (contiguous, on the GPU)."""
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous GPU tensor")
    return t.data_ptr()


_ad = None    # torch.autograd.forward_ad, once a call has asked for it


def _dual_level() -> bool:
    """Whether tensors may carry tangents: within torch's dual_level() only, whose number torch keeps (-1 outside)."""
    global _ad
    if _ad is None:
        import torch.autograd.forward_ad as _ad
    return getattr(_ad, "_current_level", 0) >= 0


class KvCache:
    """An attention cache in 8 bits: the device tensors of an etf_kv_cache, which the caller owns.

    k, v, bounds: float8_e4m3fn [pages][64][D], [pages][D][64], [pages][2][D]; scales: float32 [pages][2]; tail_k, tail_v: bfloat16 or
    float16 [B][H][2][64][D], [B][H][2][D][64]; table: int32 [B][H][max_blocks]; lens, evicted: int32 [B].  Another tensor of the same
    kind may be assigned to a field: the calls from then on use it.
    """

    FIELDS = ("k", "v", "scales", "bounds", "tail_k", "tail_v", "table", "lens", "evicted")

    def __init__(self, k, v, scales, bounds, tail_k, tail_v, table, lens, evicted):
        import torch
        given = dict(k=k, v=v, scales=scales, bounds=bounds, tail_k=tail_k, tail_v=tail_v, table=table, lens=lens, evicted=evicted)
        if tail_k.dim() != 5 or table.dim() != 3 or k.dim() != 3:
            raise ValueError("expected tail_k [B][H][2][64][D], table [B][H][max_blocks] and k [pages][64][D]")
        B, H, _, _, D = tail_k.shape
        pages, T = k.shape[0], tail_k.dtype
        if T not in (torch.bfloat16, torch.float16):
            raise ValueError("open blocks are bfloat16 or float16, not %s" % T)
        self.batch, self.heads, self.head_dim, self.max_blocks, self.pages, self.dtype, self.device = B, H, D, table.shape[2], pages, T, k.device
        for name, t in given.items():
            self._check(name, t)
        self._t = given
        c = EtfKvCache(ETF_KV_BF16 if T == torch.bfloat16 else ETF_KV_FP16, B, H, D, table.shape[2], pages)
        for name in self.FIELDS:
            setattr(c, name, given[name].data_ptr())
        self._set(c)

    def _check(self, name, t):
        import torch
        B, H, D, S, e4m3 = self.batch, self.heads, self.head_dim, ETF_KV_BLOCK, torch.float8_e4m3fn
        shape, dtype = dict(k=((self.pages, S, D), e4m3), v=((self.pages, D, S), e4m3), scales=((self.pages, 2), torch.float32),
                            bounds=((self.pages, 2, D), e4m3), tail_k=((B, H, 2, S, D), self.dtype), tail_v=((B, H, 2, D, S), self.dtype),
                            table=((B, H, self.max_blocks), torch.int32), lens=((B,), torch.int32), evicted=((B,), torch.int32))[name]
        if not isinstance(t, torch.Tensor) or tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous() or t.device != self.device:
            raise ValueError("%s: expected a contiguous %s tensor %s on %s" % (name, dtype, list(shape), self.device))

    def _set(self, c):
        import torch
        self._c, self._ref = c, ctypes.addressof(c)
        self._gpu = self.device.index if self.device.type == "cuda" else -1
        self._sizes = {}    # workspace bytes by call
        self._raw = self._t["lens"].new_empty(0, dtype=torch.uint8)    # of the kind that workspaces are

    def _field(name):
        def get(self):
            return self._t[name]

        def put(self, t):
            if t is not self._t[name]:    # `cache.lens += n` assigns the tensor that is there
                self._check(name, t)
                self._t[name] = t
                setattr(self._c, name, t.data_ptr())
        return property(get, put)

    k, v, scales, bounds, tail_k, tail_v, table, lens, evicted = map(_field, FIELDS)
    del _field

    @classmethod
    def alloc(cls, batch: int, heads: int, head_dim: int, max_tokens: int, dtype=None, pages: Optional[int] = None, device="cuda"):
        """An empty cache with room for max_tokens a sequence.  pages: None = a page for every block, already in the table;
        else the pool's pages, the table to be filled by the caller (-1 throughout)."""
        import torch
        dtype = torch.bfloat16 if dtype is None else dtype
        S, e4m3 = ETF_KV_BLOCK, torch.float8_e4m3fn
        blocks = max(1, -(-max_tokens // S))
        if pages is None:
            pages = batch * heads * blocks
            table = torch.arange(pages, dtype=torch.int32, device=device).view(batch, heads, blocks)
        else:
            table = torch.full((batch, heads, blocks), -1, dtype=torch.int32, device=device)
        zeros = lambda *shape, dtype: torch.zeros(shape, dtype=dtype, device=device)  # noqa: E731
        return cls(zeros(pages, S, head_dim, dtype=e4m3), zeros(pages, head_dim, S, dtype=e4m3), zeros(pages, 2, dtype=torch.float32),
                   zeros(pages, 2, head_dim, dtype=e4m3), zeros(batch, heads, 2, S, head_dim, dtype=dtype),
                   zeros(batch, heads, 2, head_dim, S, dtype=dtype), table, zeros(batch, dtype=torch.int32), zeros(batch, dtype=torch.int32))

    def fork(self) -> "KvCache":
        """Another table, lens and evicted (uninitialised) over the same pages and open blocks, for Context.kv_evict to write.
        Not a copy of its sequences: that is Context.kv_fork."""
        import torch
        new = KvCache.__new__(KvCache)
        new.__dict__.update(self.__dict__)
        new._t = dict(self._t)
        c = EtfKvCache.from_buffer_copy(self._c)
        for name in ("table", "lens", "evicted"):
            t = new._t[name] = torch.empty_like(self._t[name])
            setattr(c, name, t.data_ptr())
        new._set(c)
        return new


class Context:
    """One etf_ctx.  device=None makes a host-only context (train / encode / build / stats)."""

    def __init__(self, device: Optional[int] = 0, stream: Optional[int] = None):
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        rc = self._lib.etf_create(ctypes.byref(self._h), -1 if device is None else int(device), stream)
        if rc != 0:
            raise EtfError(rc, self._lib.etf_strerror(rc).decode())
        self._keep = {}     # device buffers the library refers to (index image)
        self._stream = stream
        self._device = None if device is None or int(device) < 0 else int(device)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            self._lib.etf_destroy(self._h)
            self._h = ctypes.c_void_p()
            self._keep = {}

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _ck(self, rc: int):
        if rc < 0:
            raise EtfError(int(rc), self._lib.etf_last_error(self._h).decode())
        return rc

    # ---- context
    def set_stream(self, stream: Optional[int]):
        self._ck(self._lib.etf_set_stream(self._h, stream))
        self._stream = stream

    def set_option(self, name: str, value: int):
        self._ck(self._lib.etf_set_option(self._h, name.encode(), int(value)))

    # ---- product quantiser (host)
    def pq_train(self, x: np.ndarray, M: int, K: int, iters: int, seed: int):
        x = np.ascontiguousarray(x, dtype=np.float32)
        self._ck(self._lib.etf_pq_train(self._h, _host(x), x.shape[0], x.shape[1], M, K, iters, seed))
        self._shape = (x.shape[1], M, K)

    def pq_set_codebooks(self, cb: np.ndarray):
        cb = np.ascontiguousarray(cb, dtype=np.float32)
        M, K, ds = cb.shape
        self._ck(self._lib.etf_pq_set_codebooks(self._h, _host(cb), M * ds, M, K))
        self._shape = (M * ds, M, K)

    def pq_set_rotation(self, R: Optional[np.ndarray]):
        """R: [d][d] float32 (the quantiser's space is y = R x), or None to clear."""
        if R is None:
            self._ck(self._lib.etf_pq_set_rotation(self._h, None, 0))
            self._rot_d = 0
            return
        R = np.ascontiguousarray(R, dtype=np.float32)
        if R.ndim != 2 or R.shape[0] != R.shape[1]:
            raise ValueError("expected a square matrix")
        self._ck(self._lib.etf_pq_set_rotation(self._h, _host(R), R.shape[0]))
        self._rot_d = R.shape[0]

    def pq_get_rotation(self) -> np.ndarray:
        d = getattr(self, "_rot_d", 0)
        R = np.zeros((d, d), dtype=np.float32)
        self._ck(self._lib.etf_pq_get_rotation(self._h, _host(R) if d else None))
        return R

    def rotate(self, x: np.ndarray) -> np.ndarray:
        """Host: [n][d] float32 -> R x, float32."""
        x = np.ascontiguousarray(x, dtype=np.float32)
        out = np.empty_like(x)
        if x.ndim != 2 or x.shape[1] != getattr(self, "_rot_d", 0):
            raise ValueError("expected [n][%d] vectors" % getattr(self, "_rot_d", 0))
        self._ck(self._lib.etf_rotate(self._h, _host(x) if len(x) else None, x.shape[0], _host(out) if len(x) else None))
        return out

    def rotate_workspace_bytes(self) -> int:
        return self._ck(self._lib.etf_rotate_workspace_bytes(self._h))

    def rotate_device(self, x, out=None, ws=None):
        """x: float32 device tensor [n][d]; returns R x as a float32 device tensor."""
        import torch
        d = getattr(self, "_rot_d", 0)
        if x.dim() != 2 or x.shape[1] != d or x.dtype != torch.float32 or not x.is_contiguous():
            raise ValueError("expected a contiguous float32 tensor [n][%d]" % d)
        n = x.shape[0]
        if out is None:
            out = torch.empty_like(x)
        if ws is None:
            ws = torch.empty(self.rotate_workspace_bytes() + 256, dtype=torch.uint8, device=x.device)
        p, nb = self._ws(ws)
        self._ck(self._lib.etf_rotate_device(self._h, _dev(x) if n else None, n, _dev(out) if n else None, p, nb))
        return out

    def opq_train(self, x: np.ndarray, M: int, K: int, iters: int, rounds: int, seed: int):
        x = np.ascontiguousarray(x, dtype=np.float32)
        self._ck(self._lib.etf_opq_train(self._h, _host(x), x.shape[0], x.shape[1], M, K, iters, rounds, seed))
        self._shape = (x.shape[1], M, K)
        self._rot_d = x.shape[1]

    def pq_get_codebooks(self) -> np.ndarray:
        d, M, K = self._shape
        cb = np.zeros((M, K, d // M), dtype=np.float32)
        self._ck(self._lib.etf_pq_get_codebooks(self._h, _host(cb)))
        return cb

    def pq_encode(self, x: np.ndarray) -> np.ndarray:
        x = np.ascontiguousarray(x, dtype=np.float32)
        d, M, K = self._shape
        if x.ndim != 2 or x.shape[1] != d:
            raise ValueError("expected [n][%d] vectors" % d)
        codes = np.zeros((x.shape[0], M), dtype=np.uint8)
        self._ck(self._lib.etf_pq_encode(self._h, _host(x), x.shape[0], _host(codes)))
        return codes

    # ---- index (host)
    def index_build(self, codes: np.ndarray, ids: Optional[np.ndarray] = None, T: int = 1,
                    chunk_begin: Optional[Sequence[int]] = None):
        codes = np.ascontiguousarray(codes, dtype=np.uint8)
        d, M, K = self._shape
        if codes.ndim != 2 or codes.shape[1] != M:
            raise ValueError("expected [N][%d] codes" % M)
        ids_a = None if ids is None else np.ascontiguousarray(ids, dtype=np.int32)
        cb = None if chunk_begin is None else np.ascontiguousarray(chunk_begin, dtype=np.int32)
        if cb is not None and cb.shape != (T + 1,):
            raise ValueError("chunk_begin must have T+1 entries")
        self._ck(self._lib.etf_index_build(self._h, _host(codes), codes.shape[0], _host(ids_a), T, _host(cb)))
        self._N = codes.shape[0]

    def index_set_leaf_term(self, term: Optional[np.ndarray]):
        """Additive float32 term per vector for the next index_build (None clears a pending one)."""
        t = None if term is None else np.ascontiguousarray(term, dtype=np.float32)
        self._ck(self._lib.etf_index_set_leaf_term(self._h, _host(t), 0 if t is None else t.shape[0]))

    def index_set_leaf_bytes(self, b: Optional[np.ndarray], scale: float, offset: float):
        """One byte per vector: the next index_build attaches offset + scale * b[n]."""
        a = None if b is None else np.ascontiguousarray(b, dtype=np.uint8)
        self._ck(self._lib.etf_index_set_leaf_bytes(self._h, _host(a), 0 if a is None else a.shape[0], scale, offset))

    def index_set_chunk_order(self, order: Optional[Sequence[int]]):
        """Chunk order of the next index build (a permutation of 0..M-1; None = as given)."""
        o = None if order is None else np.ascontiguousarray(order, dtype=np.int32)
        if o is not None and o.shape != (self._shape[1],):
            raise ValueError("order must have M entries")
        self._ck(self._lib.etf_index_set_chunk_order(self._h, _host(o)))

    def suggest_chunk_order(self, codes: np.ndarray, T: int = 1, chunk_begin: Optional[Sequence[int]] = None):
        """(order, lookups in the given order, lookups in the suggested order) for host codes [N][M]."""
        codes = np.ascontiguousarray(codes, dtype=np.uint8)
        M = self._shape[1]
        if codes.ndim != 2 or codes.shape[1] != M:
            raise ValueError("expected [N][%d] codes" % M)
        cb = None if chunk_begin is None else np.ascontiguousarray(chunk_begin, dtype=np.int32)
        if cb is not None and cb.shape != (T + 1,):
            raise ValueError("chunk_begin must have T+1 entries")
        order = np.zeros(M, dtype=np.int32)
        a, b = ctypes.c_int64(0), ctypes.c_int64(0)
        self._ck(self._lib.etf_suggest_chunk_order(self._h, _host(codes), codes.shape[0], T, _host(cb), _host(order),
                                                   ctypes.byref(a), ctypes.byref(b)))
        return order, int(a.value), int(b.value)

    def suggest_partition(self, codes: np.ndarray, T: int):
        """(chunk_begin, order, lookups with the equal cut, lookups with the suggested cut) for host codes [N][M]."""
        codes = np.ascontiguousarray(codes, dtype=np.uint8)
        M = self._shape[1]
        if codes.ndim != 2 or codes.shape[1] != M:
            raise ValueError("expected [N][%d] codes" % M)
        cb = np.zeros(T + 1, dtype=np.int32)
        order = np.zeros(M, dtype=np.int32)
        a, b = ctypes.c_int64(0), ctypes.c_int64(0)
        self._ck(self._lib.etf_suggest_partition(self._h, _host(codes), codes.shape[0], T, _host(cb), _host(order),
                                                 ctypes.byref(a), ctypes.byref(b)))
        return cb, order, int(a.value), int(b.value)

    def index_stats(self) -> dict:
        st = EtfStats()
        self._ck(self._lib.etf_index_stats(self._h, ctypes.byref(st)))
        return st.as_dict()

    def index_device_bytes(self) -> int:
        return self._ck(self._lib.etf_index_device_bytes(self._h))

    def index_layout(self) -> EtfLayout:
        lay = EtfLayout()
        self._ck(self._lib.etf_index_layout(self._h, ctypes.byref(lay)))
        return lay

    def index_export(self) -> np.ndarray:
        """The device image as a host byte array (what index_upload copies to the GPU)."""
        buf = np.zeros(self.index_device_bytes(), dtype=np.uint8)
        self._ck(self._lib.etf_index_export(self._h, _host(buf), buf.size))
        return buf

    def index_upload(self, dev_buf=None):
        """Uploads the index into dev_buf (uint8 GPU tensor); allocates one with torch if None."""
        import torch
        n = self.index_device_bytes()
        if dev_buf is None:
            dev_buf = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
        off = (-dev_buf.data_ptr()) % 256
        self._ck(self._lib.etf_index_upload(self._h, dev_buf.data_ptr() + off, dev_buf.numel() - off))
        self._keep["index"] = dev_buf
        return dev_buf

    # ---- device
    def workspace_bytes(self, Q: int, k: int, mode: int) -> int:
        return self._ck(self._lib.etf_workspace_bytes(self._h, Q, k, mode))

    def alloc_workspace(self, Q: int, k: int, mode: int):
        import torch
        n = self.workspace_bytes(Q, k, mode)
        return torch.empty(n + 256, dtype=torch.uint8, device="cuda")

    @staticmethod
    def _ws(ws):
        off = (-ws.data_ptr()) % 256
        return ws.data_ptr() + off, ws.numel() - off

    def encode_workspace_bytes(self) -> int:
        return self._ck(self._lib.etf_encode_workspace_bytes(self._h))

    def pq_encode_device(self, x, codes=None, ws=None):
        """x: float32 device tensor [n][d]; returns uint8 device tensor [n][M]."""
        import torch
        d, M, K = self._shape
        if x.dim() != 2 or x.shape[1] != d or x.dtype != torch.float32 or not x.is_contiguous():
            raise ValueError("expected a contiguous float32 tensor [n][%d]" % d)
        n = x.shape[0]
        if codes is None:
            codes = torch.empty((n, M), dtype=torch.uint8, device=x.device)
        if ws is None:
            ws = torch.empty(self.encode_workspace_bytes() + 256, dtype=torch.uint8, device=x.device)
        p, nb = self._ws(ws)
        self._ck(self._lib.etf_pq_encode_device(self._h, _dev(x) if n else None, n, _dev(codes) if n else None, p, nb))
        return codes

    def index_build_device_bytes(self, N: int, T: int = 1, chunk_begin: Optional[Sequence[int]] = None):
        """(image bytes that always suffice, workspace bytes) of a device-side build of N vectors."""
        a, b = ctypes.c_int64(0), ctypes.c_int64(0)
        cb = None if chunk_begin is None else np.ascontiguousarray(chunk_begin, dtype=np.int32)
        if cb is not None and cb.shape != (T + 1,):
            raise ValueError("chunk_begin must have T+1 entries")
        self._ck(self._lib.etf_index_build_device_bytes(self._h, N, T, _host(cb), ctypes.byref(a), ctypes.byref(b)))
        return int(a.value), int(b.value)

    def index_build_device(self, codes, ids=None, T: int = 1, chunk_begin: Optional[Sequence[int]] = None,
                           image=None, ws=None):
        """codes: uint8 device tensor [N][M]; ids: int32 device tensor [N] or None.  Returns the image tensor."""
        import torch
        d, M, K = self._shape
        if codes.dim() != 2 or codes.shape[1] != M or codes.dtype != torch.uint8 or not codes.is_contiguous():
            raise ValueError("expected a contiguous uint8 tensor [N][%d]" % M)
        N = codes.shape[0]
        if ids is not None and (ids.dtype != torch.int32 or ids.shape != (N,) or not ids.is_contiguous()):
            raise ValueError("expected a contiguous int32 tensor [N]")
        cb = None if chunk_begin is None else np.ascontiguousarray(chunk_begin, dtype=np.int32)
        if cb is not None and cb.shape != (T + 1,):
            raise ValueError("chunk_begin must have T+1 entries")
        nimg, nws = self.index_build_device_bytes(N, T, chunk_begin)
        if image is None:
            image = torch.empty(nimg + 256, dtype=torch.uint8, device=codes.device)
        if ws is None:
            ws = torch.empty(nws + 256, dtype=torch.uint8, device=codes.device)
        pi, ni = self._ws(image)
        pw, nw = self._ws(ws)
        self._ck(self._lib.etf_index_build_device(self._h, _dev(codes), N, None if ids is None else _dev(ids), T,
                                                  _host(cb), pi, ni, pw, nw))
        self._keep["index"] = image
        self._N = N
        return image

    def last_build_path(self) -> int:
        """ETF_BUILD_*: the way the index came to the device."""
        v = ctypes.c_int32(0)
        self._ck(self._lib.etf_last_build_path(self._h, ctypes.byref(v)))
        return int(v.value)

    def lut_build(self, queries, lut=None):
        import torch
        d, M, K = self._shape
        Q = queries.shape[0]
        if lut is None:
            lut = torch.empty((Q, M, K), dtype=torch.float32, device=queries.device)
        self._ck(self._lib.etf_lut_build(self._h, _dev(queries), Q, _dev(lut)))
        return lut

    def adc(self, queries, mode: int, dist=None, ws=None):
        import torch
        Q = queries.shape[0]
        if dist is None:
            dist = torch.empty((Q, self._N), dtype=torch.float32, device=queries.device)
        if ws is None:
            ws = self.alloc_workspace(Q, 0, mode)
        p, n = self._ws(ws)
        self._ck(self._lib.etf_adc(self._h, _dev(queries), Q, mode, _dev(dist), p, n))
        return dist

    def search(self, queries, k: int, mode: int, out_ids=None, out_dist=None, ws=None):
        import torch
        Q = queries.shape[0]
        if out_ids is None:
            out_ids = torch.empty((Q, k), dtype=torch.int32, device=queries.device)
        if out_dist is None:
            out_dist = torch.empty((Q, k), dtype=torch.float32, device=queries.device)
        if ws is None:
            ws = self.alloc_workspace(Q, k, mode)
        p, n = self._ws(ws)
        self._ck(self._lib.etf_search(self._h, _dev(queries), Q, k, mode, _dev(out_ids), _dev(out_dist), p, n))
        return out_ids, out_dist

    def search_static(self, queries, k: int, mode: int, out_ids, out_dist):
        """etf_search_static: the caller passes inputs and outputs only; nothing is allocated by the call."""
        self._ck(self._lib.etf_search_static(self._h, _dev(queries), queries.shape[0], k, mode, _dev(out_ids), _dev(out_dist)))
        return out_ids, out_dist

    def last_fallback_count(self) -> int:
        v = ctypes.c_int64(0)
        self._ck(self._lib.etf_last_fallback_count(self._h, ctypes.byref(v)))
        return int(v.value)

    def last_matrix_blocks(self) -> int:
        v = ctypes.c_int64(0)
        self._ck(self._lib.etf_last_matrix_blocks(self._h, ctypes.byref(v)))
        return int(v.value)

    def last_kept_encodings(self) -> int:
        """Encodings the last search's filter looked at, summed over its groups of 32 (M = 8) or 16 queries; 0: its queries were not put
        in order, or the matrix cores filtered all of them (last_matrix_blocks)."""
        v = ctypes.c_int64()
        self._ck(self._lib.etf_last_kept_encodings(self._h, ctypes.byref(v)))
        return int(v.value)

    # ---- IVFADC
    def ivf_set_coarse(self, centroids: np.ndarray):
        c = np.ascontiguousarray(centroids, dtype=np.float32)
        if c.ndim != 2 or c.shape[1] != self._shape[0]:
            raise ValueError("expected [cells][%d] centroids" % self._shape[0])
        self._ck(self._lib.etf_ivf_set_coarse(self._h, _host(c), c.shape[0]))

    def ivf_assign_device(self, x, ws=None):
        """x: float32 device tensor [n][d]; returns (cells int32 [n], codes uint8 [n][M]) device tensors."""
        import torch
        d, M, K = self._shape
        if x.dim() != 2 or x.shape[1] != d or x.dtype != torch.float32 or not x.is_contiguous():
            raise ValueError("expected a contiguous float32 tensor [n][%d]" % d)
        n = x.shape[0]
        cells = torch.empty((n,), dtype=torch.int32, device=x.device)
        codes = torch.empty((n, M), dtype=torch.uint8, device=x.device)
        if ws is None:
            ws = torch.empty(self._ck(self._lib.etf_ivf_assign_workspace_bytes(self._h, n)) + 256, dtype=torch.uint8, device=x.device)
        p, nb = self._ws(ws)
        self._ck(self._lib.etf_ivf_assign_device(self._h, _dev(x) if n else None, n, _dev(cells) if n else None,
                                                 _dev(codes) if n else None, p, nb))
        return cells, codes

    def ivf_build(self, cells: np.ndarray, codes: np.ndarray, ids: Optional[np.ndarray] = None):
        cells = np.ascontiguousarray(cells, dtype=np.int32)
        codes = np.ascontiguousarray(codes, dtype=np.uint8)
        if codes.ndim != 2 or codes.shape[1] != self._shape[1] or cells.shape != (codes.shape[0],):
            raise ValueError("expected cells [N] and codes [N][%d]" % self._shape[1])
        ids_a = None if ids is None else np.ascontiguousarray(ids, dtype=np.int32)
        self._ck(self._lib.etf_ivf_build(self._h, _host(cells), _host(codes), codes.shape[0], _host(ids_a)))

    def ivf_stats(self) -> dict:
        st = EtfIvfStats()
        self._ck(self._lib.etf_ivf_stats(self._h, ctypes.byref(st)))
        return st.as_dict()

    def ivf_upload(self, dev_buf=None):
        import torch
        n = self._ck(self._lib.etf_ivf_device_bytes(self._h))
        if dev_buf is None:
            dev_buf = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
        off = (-dev_buf.data_ptr()) % 256
        self._ck(self._lib.etf_ivf_upload(self._h, dev_buf.data_ptr() + off, dev_buf.numel() - off))
        self._keep["ivf"] = dev_buf
        return dev_buf

    def ivf_workspace_bytes(self, Q: int, k: int, w: int) -> int:
        return self._ck(self._lib.etf_ivf_workspace_bytes(self._h, Q, k, w))

    def ivf_search(self, queries, k: int, w: int, out_ids=None, out_dist=None, ws=None):
        import torch
        Q = queries.shape[0]
        if out_ids is None:
            out_ids = torch.empty((Q, k), dtype=torch.int32, device=queries.device)
        if out_dist is None:
            out_dist = torch.empty((Q, k), dtype=torch.float32, device=queries.device)
        if ws is None:
            ws = torch.empty(self.ivf_workspace_bytes(Q, k, w) + 256, dtype=torch.uint8, device=queries.device)
        p, n = self._ws(ws)
        self._ck(self._lib.etf_ivf_search(self._h, _dev(queries), Q, k, w, _dev(out_ids), _dev(out_dist), p, n))
        return out_ids, out_dist

    # ---- attention over a cache in 8 bits
    def _kv_here(self, cache: KvCache):
        if cache._gpu != self._device and self._device is not None:
            raise ValueError("the cache is on %s, the context on GPU %d" % (cache.device, self._device))

    @staticmethod
    def _rows(t, cache: KvCache, heads: Optional[int], what: str):
        """(pointer, strides) of rows [B][n][heads][D]; dense ones need no strides."""
        if t.dim() != 4 or t.shape[0] != cache.batch or t.shape[3] != cache.head_dim or (heads is not None and t.shape[2] != heads) or \
                t.dtype != cache.dtype or t.get_device() != cache._gpu or t.shape[1] < 1:
            raise ValueError("%s: expected a %s tensor [%d][n][%s][%d] on %s" % (what, cache.dtype, cache.batch, "heads" if heads is None else heads, cache.head_dim, cache.device))
        if t.is_contiguous():
            return t.data_ptr(), None
        s = t.stride()
        if s[3] != 1:
            raise ValueError("%s: a row's elements must be contiguous" % what)
        # of a dimension of one torch allows any stride, which nothing uses
        return t.data_ptr(), (ctypes.c_int64 * 3)(*(s[i] if t.shape[i] > 1 else 0 for i in range(3)))

    @staticmethod
    def _no_gradient(t, what: str):
        if t.requires_grad:
            import torch
            if torch.is_grad_enabled():
                raise ValueError("%s requires a gradient, and the cache calls have none: detach it, or call them under torch.no_grad()" % what)
        if _dual_level() and _ad.unpack_dual(t).tangent is not None:    # torch.no_grad() leaves tangents on
            raise ValueError("%s carries a tangent, and the cache calls have no derivative: detach it" % what)

    @staticmethod
    def _kv_dev(t, shape, dtype, cache: KvCache, what: str):
        if t is None:
            return None
        if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.get_device() != cache._gpu:
            raise ValueError("%s: expected a contiguous %s tensor %s on %s" % (what, dtype, list(shape), cache.device))
        return t.data_ptr()

    def _kv_empty(self, shape, dtype, cache: KvCache):
        """A tensor of the stream that the context's work runs on: neither its earlier nor its later use there needs a wait."""
        import torch
        mine = self._stream or 0
        if _current_stream(cache._gpu) == mine:
            return torch.empty(shape, dtype=dtype, device=cache.device)
        # torch takes a stream of its pool for a pointer of zero
        with torch.cuda.stream(torch.cuda.ExternalStream(mine, device=cache.device) if mine else torch.cuda.default_stream(cache.device)):
            return torch.empty(shape, dtype=dtype, device=cache.device)

    def _kv_scratch(self, cache: KvCache, call, *args):
        key = (call,) + args
        size = cache._sizes.get(key)
        if size is None:
            size = cache._sizes[key] = call(self, cache, *args) + 256
        if _current_stream(cache._gpu) == (self._stream or 0):
            return cache._raw.new_empty(size)    # 1.3 us; torch.empty with a device takes 2.2
        import torch
        return self._kv_empty((size,), torch.uint8, cache)

    def kv_append(self, cache: KvCache, k, v, counts=None):
        """Writes new tokens k, v [B][n][H][D] after cache.lens; the caller then advances cache.lens.  There is no gradient."""
        import torch
        self._kv_here(cache)
        self._no_gradient(k, "k")
        self._no_gradient(v, "v")
        pk, sk = self._rows(k, cache, cache.heads, "k")
        pv, sv = self._rows(v, cache, cache.heads, "v")
        if v.shape[1] != k.shape[1]:
            raise ValueError("k and v have different numbers of tokens")
        pc = self._kv_dev(counts, (cache.batch,), torch.int32, cache, "counts")
        self._ck(self._lib.etf_kv_append(self._h, cache._ref, pk, sk, pv, sv, k.shape[1], pc))

    def kv_attend_workspace_bytes(self, cache: KvCache, n: int, heads_q: int, w: int = 0, mass: bool = False) -> int:
        return self._ck(self._lib.etf_kv_attend_workspace_bytes(self._h, cache._ref, n, heads_q, w, int(mass)))

    def kv_attend(self, cache: KvCache, q, scale: Optional[float] = None, counts=None, lists=None, out=None, lse=None, mass_in=None, mass_out=None, ws=None):
        """Attention of q [B][n][heads_q][D] over the cache, over the blocks of lists (kv_select) if given.  scale: 1 / sqrt(D) by default.
        There is no gradient: tensors that require one are refused where torch would record it."""
        import torch
        self._kv_here(cache)
        self._no_gradient(q, "q")
        pq, sq = self._rows(q, cache, None, "q")
        B, n, heads_q, D = q.shape
        w = 0 if lists is None else lists.shape[-1]
        if lists is not None and w == 0:
            raise ValueError("lists: expected an entry at least (None: all tokens)")
        pl = self._kv_dev(lists, (B, n, cache.heads, w), torch.int32, cache, "lists")
        pc = self._kv_dev(counts, (B,), torch.int32, cache, "counts")
        if out is None:
            if sq is None and _current_stream(cache._gpu) == (self._stream or 0):
                out = torch.empty_like(q)
            else:
                out = self._kv_empty(q.shape, cache.dtype, cache)
            po = out.data_ptr()
        else:
            po = self._kv_dev(out, q.shape, cache.dtype, cache, "out")
        pe = self._kv_dev(lse, (B, n, heads_q), torch.float32, cache, "lse")
        blocks = (B, cache.heads, cache.max_blocks)
        pi = self._kv_dev(mass_in, blocks, torch.float32, cache, "mass_in")
        pm = self._kv_dev(mass_out, blocks, torch.float32, cache, "mass_out")
        if ws is None:
            ws = self._kv_scratch(cache, Context.kv_attend_workspace_bytes, n, heads_q, w, pm is not None)
        pw, nw = self._ws(ws)
        self._ck(self._lib.etf_kv_attend(self._h, cache._ref, pq, sq, n, heads_q, D ** -0.5 if scale is None else scale, pc, pl, w, po, pe, pi, pm, pw, nw))
        return out

    def kv_select_workspace_bytes(self, cache: KvCache, n: int, heads_q: int, w: int) -> int:
        return self._ck(self._lib.etf_kv_select_workspace_bytes(self._h, cache._ref, n, heads_q, w))

    def kv_select(self, cache: KvCache, q, w: int, sink: int = 0, recent: int = 0, counts=None, lists=None, ws=None):
        """Blocks for every token and key/value head: int32 [B][n][H][w], ascending, -1 where there are fewer."""
        import torch
        self._kv_here(cache)
        pq, sq = self._rows(q, cache, None, "q")
        B, n, heads_q, D = q.shape
        pc = self._kv_dev(counts, (B,), torch.int32, cache, "counts")
        if ws is None:
            ws = self._kv_scratch(cache, Context.kv_select_workspace_bytes, n, heads_q, w)
        if lists is None:
            lists = self._kv_empty((B, n, cache.heads, w), torch.int32, cache)
        pl = self._kv_dev(lists, (B, n, cache.heads, w), torch.int32, cache, "lists")
        pw, nw = self._ws(ws)
        self._ck(self._lib.etf_kv_select(self._h, cache._ref, pq, sq, n, heads_q, pc, w, sink, recent, pl, pw, nw))
        return lists

    def kv_evict(self, cache: KvCache, mass, budget: int, sink: int = 0, recent: int = 0, to: Optional[KvCache] = None, mass_out=None, freed=None,
                 ahead: bool = False):
        """Cuts every sequence's cache to `budget` full blocks by mass; returns (mass of what stays, pages taken out).  to: the
        cache (fork()) whose table, lens and evicted are written; None: this one's, and mass is written over.  Entries past the
        full blocks become -1, or, with ahead, stay behind the blocks that stay: pages that kv_take has given ahead of their
        tokens would else be in use for good (a cache whose pages are counted wants ahead=True)."""
        import torch
        self._kv_here(cache)
        blocks = (cache.batch, cache.heads, cache.max_blocks)
        pm = self._kv_dev(mass, blocks, torch.float32, cache, "mass")
        if to is not None and (to.batch, to.heads, to.max_blocks, to.device) != (cache.batch, cache.heads, cache.max_blocks, cache.device):
            raise ValueError("to: expected a cache with a table of the same shape on the same device")
        if mass_out is None:
            mass_out = mass if to is None else self._kv_empty(blocks, torch.float32, cache)
        if freed is None:
            freed = self._kv_empty(blocks, torch.int32, cache)
        po = self._kv_dev(mass_out, blocks, torch.float32, cache, "mass_out")
        pf = self._kv_dev(freed, blocks, torch.int32, cache, "freed")
        c = (cache if to is None else to)._c
        call = self._lib.etf_kv_evict_ahead if ahead else self._lib.etf_kv_evict
        self._ck(call(self._h, cache._ref, pm, budget, sink, recent, c.table, c.lens, c.evicted, po, pf))
        return mass_out, freed

    def kv_append_packed(self, cache: KvCache, k, v, starts):
        """kv_append for packed tokens: k, v [tokens][H][D], sequence b's new ones are [starts[b], starts[b + 1]), starts int32 [B + 1],
        ascending; the caller then advances cache.lens.  There is no gradient."""
        import torch
        self._kv_here(cache)
        if k.requires_grad or v.requires_grad or _dual_level():
            self._no_gradient(k, "k")
            self._no_gradient(v, "v")
        like, tokens = (cache.dtype, cache._gpu), k.shape[0]
        pk, sk = self._packed(k, (tokens, cache.heads, cache.head_dim), like, "k")
        pv, sv = self._packed(v, (tokens, cache.heads, cache.head_dim), like, "v")
        ps = self._kv_dev(starts, (cache.batch + 1,), torch.int32, cache, "starts")
        rc = self._lib.etf_kv_append_packed(self._h, cache._ref, pk, sk, pv, sv, tokens, ps)
        if rc < 0:
            self._ck(rc)

    # ---- pages of the cache
    def _kv_int(self, cache: KvCache):
        """An int32 [1] of the context's stream."""
        if _current_stream(cache._gpu) == (self._stream or 0):
            return cache._t["lens"].new_empty(1)
        import torch
        return self._kv_empty((1,), torch.int32, cache)

    def kv_take_workspace_bytes(self, cache: KvCache, n: int) -> int:
        return self._ck(self._lib.etf_kv_take_workspace_bytes(self._h, cache._ref, n))

    def kv_take(self, cache: KvCache, refs, n: int = 1, counts=None, table_out=None, refs_out=None, missing=None, ws=None):
        """Gives the blocks that an append of counts tokens (None: n of each sequence) completes pages of their own from the free ones of refs
        (int32 [pages]: how many entries name each).  All get one or none does: returns missing, int32 [1], the pages that are lacking.
        table_out, refs_out: written instead of cache.table and refs."""
        import torch
        self._kv_here(cache)
        pr = self._kv_dev(refs, (cache.pages,), torch.int32, cache, "refs")
        pc = self._kv_dev(counts, (cache.batch,), torch.int32, cache, "counts")
        pt = cache._c.table if table_out is None else self._kv_dev(table_out, (cache.batch, cache.heads, cache.max_blocks), torch.int32, cache, "table_out")
        po = pr if refs_out is None else self._kv_dev(refs_out, (cache.pages,), torch.int32, cache, "refs_out")
        if missing is None:
            missing = self._kv_int(cache)
            pm = missing.data_ptr()
        else:
            pm = self._kv_dev(missing, (1,), torch.int32, cache, "missing")
        if ws is None:
            ws = self._kv_scratch(cache, Context.kv_take_workspace_bytes, n)
        pw, nw = self._ws(ws)
        rc = self._lib.etf_kv_take(self._h, cache._ref, pr, n, pc, pt, po, pm, pw, nw)
        if rc < 0:
            self._ck(rc)
        return missing

    def kv_fork_workspace_bytes(self, cache: KvCache) -> int:
        return self._ck(self._lib.etf_kv_fork_workspace_bytes(self._h, cache._ref))

    def kv_fork(self, cache: KvCache, refs, source, keep=None, ws=None):
        """Sequence b becomes a copy of sequence source[b] (int32 [B]; b: it stays; -1: it is emptied), or of its first keep[b] tokens in whole
        blocks: shared pages, an open block of its own.  Writes the cache's table, lens, evicted and open blocks, and refs."""
        import torch
        self._kv_here(cache)
        pr = self._kv_dev(refs, (cache.pages,), torch.int32, cache, "refs")
        ps = self._kv_dev(source, (cache.batch,), torch.int32, cache, "source")
        pk = self._kv_dev(keep, (cache.batch,), torch.int32, cache, "keep")
        if ws is None:
            ws = self._kv_scratch(cache, Context.kv_fork_workspace_bytes)
        pw, nw = self._ws(ws)
        self._ck(self._lib.etf_kv_fork(self._h, cache._ref, pr, ps, pk, pw, nw))

    def kv_free(self, refs, pages):
        """One share less in refs (int32 [pages of the pool]) for each page of the int32 tensor pages (the freed of kv_evict(ahead=True)), entries of -1 aside."""
        import torch
        gpu = refs.get_device()
        if gpu != self._device and self._device is not None:
            raise ValueError("refs is on %s, the context on GPU %d" % (refs.device, self._device))
        if refs.dim() != 1 or refs.dtype != torch.int32 or not refs.is_contiguous():
            raise ValueError("refs: expected a contiguous int32 tensor [pages]")
        if pages.dtype != torch.int32 or not pages.is_contiguous() or pages.get_device() != gpu:
            raise ValueError("pages: expected a contiguous int32 tensor on %s" % refs.device)
        self._ck(self._lib.etf_kv_free(self._h, refs.data_ptr(), refs.numel(), pages.data_ptr(), pages.numel()))

    def kv_compact_workspace_bytes(self, cache: KvCache) -> int:
        return self._ck(self._lib.etf_kv_compact_workspace_bytes(self._h, cache._ref))

    def kv_compact(self, cache: KvCache, refs, table_out=None, refs_out=None, used=None, ws=None):
        """Brings the pages that refs says are in use to the front of the pool; returns used, int32 [1], how many they are.  table_out,
        refs_out: written instead of cache.table and refs."""
        import torch
        self._kv_here(cache)
        pr = self._kv_dev(refs, (cache.pages,), torch.int32, cache, "refs")
        pt = cache._c.table if table_out is None else self._kv_dev(table_out, (cache.batch, cache.heads, cache.max_blocks), torch.int32, cache, "table_out")
        po = pr if refs_out is None else self._kv_dev(refs_out, (cache.pages,), torch.int32, cache, "refs_out")
        if used is None:
            used = self._kv_int(cache)
            pu = used.data_ptr()
        else:
            pu = self._kv_dev(used, (1,), torch.int32, cache, "used")
        if ws is None:
            ws = self._kv_scratch(cache, Context.kv_compact_workspace_bytes)
        pw, nw = self._ws(ws)
        self._ck(self._lib.etf_kv_compact(self._h, cache._ref, pr, pt, po, pu, pw, nw))
        return used

    # ---- attention over whole prompts
    @staticmethod
    def _packed(t, shape, like, what: str):
        """(pointer, strides) of rows [tokens][heads][dim] of the type and on the GPU of `like`; dense ones need no strides."""
        if t.shape != shape or (t.dtype, t.get_device()) != like:
            raise ValueError("%s: expected a %s tensor %s on %s" % (what, like[0], list(shape), "cuda:%d" % like[1] if like[1] >= 0 else "the CPU"))
        if t.is_contiguous():
            return t.data_ptr(), None
        s = t.stride()
        if s[2] != 1:
            raise ValueError("%s: a row's elements must be contiguous" % what)
        # of a dimension of one torch allows any stride, which nothing uses
        return t.data_ptr(), (ctypes.c_int64 * 2)(*(s[i] if shape[i] > 1 else 0 for i in range(2)))

    def prompt_attend_workspace_bytes(self, tokens: int, heads_q: int, heads: int, head_dim: int, batch: int) -> int:
        """Bytes of the workspace, 0 where none is needed."""
        return self._ck(self._lib.etf_prompt_attend_workspace_bytes(self._h, head_dim, tokens, heads_q, heads, batch))

    def prompt_attend(self, q, k, v, starts, scale: Optional[float] = None, out=None, lse=None, ws=None):
        """Causal attention of packed prompts: q [tokens][heads_q][D], k, v [tokens][heads][D], bfloat16 or float16; sequence b has the tokens
        [starts[b], starts[b + 1]), starts int32 [B + 1], ascending.  scale: 1 / sqrt(D) by default; lse: float32 [tokens][heads_q], written if given.
        Rows of tokens that are no sequence's are left as they were.  There is no gradient: tensors that require one are refused
        where torch would record it."""
        import torch
        if q.requires_grad or k.requires_grad or v.requires_grad or _dual_level():
            for t, what in ((q, "q"), (k, "k"), (v, "v")):
                self._no_gradient(t, what)
        dtype, gpu, shape, of_k = q.dtype, q.get_device(), q.shape, k.shape
        if len(shape) != 3 or len(of_k) != 3 or (dtype is not torch.bfloat16 and dtype is not torch.float16):
            raise ValueError("expected q [tokens][heads_q][D] and k [tokens][heads][D], bfloat16 or float16")
        if gpu != self._device and self._device is not None:
            raise ValueError("q is on %s, the context on GPU %d" % (q.device, self._device))
        (tokens, heads_q, D), heads, like = shape, of_k[1], (dtype, gpu)
        pq, sq = self._packed(q, shape, like, "q")
        pk, sk = self._packed(k, (tokens, heads, D), like, "k")
        pv, sv = self._packed(v, (tokens, heads, D), like, "v")
        batch = starts.numel() - 1
        if batch < 1 or starts.dim() != 1 or starts.dtype != torch.int32 or not starts.is_contiguous() or starts.get_device() != gpu:
            raise ValueError("starts: expected a contiguous int32 tensor [B + 1] on %s, B at least 1" % q.device)
        here = _current_stream(gpu) == (self._stream or 0)
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format) if here else self._empty(q, shape, dtype)
        elif out.shape != shape or out.dtype != dtype or not out.is_contiguous() or out.get_device() != gpu:
            raise ValueError("out: expected a contiguous %s tensor %s on %s" % (dtype, list(shape), q.device))
        if lse is not None and (lse.shape != (tokens, heads_q) or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.get_device() != gpu):
            raise ValueError("lse: expected a contiguous float32 tensor [%d][%d] on %s" % (tokens, heads_q, q.device))
        pw, nw = None, 0
        if ws is not None:
            pw, nw = self._ws(ws)
        else:
            size = self.prompt_attend_workspace_bytes(tokens, heads_q, heads, D, batch)
            if size:
                ws = self._empty(q, (size + 256,), torch.uint8)
                pw, nw = self._ws(ws)
        rc = self._lib.etf_prompt_attend(self._h, ETF_KV_BF16 if dtype is torch.bfloat16 else ETF_KV_FP16, D, pq, sq, pk, sk, pv, sv, tokens, heads_q, heads,
                                         starts.data_ptr(), batch, D ** -0.5 if scale is None else scale, out.data_ptr(), None if lse is None else lse.data_ptr(), pw, nw)
        if rc < 0:
            self._ck(rc)
        return out

    def _empty(self, like, shape, dtype):
        """A tensor of the stream that the context's work runs on: neither its earlier nor its later use there needs a wait."""
        import torch
        mine = self._stream or 0
        if _current_stream(like.get_device()) == mine:
            return torch.empty(shape, dtype=dtype, device=like.device)
        # torch takes a stream of its pool for a pointer of zero
        with torch.cuda.stream(torch.cuda.ExternalStream(mine, device=like.device) if mine else torch.cuda.default_stream(like.device)):
            return torch.empty(shape, dtype=dtype, device=like.device)

    def probe_bandwidth(self, kind: int, a, b, nbytes: int):
        """One launch of a streaming probe kernel over the uint8 device tensors a and b (256-byte aligned)."""
        self._ck(self._lib.etf_probe_bandwidth(self._h, kind, _dev(a), _dev(b), nbytes))

    def profile_enable(self, on: bool):
        self._ck(self._lib.etf_profile_enable(self._h, 1 if on else 0))

    def profile_read(self) -> dict:
        """{kernel class: (milliseconds, launches)} since the last read."""
        n = len(KERNEL_CLASSES)
        ms = (ctypes.c_double * n)()
        cnt = (ctypes.c_int64 * n)()
        self._ck(self._lib.etf_profile_read(self._h, ms, cnt))
        return {name: (float(ms[i]), int(cnt[i])) for i, name in enumerate(KERNEL_CLASSES)}
