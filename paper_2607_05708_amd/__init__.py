"""Python binding of libmemattn.so: dense MemAttention retrieval and chunk
materialisation on one MI355X.

Argument marshalling only: every step runs in the library's HIP kernels;
PyTorch supplies device memory and the current stream.  The library must
have been built (``python -m paper_2607_05708_amd.build``); nothing here
falls back to another implementation.

Names follow the C ABI in ``include/memattn.h``:

* ``mem_retrieve_topk``   -- query-aware retrieval (LLMSelect of Algorithm 1
  in the Dense-only form of Section 5.5)
* ``mem_build_relations`` -- cross-chunk relations of every bank row
* ``mem_retrieve_topk_scoped`` / ``mem_build_relations_scoped`` -- the same,
  restricted to each key's (user, session) namespace and to live rows
  (T[u][s] of Section 4.1, tombstones of Section 4.2)
* ``mem_retrieve_topk_grouped`` -- the scoped retrieval over per-namespace
  chunk tables, each query scored against its own table only
* ``mem_gather_chunks``   -- FetchByID + SortByTime through the page table
* ``mem_gather_budget``   -- the same within a memory token budget, packed as
  token rows (the prompt prefix of Section 4.3)
* ``mem_append_chunks``   -- Insert with append-only page allocation
* ``mem_compact_blocks``  -- background block compaction (Eq. 2, Algorithm 2)
* ``mem_colocate``        -- association-aware relocation (Algorithm 2, online stage)

in ``include/memattn_kv.h``, over the same pages and directory:

* ``KvCache``, ``mem_kv_page_bytes`` -- a paged cache of keys and values in 16, 8 or 4 bits
* ``mem_kv_write`` / ``mem_kv_read`` -- quantise tokens into it, read them back
* ``mem_attend``          -- attention of each request's new tokens over its chunks

in ``include/memattn_append.h``:

* ``mem_kv_append``       -- mem_kv_write with the position rotation applied on the way, to keys and queries

and in ``include/memattn_latent.h``:

* ``LatentCache``, ``mem_latent_page_bytes`` -- a paged cache of one latent vector and one rotated key part per token
* ``mem_latent_append`` / ``mem_latent_read`` -- tokens into it, and back
* ``mem_latent_attend``   -- attention with keys and values from the latent vectors, expanded or absorbed
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os

import torch  # noqa: F401  (loads the HIP runtime the library binds to)

__all__ = ["MemError", "MEM_F32", "MEM_BF16", "MEM_ORDER_RANK", "MEM_ORDER_TIME", "library_path", "lib",
           "mem_workspace_bytes", "mem_retrieve_topk", "mem_retrieve_topk_noalloc", "mem_scratch_bytes",
           "mem_build_relations", "mem_retrieve_topk_scoped",
           "mem_build_relations_scoped", "mem_workspace_bytes_grouped", "mem_retrieve_topk_grouped", "mem_gather_chunks", "mem_gather_budget", "mem_append_chunks",
           "mem_compact_workspace_bytes", "mem_compact_blocks", "mem_colocate_workspace_bytes", "mem_colocate",
           "BankState", "MEM_KV_BF16", "MEM_KV_FP8", "MEM_KV_FP4", "KvCache", "mem_kv_page_bytes", "mem_kv_write",
           "mem_kv_append", "mem_kv_read", "mem_attend_workspace_bytes", "mem_attend", "MEM_LATENT_AUTO",
           "MEM_LATENT_ABSORBED", "MEM_LATENT_EXPANDED", "LatentCache", "mem_latent_page_bytes", "mem_latent_append",
           "mem_latent_read", "mem_latent_attend_workspace_bytes", "mem_latent_attend"]

_HERE = os.path.dirname(os.path.abspath(__file__))
MEM_F32, MEM_BF16 = 0, 1
MEM_ORDER_RANK, MEM_ORDER_TIME = 0, 1
MEM_KV_BF16, MEM_KV_FP8, MEM_KV_FP4 = 0, 1, 2
MEM_ROTATE_HALVES, MEM_ROTATE_PAIRS = 0, 1
MEM_LATENT_AUTO, MEM_LATENT_ABSORBED, MEM_LATENT_EXPANDED = 0, 1, 2


class MemBank(C.Structure):
    _fields_ = [("emb", C.c_void_p), ("n", C.c_int64), ("d", C.c_int32), ("dtype", C.c_int32),
                ("row_stride", C.c_int64)]


class MemTopkOut(C.Structure):
    _fields_ = [("idx", C.c_void_p), ("score", C.c_void_p), ("prob", C.c_void_p), ("lse", C.c_void_p)]


class MemPages(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("n_pages", C.c_int64), ("page_bytes", C.c_int64), ("table", C.c_void_p),
                ("n_chunks", C.c_int64), ("pages_per_chunk", C.c_int32)]


class MemChunkTables(C.Structure):
    _fields_ = [("offsets", C.c_void_p), ("chunks", C.c_void_p), ("n_ns", C.c_int32), ("n_entries", C.c_int64)]


class MemCompactResult(C.Structure):
    _fields_ = [("moved_pages", C.c_int64), ("released_blocks", C.c_int64), ("next_free_page", C.c_int64)]


class MemColocateResult(C.Structure):
    _fields_ = [("moved_chunks", C.c_int64), ("groups", C.c_int64), ("next_free_page", C.c_int64)]


class MemKv(C.Structure):
    _fields_ = [("pages", MemPages), ("page_tokens", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32),
                ("format", C.c_int32)]


class MemKvRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class MemRotation(C.Structure):
    _fields_ = [("pos", C.c_void_p), ("freq", C.c_void_p), ("dim", C.c_int32), ("style", C.c_int32)]


class MemLatent(C.Structure):
    _fields_ = [("pages", MemPages), ("page_tokens", C.c_int32), ("latent_dim", C.c_int32), ("rope_dim", C.c_int32),
                ("format", C.c_int32)]


class MemLatentWeights(C.Structure):
    _fields_ = [("data", C.c_void_p), ("head_stride", C.c_int64), ("row_stride", C.c_int64), ("head_dim", C.c_int32)]


class MemAttendArgs(C.Structure):
    _fields_ = [("tok_len", C.c_void_p), ("ids", C.c_void_p), ("m", C.c_int64), ("k", C.c_int32),
                ("heads_q", C.c_int32), ("q_offsets", C.c_void_p), ("q_pos", C.c_void_p), ("scale", C.c_float),
                ("softcap", C.c_float), ("slopes", C.c_void_p), ("causal", C.c_int32), ("window", C.c_int32),
                ("prefix_len", C.c_void_p), ("chunk_ns", C.c_void_p), ("query_ns", C.c_void_p)]


class MemError(RuntimeError):
    def __init__(self, call: str, status: int, message: str):
        super().__init__(f"{call}: status {status}: {message}")
        self.status = status


_lib = None


def library_path() -> str:
    return os.path.join(_HERE, "libmemattn.so")


def lib():
    """Load libmemattn.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python -m paper_2607_05708_amd.build`")
        L = C.CDLL(path)
        P, i64, i32, f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_float
        L.mem_workspace_bytes.argtypes = [i64, i64, i32, i32, i32]
        L.mem_workspace_bytes.restype = C.c_size_t
        L.mem_retrieve_topk.argtypes = [C.POINTER(MemBank), P, i64, i64, i32, f32, MemTopkOut, P, P, C.c_size_t, P]
        L.mem_retrieve_topk.restype = C.c_int
        L.mem_retrieve_topk_noalloc.argtypes = [C.POINTER(MemBank), P, i64, i64, i32, f32, MemTopkOut, P, P]
        L.mem_retrieve_topk_noalloc.restype = C.c_int
        L.mem_scratch_bytes.argtypes = []
        L.mem_scratch_bytes.restype = C.c_size_t
        L.mem_build_relations.argtypes = [C.POINTER(MemBank), i32, f32, i32, MemTopkOut, P, C.c_size_t, P]
        L.mem_build_relations.restype = C.c_int
        L.mem_retrieve_topk_scoped.argtypes = [C.POINTER(MemBank), P, P, P, i64, i64, i32, f32, MemTopkOut, P, P,
                                               C.c_size_t, P]
        L.mem_retrieve_topk_scoped.restype = C.c_int
        L.mem_build_relations_scoped.argtypes = [C.POINTER(MemBank), P, i32, f32, i32, MemTopkOut, P, C.c_size_t, P]
        L.mem_build_relations_scoped.restype = C.c_int
        L.mem_gather_chunks.argtypes = [C.POINTER(MemPages), P, i64, i32, i32, P, P]
        L.mem_gather_chunks.restype = C.c_int
        L.mem_workspace_bytes_grouped.argtypes = [i64, i32, i64, i32, i32]
        L.mem_workspace_bytes_grouped.restype = C.c_size_t
        L.mem_retrieve_topk_grouped.argtypes = [C.POINTER(MemBank), C.POINTER(MemChunkTables), P, P, i64, i64, i32,
                                                f32, MemTopkOut, P, C.c_size_t, P]
        L.mem_retrieve_topk_grouped.restype = C.c_int
        L.mem_gather_budget.argtypes = [C.POINTER(MemPages), P, i32, P, i64, i32, i32, P, P, P, P]
        L.mem_gather_budget.restype = C.c_int
        L.mem_compact_workspace_bytes.argtypes = [i64, i32, i64, i32, i32]
        L.mem_compact_workspace_bytes.restype = C.c_size_t
        L.mem_compact_blocks.argtypes = [P, i64, i64, P, i64, i32, C.POINTER(MemChunkTables), i32, f32, i64, P, P,
                                         C.POINTER(MemCompactResult), P, C.c_size_t, P]
        L.mem_compact_blocks.restype = C.c_int
        L.mem_colocate_workspace_bytes.argtypes = [i64, i32, i64]
        L.mem_colocate_workspace_bytes.restype = C.c_size_t
        L.mem_colocate.argtypes = [P, i64, i64, P, i64, i32, P, P, i64, i32, f32, i32, i64,
                                   C.POINTER(MemColocateResult), P, C.c_size_t, P]
        L.mem_colocate.restype = C.c_int
        L.mem_append_chunks.argtypes = [C.POINTER(MemBank), i64, P, i64, i64, P, i32, C.POINTER(C.c_int64), i64, P]
        L.mem_append_chunks.restype = C.c_int
        L.mem_kv_page_bytes.argtypes = [i32, i32, i32, i32]
        L.mem_kv_page_bytes.restype = C.c_size_t
        for f in (L.mem_kv_write, L.mem_kv_read):
            f.argtypes = [C.POINTER(MemKv), C.POINTER(MemKvRows), C.POINTER(MemKvRows), i32, P, P, i64, P]
            f.restype = C.c_int
        L.mem_attend_workspace_bytes.argtypes = [C.POINTER(MemKv), i64, i32, i64, i32]
        L.mem_attend_workspace_bytes.restype = C.c_size_t
        L.mem_attend.argtypes = [C.POINTER(MemKv), C.POINTER(MemAttendArgs), P, i64, i64, i64, P, P, P, C.c_size_t, P]
        L.mem_attend.restype = C.c_int
        rows = C.POINTER(MemKvRows)
        L.mem_kv_append.argtypes = [C.POINTER(MemKv), rows, rows, rows, rows, i32, i32, C.POINTER(MemRotation), P, P,
                                    i64, P]
        L.mem_kv_append.restype = C.c_int
        L.mem_latent_page_bytes.argtypes = [i32, i32, i32, i32]
        L.mem_latent_page_bytes.restype = C.c_size_t
        L.mem_latent_append.argtypes = [C.POINTER(MemLatent), rows, rows, rows, rows, i32, i32, C.POINTER(MemRotation),
                                        P, P, i64, P]
        L.mem_latent_append.restype = C.c_int
        L.mem_latent_read.argtypes = [C.POINTER(MemLatent), rows, rows, i32, P, P, i64, P]
        L.mem_latent_read.restype = C.c_int
        L.mem_latent_attend_workspace_bytes.argtypes = [C.POINTER(MemLatent), i64, i32, i64, i32, i32, i32]
        L.mem_latent_attend_workspace_bytes.restype = C.c_size_t
        L.mem_latent_attend.argtypes = [C.POINTER(MemLatent), C.POINTER(MemAttendArgs), rows, rows, i64,
                                        C.POINTER(MemLatentWeights), i32, P, P, P, C.c_size_t, P]
        L.mem_latent_attend.restype = C.c_int
        L.mem_status_string.argtypes = [C.c_int]
        L.mem_status_string.restype = C.c_char_p
        L.mem_last_error.argtypes = []
        L.mem_last_error.restype = C.c_char_p
        _lib = L
    return _lib


def _check(call: str, status: int) -> None:
    if status != 0:
        L = lib()
        raise MemError(call, status, f"{L.mem_status_string(status).decode()}: {L.mem_last_error().decode()}")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return MEM_F32
    if t.dtype in (torch.bfloat16, torch.int16, torch.uint16):
        return MEM_BF16
    raise TypeError(f"embeddings must be float32 or bfloat16 (or int16/uint16 bf16 bits), got {t.dtype}")


def _dev(t: torch.Tensor, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    return t


def _rows(t: torch.Tensor, name: str):
    _dev(t, name)
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{name} must be 2-D with unit stride along the embedding dimension")
    return t.shape[0], t.shape[1], t.stride(0)


# The current stream's handle without building a Stream object (2.7 of a small call's 7.6 us on the host).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _get_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_get_device())


def _bank(emb: torch.Tensor, n: int | None = None) -> MemBank:
    rows, d, stride = _rows(emb, "bank")
    return MemBank(emb.data_ptr(), rows if n is None else n, d, _dtype_code(emb), stride)


def mem_workspace_bytes(m: int, n: int, d: int, k: int, dtype: int) -> int:
    return int(lib().mem_workspace_bytes(m, n, d, k, dtype))


def _topk_out(m, k, device, out):
    if out is None:
        out = (torch.empty((m, k), dtype=torch.int32, device=device),
               torch.empty((m, k), dtype=torch.float32, device=device),
               torch.empty((m, k), dtype=torch.float32, device=device),
               torch.empty((m,), dtype=torch.float32, device=device))
    if len(out) != 4:
        raise ValueError("out must be a tuple (idx, score, prob, lse)")
    idx, score, prob, lse = out
    if idx is None:
        raise ValueError("out.idx is required")
    # the kernels write m*k int32/float values (m for lse) through these
    # pointers, so dtype and shape are checked here, before any launch
    for t, nm, dt, shape in ((idx, "idx", torch.int32, (m, k)), (score, "score", torch.float32, (m, k)),
                             (prob, "prob", torch.float32, (m, k)), (lse, "lse", torch.float32, (m,))):
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or t.dtype != dt or t.shape != shape:
            got = f"{t.dtype} {list(t.shape)}" if isinstance(t, torch.Tensor) else type(t).__name__
            raise ValueError(f"out.{nm} must be {dt} of shape {list(shape)}, got {got}")
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"out.{nm} must be a contiguous GPU tensor")
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    return out, MemTopkOut(ptr(idx), ptr(score), ptr(prob), ptr(lse))


def _workspace(device, workspace, size, *args):
    """The caller's workspace (the library checks its size), or one of size(*args) bytes."""
    if workspace is None:
        workspace = torch.empty(max(size(*args), 1), dtype=torch.uint8, device=device)
    _dev(workspace, "workspace")
    return workspace, workspace.numel() * workspace.element_size()


def _full_prob(full_prob, m, n):
    if full_prob is None:
        return None
    _dev(full_prob, "full_prob")
    if full_prob.dtype != torch.float32 or not full_prob.is_contiguous() or tuple(full_prob.shape) != (m, n):
        raise ValueError("full_prob must be a contiguous float32 [m, n] GPU tensor")
    return full_prob.data_ptr()


def _ns(t: torch.Tensor, length: int, name: str) -> int:
    _dev(t, name)
    if t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous() or t.shape[0] != length:
        raise ValueError(f"{name} must be a contiguous int32 [{length}] GPU tensor")
    return t.data_ptr()


def mem_retrieve_topk(bank: torch.Tensor, queries: torch.Tensor, k: int, scale: float = 1.0, *, out=None,
                      full_prob: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """Top-k chunk ids, scores, probabilities and lse per query: (idx, score, prob, lse)."""
    b = _bank(bank)
    m, d, q_stride = _rows(queries, "queries")
    if d != b.d or _dtype_code(queries) != b.dtype:
        raise ValueError("queries must match the bank's dtype and dimension")
    out, o = _topk_out(m, k, bank.device, out)
    ws, ws_bytes = _workspace(bank.device, workspace, mem_workspace_bytes, m, b.n, b.d, k, b.dtype)
    fp = _full_prob(full_prob, m, b.n)
    _check("mem_retrieve_topk", lib().mem_retrieve_topk(C.byref(b), queries.data_ptr(), m, q_stride, k, scale, o, fp,
                                                        ws.data_ptr(), ws_bytes, _stream(stream)))
    return out


def mem_scratch_bytes() -> int:
    return int(lib().mem_scratch_bytes())


def mem_retrieve_topk_noalloc(bank: torch.Tensor, queries: torch.Tensor, k: int, scale: float = 1.0, *, out,
                              full_prob: torch.Tensor | None = None, stream=None):
    """mem_retrieve_topk with the library's fixed scratch array as workspace: the library allocates nothing.
    ``out`` (idx, score, prob, lse) must be supplied by the caller."""
    b = _bank(bank)
    m, d, q_stride = _rows(queries, "queries")
    if d != b.d or _dtype_code(queries) != b.dtype:
        raise ValueError("queries must match the bank's dtype and dimension")
    if out is None:
        raise ValueError("out must be supplied (this call allocates nothing)")
    out, o = _topk_out(m, k, bank.device, out)
    fp = _full_prob(full_prob, m, b.n)
    _check("mem_retrieve_topk_noalloc", lib().mem_retrieve_topk_noalloc(C.byref(b), queries.data_ptr(), m, q_stride,
                                                                        k, scale, o, fp, _stream(stream)))
    return out


def mem_retrieve_topk_scoped(bank: torch.Tensor, row_ns: torch.Tensor, queries: torch.Tensor,
                             query_ns: torch.Tensor, k: int, scale: float = 1.0, *, out=None,
                             full_prob: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                             stream=None):
    """mem_retrieve_topk over each query's namespace: candidates of query i are the bank rows j with
    row_ns[j] >= 0 and row_ns[j] == query_ns[i] (int32 GPU tensors; negative row_ns = tombstoned).
    Rows with fewer than k candidates are padded with id -1, score -inf, p 0."""
    b = _bank(bank)
    m, d, q_stride = _rows(queries, "queries")
    if d != b.d or _dtype_code(queries) != b.dtype:
        raise ValueError("queries must match the bank's dtype and dimension")
    rn, qn = _ns(row_ns, b.n, "row_ns"), _ns(query_ns, m, "query_ns")
    out, o = _topk_out(m, k, bank.device, out)
    ws, ws_bytes = _workspace(bank.device, workspace, mem_workspace_bytes, m, b.n, b.d, k, b.dtype)
    fp = _full_prob(full_prob, m, b.n)
    _check("mem_retrieve_topk_scoped",
           lib().mem_retrieve_topk_scoped(C.byref(b), rn, queries.data_ptr(), qn, m, q_stride, k, scale, o, fp,
                                          ws.data_ptr(), ws_bytes, _stream(stream)))
    return out


def mem_build_relations(bank: torch.Tensor, k: int, scale: float = 1.0, exclude_self: bool = True, *, out=None,
                        workspace: torch.Tensor | None = None, stream=None):
    """Top-k related chunks of every bank row: (idx, score, prob, lse), each [n, ...]."""
    b = _bank(bank)
    out, o = _topk_out(b.n, k, bank.device, out)
    ws, ws_bytes = _workspace(bank.device, workspace, mem_workspace_bytes, b.n, b.n, b.d, k, b.dtype)
    _check("mem_build_relations", lib().mem_build_relations(C.byref(b), k, scale, 1 if exclude_self else 0, o,
                                                            ws.data_ptr(), ws_bytes, _stream(stream)))
    return out


def mem_workspace_bytes_grouped(m: int, n_ns: int, n_entries: int, d: int, k: int) -> int:
    return int(lib().mem_workspace_bytes_grouped(m, n_ns, n_entries, d, k))


def mem_retrieve_topk_grouped(bank: torch.Tensor, offsets: torch.Tensor, chunks: torch.Tensor,
                              queries: torch.Tensor, query_ns: torch.Tensor, k: int, scale: float = 1.0, *,
                              out=None, workspace: torch.Tensor | None = None, stream=None):
    """Retrieval of each query within its own namespace's chunk table (CSR: ``offsets`` int32 [n_ns + 1],
    ``chunks`` int32 bank rows, ascending within a namespace): (idx, score, prob, lse), padded with -1."""
    b = _bank(bank)
    m, d, q_stride = _rows(queries, "queries")
    if d != b.d or _dtype_code(queries) != b.dtype:
        raise ValueError("queries must match the bank's dtype and dimension")
    n_ns = offsets.shape[0] - 1
    _ns(offsets, n_ns + 1, "offsets")
    qn = _ns(query_ns, m, "query_ns")
    n_entries = chunks.shape[0]
    if n_entries:
        _ns(chunks, n_entries, "chunks")
    T = MemChunkTables(offsets.data_ptr(), chunks.data_ptr() if n_entries else None, n_ns, n_entries)
    out, o = _topk_out(m, k, bank.device, out)
    ws, ws_bytes = _workspace(bank.device, workspace, mem_workspace_bytes_grouped, m, n_ns, n_entries, b.d, k)
    _check("mem_retrieve_topk_grouped",
           lib().mem_retrieve_topk_grouped(C.byref(b), C.byref(T), queries.data_ptr(), qn, m, q_stride, k, scale, o,
                                           ws.data_ptr(), ws_bytes, _stream(stream)))
    return out


def mem_build_relations_scoped(bank: torch.Tensor, row_ns: torch.Tensor, k: int, scale: float = 1.0,
                               exclude_self: bool = True, *, out=None, workspace: torch.Tensor | None = None,
                               stream=None):
    """mem_build_relations with each row's candidates limited to the live rows of its own namespace
    (row_ns int32 [n]; a tombstoned row, row_ns < 0, gets an all-padding result)."""
    b = _bank(bank)
    rn = _ns(row_ns, b.n, "row_ns")
    out, o = _topk_out(b.n, k, bank.device, out)
    ws, ws_bytes = _workspace(bank.device, workspace, mem_workspace_bytes, b.n, b.n, b.d, k, b.dtype)
    _check("mem_build_relations_scoped",
           lib().mem_build_relations_scoped(C.byref(b), rn, k, scale, 1 if exclude_self else 0, o, ws.data_ptr(),
                                            ws_bytes, _stream(stream)))
    return out


def mem_gather_chunks(pool: torch.Tensor, table: torch.Tensor, ids: torch.Tensor, order: int = MEM_ORDER_RANK,
                      group: int = 1, *, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Gathered blocks, uint8 [count, pages_per_chunk, page_bytes].

    ``pool``: uint8 [n_pages, page_bytes]; ``table``: int32 [n_chunks, ppc]; ``ids``: int32, any shape
    (flattened in row-major order; with MEM_ORDER_TIME each consecutive ``group`` ids are time-sorted).
    """
    for t, nm in ((pool, "pool"), (table, "table"), (ids, "ids")):
        _dev(t, nm)
        if not t.is_contiguous():
            raise ValueError(f"{nm} must be contiguous")
    if pool.dim() != 2 or table.dim() != 2 or table.dtype != torch.int32 or ids.dtype != torch.int32:
        raise ValueError("pool must be [n_pages, page_bytes]; table and ids int32")
    n_pages, page_bytes = pool.shape[0], pool.shape[1] * pool.element_size()
    n_chunks, ppc = table.shape
    count = ids.numel()
    if out is None:
        out = torch.empty((count, ppc, page_bytes), dtype=torch.uint8, device=pool.device)
    _dev(out, "out")
    if not out.is_contiguous() or out.numel() * out.element_size() != count * ppc * page_bytes:
        raise ValueError("out must be contiguous with count * ppc * page_bytes bytes")
    pg = MemPages(pool.data_ptr(), n_pages, page_bytes, table.data_ptr(), n_chunks, ppc)
    _check("mem_gather_chunks", lib().mem_gather_chunks(C.byref(pg), ids.data_ptr(), count, order, group,
                                                        out.data_ptr(), _stream(stream)))
    return out


def mem_gather_budget(pool: torch.Tensor, table: torch.Tensor, tok_len: torch.Tensor, ids: torch.Tensor,
                      budget_tokens: int, row_bytes: int, *, out=None, stream=None):
    """Budget-aware time-ordered token rows of rank-ordered ids [m, k]:
    (rows uint8 [m, budget_tokens, row_bytes], tokens int32 [m], kept ids int32 [m, k])."""
    for t, nm in ((pool, "pool"), (table, "table"), (tok_len, "tok_len"), (ids, "ids")):
        _dev(t, nm)
        if not t.is_contiguous():
            raise ValueError(f"{nm} must be contiguous")
    if (pool.dim() != 2 or table.dim() != 2 or ids.dim() != 2 or table.dtype != torch.int32
            or ids.dtype != torch.int32 or tok_len.dtype != torch.int32 or tok_len.shape != (table.shape[0],)):
        raise ValueError("pool [n_pages, page_bytes]; table int32 [n_chunks, ppc]; tok_len int32 [n_chunks]; "
                         "ids int32 [m, k]")
    n_pages, page_bytes = pool.shape[0], pool.shape[1] * pool.element_size()
    n_chunks, ppc = table.shape
    m, k = ids.shape
    if out is None:
        out = (torch.empty((m, budget_tokens, row_bytes), dtype=torch.uint8, device=pool.device),
               torch.empty((m,), dtype=torch.int32, device=pool.device),
               torch.empty((m, k), dtype=torch.int32, device=pool.device))
    rows, tokens, kept = out
    _dev(rows, "out rows")
    if not rows.is_contiguous() or rows.numel() * rows.element_size() != m * budget_tokens * row_bytes:
        raise ValueError("out rows must be contiguous with m * budget_tokens * row_bytes bytes")
    pg = MemPages(pool.data_ptr(), n_pages, page_bytes, table.data_ptr(), n_chunks, ppc)
    _check("mem_gather_budget", lib().mem_gather_budget(
        C.byref(pg), tok_len.data_ptr(), row_bytes, ids.data_ptr(), m, k, budget_tokens,
        rows.data_ptr() if rows.numel() else None, _dev(tokens, "out tokens").data_ptr(),
        None if kept is None else _dev(kept, "out ids").data_ptr(), _stream(stream)))
    return out


def mem_compact_workspace_bytes(next_free_page: int, pages_per_block: int, n_entries: int, ppc: int,
                                n_ns: int) -> int:
    return int(lib().mem_compact_workspace_bytes(next_free_page, pages_per_block, n_entries, ppc, n_ns))


def mem_compact_blocks(pool: torch.Tensor, table: torch.Tensor, offsets: torch.Tensor, chunks: torch.Tensor,
                       pages_per_block: int, theta: float, next_free_page: int, *, phi: torch.Tensor | None = None,
                       released: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """Compact blocks whose invalid ratio is >= theta (pool and table updated in place).

    ``offsets`` int32 [n_ns + 1] / ``chunks`` int32: per-namespace live chunk ids (CSR).
    Returns (dict of moved_pages, released_blocks, next_free_page; phi float [n_blocks]; released uint8 [n_blocks]).
    """
    for t, nm in ((pool, "pool"), (table, "table"), (offsets, "offsets"), (chunks, "chunks")):
        _dev(t, nm)
        if not t.is_contiguous():
            raise ValueError(f"{nm} must be contiguous")
    if table.dtype != torch.int32 or offsets.dtype != torch.int32 or chunks.dtype != torch.int32 or pool.dim() != 2:
        raise ValueError("pool [n_pages, page_bytes]; table, offsets and chunks int32")
    n_pages, page_bytes = pool.shape[0], pool.shape[1] * pool.element_size()
    n_chunks, ppc = table.shape
    n_ns, n_entries = offsets.shape[0] - 1, chunks.shape[0]
    n_blocks = (next_free_page + pages_per_block - 1) // pages_per_block
    if phi is None:
        phi = torch.empty(n_blocks, dtype=torch.float32, device=pool.device)
    if released is None:
        released = torch.empty(n_blocks, dtype=torch.uint8, device=pool.device)
    ws, ws_bytes = _workspace(pool.device, workspace, mem_compact_workspace_bytes, next_free_page, pages_per_block,
                              n_entries, ppc, n_ns)
    T = MemChunkTables(offsets.data_ptr(), chunks.data_ptr() if n_entries else None, n_ns, n_entries)
    res = MemCompactResult()
    _check("mem_compact_blocks", lib().mem_compact_blocks(
        pool.data_ptr(), n_pages, page_bytes, table.data_ptr(), n_chunks, ppc, C.byref(T), pages_per_block, theta,
        next_free_page, phi.data_ptr() if n_blocks else None, released.data_ptr() if n_blocks else None,
        C.byref(res), ws.data_ptr(), ws_bytes, _stream(stream)))
    return ({"moved_pages": res.moved_pages, "released_blocks": res.released_blocks,
             "next_free_page": res.next_free_page}, phi, released)


def mem_colocate_workspace_bytes(m: int, k: int, n_chunks: int) -> int:
    return int(lib().mem_colocate_workspace_bytes(m, k, n_chunks))


def mem_colocate(pool: torch.Tensor, table: torch.Tensor, ids: torch.Tensor, scores: torch.Tensor, tau: float,
                 min_group: int, next_free_page: int, *, workspace: torch.Tensor | None = None, stream=None) -> dict:
    """Relocate each key's chunks with score >= tau (groups of at least min_group) into fresh pages, in time
    order; pool and table updated in place.  Returns moved_chunks, groups and next_free_page."""
    for t, nm in ((pool, "pool"), (table, "table"), (ids, "ids"), (scores, "scores")):
        _dev(t, nm)
        if not t.is_contiguous():
            raise ValueError(f"{nm} must be contiguous")
    if (table.dtype != torch.int32 or ids.dtype != torch.int32 or scores.dtype != torch.float32
            or ids.dim() != 2 or scores.shape != ids.shape or pool.dim() != 2):
        raise ValueError("pool [n_pages, page_bytes]; table and ids int32; scores float32 shaped like ids")
    n_pages, page_bytes = pool.shape[0], pool.shape[1] * pool.element_size()
    n_chunks, ppc = table.shape
    m, k = ids.shape
    ws, ws_bytes = _workspace(pool.device, workspace, mem_colocate_workspace_bytes, m, k, n_chunks)
    res = MemColocateResult()
    _check("mem_colocate", lib().mem_colocate(pool.data_ptr(), n_pages, page_bytes, table.data_ptr(), n_chunks, ppc,
                                              ids.data_ptr(), scores.data_ptr(), m, k, tau, min_group,
                                              next_free_page, C.byref(res), ws.data_ptr(), ws_bytes,
                                              _stream(stream)))
    return {"moved_chunks": res.moved_chunks, "groups": res.groups, "next_free_page": res.next_free_page}


class BankState:
    """A bank tensor with spare capacity plus its page table and page allocator.

    ``emb``: [capacity, d] GPU tensor of which the first ``n`` rows are live;
    ``table``: int32 [capacity, ppc] GPU tensor; ``next_free_page``: host counter.
    """

    def __init__(self, emb: torch.Tensor, n: int, table: torch.Tensor, next_free_page: int, n_pages_cap: int):
        self.emb, self.n, self.table = emb, n, table
        self.next_free_page, self.n_pages_cap = next_free_page, n_pages_cap

    @property
    def live(self) -> torch.Tensor:
        return self.emb[: self.n]


def mem_append_chunks(state: BankState, new_emb: torch.Tensor, stream=None) -> BankState:
    """Insert new chunks: bank rows and page-table rows [n, n + m); advances n and the page counter."""
    cap, d, stride = _rows(state.emb, "bank")
    m, d2, new_stride = _rows(new_emb, "new_emb")
    if d2 != d or _dtype_code(new_emb) != _dtype_code(state.emb):
        raise ValueError("new_emb must match the bank's dtype and dimension")
    _dev(state.table, "table")
    if state.table.dtype != torch.int32 or not state.table.is_contiguous() or state.table.shape[0] < cap:
        raise ValueError("table must be a contiguous int32 [capacity, ppc] GPU tensor")
    b = MemBank(state.emb.data_ptr(), state.n, d, _dtype_code(state.emb), stride)
    nfp = C.c_int64(state.next_free_page)
    _check("mem_append_chunks", lib().mem_append_chunks(C.byref(b), cap, new_emb.data_ptr(), m, new_stride,
                                                        state.table.data_ptr(), state.table.shape[1], C.byref(nfp),
                                                        state.n_pages_cap, _stream(stream)))
    state.n, state.next_free_page = int(b.n), int(nfp.value)
    return state


def _stream_for(cache, stream):
    """_stream(stream) for a call over ``cache``, whose GPU has to be the current one (and the stream's): elsewhere the
    kernels would run on another GPU than the one that holds its memory."""
    here = torch.cuda.current_device() if _get_device is None else _get_device()
    if here != cache._dev or (stream is not None and stream.device.index not in (None, here)):
        raise ValueError(f"the cache is on GPU {cache._dev}: make it the current one, and use a stream of it")
    return _stream(stream)


_HERE_TOO = contextlib.nullcontext()


def _memory_of(stream):
    """A context whose allocations are ``stream``'s memory: what held it before is done with when the call's kernels
    write it.  (Memory of the current stream may still be in use there by work that ``stream`` does not wait for.)"""
    return _HERE_TOO if stream is None or stream.cuda_stream == _stream(None) else torch.cuda.stream(stream)


def _used_here(stream, *tensors):
    """Results allocated in ``stream``'s memory may be used on the current stream, and freed, without further notice."""
    if stream is not None and stream.cuda_stream != _stream(None):
        for t in tensors:
            t.record_stream(torch.cuda.current_stream())


def _array(t: torch.Tensor, shape: tuple, name: str, dev: int, dtype=torch.int32) -> int:
    """Pointer of a contiguous array of the given shape on GPU `dev`."""
    if (not isinstance(t, torch.Tensor) or t.get_device() != dev or t.dtype is not dtype or t.shape != shape
            or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} {list(shape)} tensor on the cache's GPU")
    return t.data_ptr()


def _i32(x: int, name: str) -> int:
    """An integer that 32 bits hold (ctypes would cut it to its low bits)."""
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} = {x} does not fit 32 bits")
    return x


def mem_kv_page_bytes(page_tokens: int, heads: int, head_dim: int, format: int) -> int:
    """Bytes of one page of a key/value cache (0 on invalid sizes)."""
    return int(lib().mem_kv_page_bytes(_i32(page_tokens, "page_tokens"), _i32(heads, "heads"),
                                       _i32(head_dim, "head_dim"), _i32(format, "format")))


class KvCache:
    """One layer's paged cache of keys and values over a page pool and its directory.

    ``pool``: uint8 [n_pages, page_bytes] GPU tensor, page_bytes >= mem_kv_page_bytes(...);
    ``table``: int32 [n_chunks, pages_per_chunk] GPU tensor; ``page_tokens`` tokens per page of ``heads`` heads of
    ``head_dim``; ``format``: MEM_KV_BF16, MEM_KV_FP8 or MEM_KV_FP4.  The tensors are kept, not copied: pages may be
    written, gathered, compacted and relocated by the other calls in between.
    """

    def __init__(self, pool: torch.Tensor, table: torch.Tensor, page_tokens: int, heads: int, head_dim: int,
                 format: int):
        _dev(pool, "pool")
        if pool.dim() != 2 or not pool.is_contiguous():
            raise ValueError("pool must be contiguous [n_pages, page_bytes]")
        if table.dim() != 2:
            raise ValueError("table must be int32 [n_chunks, pages_per_chunk]")
        self._dev = pool.get_device()
        ptr = _array(table, tuple(table.shape), "table", self._dev)
        self.pool, self.table = pool, table
        self.page_tokens, self.heads, self.head_dim, self.format = page_tokens, heads, head_dim, format
        pages = MemPages(pool.data_ptr(), pool.shape[0], pool.shape[1] * pool.element_size(), ptr, table.shape[0],
                         table.shape[1])
        self._c = MemKv(pages, _i32(page_tokens, "page_tokens"), _i32(heads, "heads"), _i32(head_dim, "head_dim"),
                        _i32(format, "format"))
        self._ref = C.byref(self._c)


_KV_DTYPES = {torch.float32: MEM_F32, torch.bfloat16: MEM_BF16}


def _kv_rows(cache: KvCache, t: torch.Tensor, n: int, dtype, name: str):
    if (not isinstance(t, torch.Tensor) or t.get_device() != cache._dev or t.dtype is not dtype
            or t.shape != (n, cache.heads, cache.head_dim)):
        raise ValueError(f"{name} must be {dtype} [{n}, {cache.heads}, {cache.head_dim}] on the cache's GPU")
    token, head, one = t.stride()
    if one != 1 and n:
        raise ValueError(f"{name} must have unit stride along its last dimension")
    return C.byref(MemKvRows(t.data_ptr(), token, head))


def _kv_dtype(dtype) -> int:
    code = _KV_DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"keys and values must be float32 or bfloat16, got {dtype}")
    return code


def mem_kv_write(cache: KvCache, k: torch.Tensor, v: torch.Tensor, chunk: torch.Tensor, pos: torch.Tensor, *,
                 stream=None) -> None:
    """Quantise tokens into the cache: rows i of ``k`` and ``v`` ([n, heads, head_dim], float32 or bfloat16, any
    token and head strides) become token ``pos[i]`` of chunk ``chunk[i]`` (int32 [n]).  A chunk of -1 skips the
    token; no two tokens may name one place."""
    n, dtype, dev = k.shape[0], k.dtype, cache._dev
    on = _stream_for(cache, stream)
    status = lib().mem_kv_write(cache._ref, _kv_rows(cache, k, n, dtype, "k"), _kv_rows(cache, v, n, dtype, "v"),
                                _kv_dtype(dtype), _array(chunk, (n,), "chunk", dev), _array(pos, (n,), "pos", dev), n,
                                on)
    _check("mem_kv_write", status)


def _head_rows(cache, t: torch.Tensor, shape: tuple, dtype, name: str):
    """Rows [n, heads, length] of any token and head strides."""
    if not isinstance(t, torch.Tensor) or t.get_device() != cache._dev or t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {list(shape)} on the cache's GPU")
    token, head, one = t.stride()
    if one != 1 and t.numel():
        raise ValueError(f"{name} must have unit stride along its last dimension")
    return MemKvRows(t.data_ptr(), token, head)


def _rotation(cache, at, freq, n: int, pairs: bool) -> MemRotation:
    if not isinstance(freq, torch.Tensor) or freq.dim() != 1:
        raise ValueError("freq must be float32 [pairs]")
    return MemRotation(_array(at, (n,), "at", cache._dev),
                       _array(freq, (freq.shape[0],), "freq", cache._dev, torch.float32), 2 * freq.shape[0],
                       MEM_ROTATE_PAIRS if pairs else MEM_ROTATE_HALVES)


def _turned_queries(cache, q, q_out, n: int, length: int, dtype, stream):
    """(rows of q, rows of q_out, heads, q_out) of an append call; q_out is allocated if it is not given."""
    if q is None:
        if q_out is not None:
            raise ValueError("q_out without q")
        return None, None, 0, None
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError(f"q must be {dtype} [{n}, heads, {length}]")
    shape = (n, q.shape[1], length)
    rows = _head_rows(cache, q, shape, dtype, "q")
    if q_out is None:
        with _memory_of(stream):
            q_out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
        _used_here(stream, q_out)
    return rows, _head_rows(cache, q_out, shape, torch.bfloat16, "q_out"), shape[1], q_out


def _ref(x):
    return None if x is None else C.byref(x)


def mem_kv_append(cache: KvCache, k: torch.Tensor, v: torch.Tensor, chunk: torch.Tensor, pos: torch.Tensor,
                  at: torch.Tensor, freq: torch.Tensor, *, q: torch.Tensor | None = None,
                  q_out: torch.Tensor | None = None, pairs: bool = False, stream=None):
    """mem_kv_write with the keys rotated on the way: the first 2 len(freq) elements of token i's rows by the angles
    ``at[i] * freq`` (``at`` int32 [n], ``freq`` float32; elements j and j + len(freq) are a pair, with ``pairs`` 2 j
    and 2 j + 1).  With ``q`` ([n, heads_q, head_dim], dtype of ``k``) the queries are rotated too: returns them as
    bfloat16, written to ``q_out`` if it is given (q itself, or rows apart from q, k and v)."""
    n, dtype, dev = k.shape[0], k.dtype, cache._dev
    on = _stream_for(cache, stream)
    rot = _rotation(cache, at, freq, n, pairs)
    kr, vr, code = _kv_rows(cache, k, n, dtype, "k"), _kv_rows(cache, v, n, dtype, "v"), _kv_dtype(dtype)
    c_ptr, p_ptr = _array(chunk, (n,), "chunk", dev), _array(pos, (n,), "pos", dev)
    qr, qo, heads_q, q_out = _turned_queries(cache, q, q_out, n, cache.head_dim, dtype, stream)
    _check("mem_kv_append", lib().mem_kv_append(cache._ref, kr, vr, _ref(qr), _ref(qo), heads_q, code, C.byref(rot),
                                                c_ptr, p_ptr, n, on))
    return q_out


def mem_kv_read(cache: KvCache, chunk: torch.Tensor, pos: torch.Tensor, *, dtype=torch.bfloat16, out=None,
                stream=None):
    """Tokens ``pos[i]`` of chunks ``chunk[i]`` (int32 [n]) as dense rows: (k, v), each [n, heads, head_dim] of
    ``dtype`` (or written into ``out``, a pair of such tensors).  Both dtypes hold the cache's values exactly;
    places outside the cache give zeros."""
    n, dev = chunk.shape[0], cache._dev
    on = _stream_for(cache, stream)
    if out is None:
        with _memory_of(stream):
            k = torch.empty((n, cache.heads, cache.head_dim), dtype=dtype, device=cache.pool.device)
            v = torch.empty_like(k)
        _used_here(stream, k, v)
    else:
        k, v = out
        dtype = k.dtype
    status = lib().mem_kv_read(cache._ref, _kv_rows(cache, k, n, dtype, "out k"),
                               _kv_rows(cache, v, n, dtype, "out v"), _kv_dtype(dtype),
                               _array(chunk, (n,), "chunk", dev), _array(pos, (n,), "pos", dev), n, on)
    _check("mem_kv_read", status)
    return k, v


def mem_attend_workspace_bytes(cache: KvCache, m: int, k: int, total_q: int, heads_q: int) -> int:
    return int(lib().mem_attend_workspace_bytes(cache._ref, m, _i32(k, "k"), total_q, _i32(heads_q, "heads_q")))


def mem_attend(cache: KvCache, tok_len: torch.Tensor, ids: torch.Tensor, q: torch.Tensor, scale: float, *,
               q_offsets: torch.Tensor | None = None, q_pos: torch.Tensor | None = None, causal: bool = False,
               window: int = 0, prefix_len: torch.Tensor | None = None, chunk_ns: torch.Tensor | None = None,
               query_ns: torch.Tensor | None = None, softcap: float = 0.0, slopes: torch.Tensor | None = None,
               out=None, workspace: torch.Tensor | None = None, stream=None):
    """Attention of each request's new tokens over its chunks: (out bfloat16 [total_q, heads_q, head_dim], lse
    float32 [total_q, heads_q]).

    ``tok_len`` int32 [n_chunks]: tokens held by each chunk; ``ids`` int32 [m, k]: each request's chunks in context
    order (-1 = none); ``q`` bfloat16 [total_q, heads_q, head_dim], any token and head strides.  Request i's new
    tokens are rows ``q_offsets[i]`` to ``q_offsets[i + 1]`` of q (int32 [m + 1]; None: total_q / m each) and are
    the last of their context unless ``q_pos`` (int32 [total_q]) says where they are.  A token sees positions up to
    its own with ``causal``, above its own minus ``window`` (0: all), always those below ``prefix_len`` (int32 [m]),
    and only chunks whose ``chunk_ns`` (int32 [n_chunks], negative: deleted) equals its ``query_ns`` (int32
    [total_q]).  Scores are ``softcap * tanh(scale <q, k> / softcap) - slopes[head] * distance`` (float32 [heads_q]).
    A token that sees nothing gets zeros and an lse of -inf.
    """
    if ids.dim() != 2 or q.dim() != 3:
        raise ValueError("ids must be int32 [m, k]; q bfloat16 [total_q, heads_q, head_dim]")
    m, k = ids.shape
    total_q, heads_q, d = q.shape
    dev, n_chunks = cache._dev, cache.table.shape[0]
    on = _stream_for(cache, stream)
    token, head, one = q.stride()
    if q.dtype is not torch.bfloat16 or q.get_device() != dev or d != cache.head_dim or (total_q and one != 1):
        raise ValueError(f"q must be bfloat16 [total_q, heads_q, {cache.head_dim}] on the cache's GPU with unit "
                         "stride along the last dimension")
    a = MemAttendArgs(
        _array(tok_len, (n_chunks,), "tok_len", dev), _array(ids, (m, k), "ids", dev), m, k, heads_q,
        None if q_offsets is None else _array(q_offsets, (m + 1,), "q_offsets", dev),
        None if q_pos is None else _array(q_pos, (total_q,), "q_pos", dev), scale, softcap,
        None if slopes is None else _array(slopes, (heads_q,), "slopes", dev, torch.float32), 1 if causal else 0,
        _i32(window, "window"),
        None if prefix_len is None else _array(prefix_len, (m,), "prefix_len", dev),
        None if chunk_ns is None else _array(chunk_ns, (n_chunks,), "chunk_ns", dev),
        None if query_ns is None else _array(query_ns, (total_q,), "query_ns", dev))
    if out is None:
        with _memory_of(stream):
            o = torch.empty((total_q, heads_q, d), dtype=torch.bfloat16, device=q.device)
            lse = torch.empty((total_q, heads_q), dtype=torch.float32, device=q.device)
        _used_here(stream, o, lse)
        o_ptr, lse_ptr = o.data_ptr(), lse.data_ptr()
    else:
        o, lse = out
        o_ptr = _array(o, (total_q, heads_q, d), "out", dev, torch.bfloat16)
        lse_ptr = None if lse is None else _array(lse, (total_q, heads_q), "out lse", dev, torch.float32)
    if workspace is None:
        with _memory_of(stream):
            workspace = torch.empty(max(mem_attend_workspace_bytes(cache, m, k, total_q, heads_q), 1),
                                    dtype=torch.uint8, device=q.device)
    if not isinstance(workspace, torch.Tensor) or workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the cache's GPU")
    status = lib().mem_attend(cache._ref, C.byref(a), q.data_ptr(), total_q, token, head, o_ptr, lse_ptr,
                              workspace.data_ptr(), workspace.nbytes, on)
    _check("mem_attend", status)
    return o, lse


def mem_latent_page_bytes(page_tokens: int, latent_dim: int, rope_dim: int, format: int) -> int:
    """Bytes of one page of a latent cache (0 on invalid sizes)."""
    return int(lib().mem_latent_page_bytes(_i32(page_tokens, "page_tokens"), _i32(latent_dim, "latent_dim"),
                                           _i32(rope_dim, "rope_dim"), _i32(format, "format")))


class LatentCache:
    """One layer's paged cache of a latent vector and a rotated key part per token, over a page pool and its directory.

    ``pool``: uint8 [n_pages, page_bytes] GPU tensor, page_bytes >= mem_latent_page_bytes(...); ``table``: int32
    [n_chunks, pages_per_chunk] GPU tensor; ``page_tokens`` tokens per page of ``latent_dim`` elements in ``format``
    (MEM_KV_BF16, MEM_KV_FP8 or MEM_KV_FP4) and ``rope_dim`` in bf16.  The tensors are kept, not copied.
    """

    def __init__(self, pool: torch.Tensor, table: torch.Tensor, page_tokens: int, latent_dim: int, rope_dim: int,
                 format: int):
        _dev(pool, "pool")
        if pool.dim() != 2 or not pool.is_contiguous():
            raise ValueError("pool must be contiguous [n_pages, page_bytes]")
        if table.dim() != 2:
            raise ValueError("table must be int32 [n_chunks, pages_per_chunk]")
        self._dev = pool.get_device()
        ptr = _array(table, tuple(table.shape), "table", self._dev)
        self.pool, self.table = pool, table
        self.page_tokens, self.latent_dim, self.rope_dim, self.format = page_tokens, latent_dim, rope_dim, format
        pages = MemPages(pool.data_ptr(), pool.shape[0], pool.shape[1] * pool.element_size(), ptr, table.shape[0],
                         table.shape[1])
        self._c = MemLatent(pages, _i32(page_tokens, "page_tokens"), _i32(latent_dim, "latent_dim"),
                            _i32(rope_dim, "rope_dim"), _i32(format, "format"))
        self._ref = C.byref(self._c)


def _token_rows(cache: LatentCache, t: torch.Tensor, n: int, length: int, dtype, name: str):
    """Rows [n, length] of any token stride."""
    if (not isinstance(t, torch.Tensor) or t.get_device() != cache._dev or t.dtype is not dtype
            or t.shape != (n, length)):
        raise ValueError(f"{name} must be {dtype} [{n}, {length}] on the cache's GPU")
    token, one = t.stride()
    if one != 1 and n:
        raise ValueError(f"{name} must have unit stride along its last dimension")
    return MemKvRows(t.data_ptr(), token, 0)


def mem_latent_append(cache: LatentCache, c: torch.Tensor, r: torch.Tensor, chunk: torch.Tensor, pos: torch.Tensor,
                      at: torch.Tensor | None = None, freq: torch.Tensor | None = None, *,
                      q: torch.Tensor | None = None, q_out: torch.Tensor | None = None, pairs: bool = False,
                      stream=None):
    """Append tokens: rows i of ``c`` [n, latent_dim] and ``r`` [n, rope_dim] (float32 or bfloat16, any token stride)
    become token ``pos[i]`` of chunk ``chunk[i]`` (int32 [n]; a chunk of -1 skips the token), ``r`` rotated by the
    angles ``at[i] * freq`` as in mem_kv_append (without ``at`` and ``freq`` it is rotated already).  With ``q``
    ([n, heads, rope_dim], dtype of ``c``: the rotated part of the queries) these are rotated too: returns them as
    bfloat16, written to ``q_out`` if it is given."""
    n, dtype, dev = c.shape[0], c.dtype, cache._dev
    on = _stream_for(cache, stream)
    if (at is None) != (freq is None):
        raise ValueError("at and freq belong together")
    rot = None if at is None else _rotation(cache, at, freq, n, pairs)
    cr = _token_rows(cache, c, n, cache.latent_dim, dtype, "c")
    rr = _token_rows(cache, r, n, cache.rope_dim, dtype, "r")
    code = _kv_dtype(dtype)
    c_ptr, p_ptr = _array(chunk, (n,), "chunk", dev), _array(pos, (n,), "pos", dev)
    qr, qo, heads_q, q_out = _turned_queries(cache, q, q_out, n, cache.rope_dim, dtype, stream)
    _check("mem_latent_append", lib().mem_latent_append(cache._ref, C.byref(cr), C.byref(rr), _ref(qr), _ref(qo),
                                                        heads_q, code, _ref(rot), c_ptr, p_ptr, n, on))
    return q_out


def mem_latent_read(cache: LatentCache, chunk: torch.Tensor, pos: torch.Tensor, *, dtype=torch.bfloat16, out=None,
                    stream=None):
    """Tokens ``pos[i]`` of chunks ``chunk[i]`` (int32 [n]) as dense rows: (c [n, latent_dim], r [n, rope_dim]) of
    ``dtype`` (or written into ``out``, a pair of such tensors).  Both dtypes hold the cache's values exactly; places
    outside the cache give zeros."""
    n, dev = chunk.shape[0], cache._dev
    on = _stream_for(cache, stream)
    if out is None:
        with _memory_of(stream):
            c = torch.empty((n, cache.latent_dim), dtype=dtype, device=cache.pool.device)
            r = torch.empty((n, cache.rope_dim), dtype=dtype, device=cache.pool.device)
        _used_here(stream, c, r)
    else:
        c, r = out
        dtype = c.dtype
    cr = _token_rows(cache, c, n, cache.latent_dim, dtype, "out c")
    rr = _token_rows(cache, r, n, cache.rope_dim, dtype, "out r")
    _check("mem_latent_read", lib().mem_latent_read(cache._ref, C.byref(cr), C.byref(rr), _kv_dtype(dtype),
                                                    _array(chunk, (n,), "chunk", dev), _array(pos, (n,), "pos", dev),
                                                    n, on))
    return c, r


def mem_latent_attend_workspace_bytes(cache: LatentCache, m: int, k: int, total_q: int, heads: int, head_dim: int,
                                      form: int = MEM_LATENT_AUTO) -> int:
    return int(lib().mem_latent_attend_workspace_bytes(cache._ref, m, _i32(k, "k"), total_q, _i32(heads, "heads"),
                                                       _i32(head_dim, "head_dim"), _i32(form, "form")))


def mem_latent_attend(cache: LatentCache, tok_len: torch.Tensor, ids: torch.Tensor, q: torch.Tensor, t: torch.Tensor,
                      w: torch.Tensor, scale: float, *, q_offsets: torch.Tensor | None = None,
                      q_pos: torch.Tensor | None = None, causal: bool = False, window: int = 0,
                      prefix_len: torch.Tensor | None = None, chunk_ns: torch.Tensor | None = None,
                      query_ns: torch.Tensor | None = None, form: int = MEM_LATENT_AUTO,
                      out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Attention of each request's new tokens over its chunks, keys and values from the latent vectors: out bfloat16
    [total_q, heads, head_dim].

    ``q`` [total_q, heads, head_dim] and ``t`` [total_q, heads, rope_dim] (bfloat16, any token and head strides): the
    queries and their rotated part; ``w`` bfloat16 [heads, 2 * head_dim, latent_dim] (any head and row strides): a
    head's keys are ``[w[h, :head_dim] c, r]``, its values ``w[h, head_dim:] c``.  Scores are ``scale (<q, W c> + <t,
    r>)``.  Requests, positions and masks as in mem_attend.  ``form``: MEM_LATENT_ABSORBED, MEM_LATENT_EXPANDED, or
    MEM_LATENT_AUTO, which goes by the mean of the requests' new tokens alone: with a short window, turns of unlike
    length, or lists with room for much more than they hold (the expanded form's workspace grows with it), name the
    form.  ``lse`` (float32 [total_q, heads]) receives the log sums if it is given.  A token that
    sees nothing gets zeros and an lse of -inf.
    """
    if ids.dim() != 2 or q.dim() != 3 or w.dim() != 3:
        raise ValueError("ids must be int32 [m, k]; q [total_q, heads, head_dim], w [heads, 2 * head_dim, latent_dim]")
    m, k = ids.shape
    total_q, heads, d = q.shape
    dev, n_chunks = cache._dev, cache.table.shape[0]
    on = _stream_for(cache, stream)
    qr = _head_rows(cache, q, (total_q, heads, d), torch.bfloat16, "q")
    tr = _head_rows(cache, t, (total_q, heads, cache.rope_dim), torch.bfloat16, "t")
    wr = _head_rows(cache, w, (heads, 2 * d, cache.latent_dim), torch.bfloat16, "w")
    weights = MemLatentWeights(wr.data, wr.token_stride, wr.head_stride, d)
    a = MemAttendArgs(
        _array(tok_len, (n_chunks,), "tok_len", dev), _array(ids, (m, k), "ids", dev), m, k, heads,
        None if q_offsets is None else _array(q_offsets, (m + 1,), "q_offsets", dev),
        None if q_pos is None else _array(q_pos, (total_q,), "q_pos", dev), scale, 0.0, None, 1 if causal else 0,
        _i32(window, "window"),
        None if prefix_len is None else _array(prefix_len, (m,), "prefix_len", dev),
        None if chunk_ns is None else _array(chunk_ns, (n_chunks,), "chunk_ns", dev),
        None if query_ns is None else _array(query_ns, (total_q,), "query_ns", dev))
    if out is None:
        with _memory_of(stream):
            out = torch.empty((total_q, heads, d), dtype=torch.bfloat16, device=q.device)
        _used_here(stream, out)
    o_ptr = _array(out, (total_q, heads, d), "out", dev, torch.bfloat16)
    lse_ptr = None if lse is None else _array(lse, (total_q, heads), "lse", dev, torch.float32)
    if workspace is None:
        with _memory_of(stream):
            workspace = torch.empty(max(mem_latent_attend_workspace_bytes(cache, m, k, total_q, heads, d, form), 1),
                                    dtype=torch.uint8, device=q.device)
    if not isinstance(workspace, torch.Tensor) or workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the cache's GPU")
    _check("mem_latent_attend", lib().mem_latent_attend(
        cache._ref, C.byref(a), C.byref(qr), C.byref(tr), total_q, C.byref(weights), _i32(form, "form"), o_ptr, lse_ptr,
        workspace.data_ptr(), workspace.nbytes, on))
    return out
