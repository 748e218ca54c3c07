"""ctypes binding of libchunkkv.so: argument marshalling only.

Every function has the name and argument order of its C-ABI entry point in include/chunkkv.h
(ChunkKV Algorithms 1-3); tensors are passed as device pointers, the current torch stream is used,
and a non-zero status raises ChunkKVError.  There is no fallback: without the built HIP library every
call raises.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libchunkkv.so")

F32, BF16, F16 = 0, 1, 2
FLAG_WHOLE_CHUNKS, FLAG_TWO_PASS = 1, 2     # chunkkv_problem.flags
SYMBOLS = ("chunkkv_status_string", "chunkkv_workspace_bytes", "chunkkv_score", "chunkkv_chunk_topk",
           "chunkkv_compact", "chunkkv_compress_stack", "chunkkv_score_lse", "chunkkv_compress_stack_lse",
           "chunkkv_compress_layer", "chunkkv_workspace_bytes_hybrid", "chunkkv_compress_stack_hybrid", "chunkkv_jaccard", "chunkkv_decode_workspace_bytes", "chunkkv_decode_attention",
           "chunkkv_decode_attention_static", "chunkkv_quality_workspace_bytes", "chunkkv_quality_metrics",
           "chunkkv_paged_compact", "chunkkv_paged_append", "chunkkv_paged_decode_workspace_bytes", "chunkkv_paged_decode_attention",
           "chunkkv_paged_evict_workspace_bytes", "chunkkv_paged_evict",
           "chunkkv_timing_begin",
           "chunkkv_timing_end")
TIMING_KINDS = ("score_stats", "stats_merge", "score_colsum", "chunk_sums", "chunk_topk", "compact", "decode")


class ChunkKVError(RuntimeError):
    def __init__(self, status: int, where: str, msg: str):
        super().__init__(f"{where}: status {status} ({msg})")
        self.status = status


class _CProblem(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("window", C.c_int32), ("chunk", C.c_int32), ("dtype", C.c_int32), ("softmax_scale", C.c_float),
        ("seqlen", C.POINTER(C.c_int32)), ("n_keep", C.POINTER(C.c_int32)), ("kv_base", C.POINTER(C.c_int64)),
        ("kv_stride_head", C.c_int64), ("kv_stride_tok", C.c_int64),
        ("out_base", C.POINTER(C.c_int64)), ("out_stride_head", C.c_int64), ("out_stride_tok", C.c_int64),
        ("sel_cap", C.c_int32), ("score_cap", C.c_int32), ("flags", C.c_uint32),
    ]


class _KeepsStruct:
    __slots__ = ("_kept",)   # beside the fields, not among them: vars() of a Problem holds its fields only


@dataclass
class Problem(_KeepsStruct):
    """Python mirror of chunkkv_problem (see include/chunkkv.h for the meaning of every field)."""
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    window: int
    chunk: int
    dtype: int
    seqlen: Sequence[int]
    n_keep: Sequence[int]
    kv_base: Sequence[int]
    kv_stride_head: int
    kv_stride_tok: int
    out_base: Optional[Sequence[int]] = None
    out_stride_head: int = 0
    out_stride_tok: int = 0
    sel_cap: int = 0
    score_cap: int = 0
    softmax_scale: float = 0.0
    flags: int = 0

    def __post_init__(self):
        c = self.chunk if self.chunk > 0 else 1
        if self.sel_cap == 0:
            self.sel_cap = max((max(int(n), 0) + c - 1) // c + 1 for n in self.n_keep)
        if self.score_cap == 0:
            self.score_cap = max(1, max((int(L) - self.window + c - 1) // c for L in self.seqlen))
        if self.out_base is None:
            kept = [int(n) + self.window for n in self.n_keep]
            if len(set(kept)) == 1:
                # default output [B][Hkv][n_kept][d]
                per_seq = self.n_kv_heads * kept[0] * self.head_dim
                self.out_base = [b * per_seq for b in range(len(kept))]
                self.out_stride_head = kept[0] * self.head_dim
                self.out_stride_tok = self.head_dim
            else:
                # ragged budgets: packed [sum n_kept][Hkv][d]
                run, base = 0, []
                for n in kept:
                    base.append(run * self.n_kv_heads * self.head_dim)
                    run += n
                self.out_base = base
                self.out_stride_head = self.head_dim
                self.out_stride_tok = self.n_kv_heads * self.head_dim

    def out_elements(self) -> int:
        """Elements of one output buffer (K' or V') under the default output layouts."""
        return sum(int(n) + self.window for n in self.n_keep) * self.n_kv_heads * self.head_dim

    @property
    def batch(self) -> int:
        return len(self.seqlen)

    # The C struct of a Problem is kept between calls: building it costs 5 us (8 us for a batch of 8), as much as a
    # decoding step's two launches.  Any field can change in place, a tensor or an array among them, so the struct is
    # kept with the plain numbers it holds, and every field is compared with them on every call (0.5 us, 0.6 us for a batch of 8).
    def _c(self):
        now = (self.n_q_heads, self.n_kv_heads, self.head_dim, self.window, self.chunk, self.dtype, self.softmax_scale,
               self.kv_stride_head, self.kv_stride_tok, self.out_stride_head, self.out_stride_tok, self.sel_cap, self.score_cap,
               self.flags, tuple(self.seqlen), tuple(self.n_keep), tuple(self.kv_base), tuple(self.out_base))
        kept = getattr(self, "_kept", None)
        if kept is None or kept[0] != now:
            cp = self.as_c()
            plain = tuple(tuple(map(int, x)) if isinstance(x, tuple) else float(x) if isinstance(x, float) else int(x) for x in now)
            kept = self._kept = (plain, cp, C.byref(cp), self._kv_elements(cp))
        return kept[2]

    @staticmethod
    def _kv_elements(cp) -> int:
        """Elements from the start of a cache to the end of its last row, by the struct: a list that is too short goes on with zeros there."""
        return (max((cp.kv_base[b] + (cp.seqlen[b] - 1) * cp.kv_stride_tok for b in range(cp.batch)), default=0)
                + (cp.n_kv_heads - 1) * cp.kv_stride_head + cp.head_dim)

    def __getstate__(self):
        return self.__dict__.copy()   # the kept struct is neither copied nor pickled

    def as_c(self):
        B = self.batch
        keep = {
            "seqlen": (C.c_int32 * B)(*[int(x) for x in self.seqlen]),
            "n_keep": (C.c_int32 * B)(*[int(x) for x in self.n_keep]),
            "kv_base": (C.c_int64 * B)(*[int(x) for x in self.kv_base]),
            "out_base": (C.c_int64 * B)(*[int(x) for x in self.out_base]),
        }
        cp = _CProblem(B, self.n_q_heads, self.n_kv_heads, self.head_dim, self.window, self.chunk, self.dtype,
                       self.softmax_scale, keep["seqlen"], keep["n_keep"], keep["kv_base"],
                       self.kv_stride_head, self.kv_stride_tok, keep["out_base"], self.out_stride_head,
                       self.out_stride_tok, self.sel_cap, self.score_cap, int(self.flags))
        cp._keep = keep
        return cp


class _CPages(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
        ("softmax_scale", C.c_float), ("page_tokens", C.c_int32), ("n_pages", C.c_int32), ("table_pitch", C.c_int32), ("slot_pitch", C.c_int32),
        ("stride_page", C.c_int64), ("stride_head", C.c_int64), ("stride_tok", C.c_int64), ("max_tokens", C.POINTER(C.c_int32)),
    ]


@dataclass
class Pages(_KeepsStruct):
    """Python mirror of chunkkv_pages (see include/chunkkv.h for the meaning of every field).  Without strides the pools are
    [n_pages][n_kv_heads][page_tokens][head_dim]; without pitches the arrays are as wide as max_tokens needs."""
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    dtype: int
    page_tokens: int
    n_pages: int
    max_tokens: Sequence[int]
    stride_page: int = 0
    stride_head: int = 0
    stride_tok: int = 0
    table_pitch: int = 0
    slot_pitch: int = 0
    softmax_scale: float = 0.0

    def __post_init__(self):
        if self.stride_tok == 0:
            self.stride_tok = self.head_dim
            self.stride_head = self.page_tokens * self.head_dim
            self.stride_page = self.n_kv_heads * self.stride_head
        most = max([1] + [int(n) for n in self.max_tokens])
        if self.table_pitch == 0:
            self.table_pitch = -(-most // max(1, self.page_tokens))
        if self.slot_pitch == 0:
            self.slot_pitch = most

    @property
    def batch(self) -> int:
        return len(self.max_tokens)

    def pool_elements(self) -> int:
        """Elements from the start of a pool to the end of its last row."""
        return ((self.n_pages - 1) * self.stride_page + (self.n_kv_heads - 1) * self.stride_head
                + (self.page_tokens - 1) * self.stride_tok + self.head_dim)

    # As the struct of a Problem: kept with the numbers it holds, which are compared on every call.
    def _c(self):
        now = (self.n_q_heads, self.n_kv_heads, self.head_dim, self.dtype, self.page_tokens, self.n_pages, self.stride_page, self.stride_head,
               self.stride_tok, self.table_pitch, self.slot_pitch, self.softmax_scale, tuple(self.max_tokens))
        kept = getattr(self, "_kept", None)
        if kept is None or kept[0] != now:
            cp = self.as_c()
            plain = tuple(tuple(map(int, x)) if isinstance(x, tuple) else float(x) if isinstance(x, float) else int(x) for x in now)
            kept = self._kept = (plain, cp, C.byref(cp), self.pool_elements())
        return kept[2]

    def _pool_elements(self) -> int:   # of the struct that _c() has just returned
        return self._kept[3]

    def __getstate__(self):
        return self.__dict__.copy()

    def as_c(self):
        B = self.batch
        most = (C.c_int32 * B)(*[int(x) for x in self.max_tokens])
        cp = _CPages(B, self.n_q_heads, self.n_kv_heads, self.head_dim, self.dtype, self.softmax_scale, self.page_tokens, self.n_pages,
                     self.table_pitch, self.slot_pitch, self.stride_page, self.stride_head, self.stride_tok, most)
        # a number that does not fit its type would be another one for the library than for the checks of sizes
        for name, kind in _CPages._fields_[:-1]:
            if kind is not C.c_float and getattr(cp, name) != getattr(self, name, B):
                raise ValueError(f"chunkkv_pages.{name}: {getattr(self, name)} does not fit")
        _fits("chunkkv_pages.max_tokens", most, self.max_tokens)
        cp._keep = most
        return cp


def _fits(what: str, host, numbers: Sequence[int]):
    if list(host) != [int(x) for x in numbers]:
        raise ValueError(f"{what}: {list(numbers)} does not fit")


_lib = None


def load_library(path: Optional[str] = None):
    """Loads libchunkkv.so (built in-tree by `python -m paper_2502_00299_amd.build`)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is missing: build it with `python -m paper_2502_00299_amd.build` "
                           "(there is no CPU fallback)")
    lib = C.CDLL(p)
    vp, i32p, f32p = C.c_void_p, C.c_void_p, C.c_void_p
    lib.chunkkv_status_string.restype = C.c_char_p
    lib.chunkkv_status_string.argtypes = [C.c_int]
    lib.chunkkv_workspace_bytes.restype = C.c_size_t
    lib.chunkkv_workspace_bytes.argtypes = [C.POINTER(_CProblem), C.c_int32, C.c_int32]
    lib.chunkkv_score.restype = C.c_int
    lib.chunkkv_score.argtypes = [C.POINTER(_CProblem), vp, vp, f32p, f32p, vp, C.c_size_t, vp]
    lib.chunkkv_chunk_topk.restype = C.c_int
    lib.chunkkv_chunk_topk.argtypes = [C.POINTER(_CProblem), f32p, i32p, i32p, i32p, vp, C.c_size_t, vp]
    lib.chunkkv_compact.restype = C.c_int
    lib.chunkkv_compact.argtypes = [C.POINTER(_CProblem), vp, vp, i32p, i32p, i32p, vp, vp, vp]
    lib.chunkkv_compress_stack.restype = C.c_int
    lib.chunkkv_compress_stack.argtypes = [C.POINTER(_CProblem), C.c_int32, C.c_int32, C.POINTER(vp), C.POINTER(vp),
                                           C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), i32p, i32p, i32p, vp,
                                           C.c_size_t, vp]
    lib.chunkkv_score_lse.restype = C.c_int
    lib.chunkkv_score_lse.argtypes = [C.POINTER(_CProblem), vp, vp, f32p, f32p, f32p, vp, C.c_size_t, vp]
    lib.chunkkv_compress_stack_lse.restype = C.c_int
    lib.chunkkv_compress_stack_lse.argtypes = [C.POINTER(_CProblem), C.c_int32, C.c_int32, C.POINTER(vp),
                                               C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp),
                                               C.POINTER(vp), i32p, i32p, i32p, vp, C.c_size_t, vp]
    lib.chunkkv_compress_layer.restype = C.c_int
    lib.chunkkv_compress_layer.argtypes = [C.POINTER(_CProblem), C.c_int32, C.c_int32, vp, f32p, vp, vp, vp, vp,
                                           i32p, i32p, i32p, vp, C.c_size_t, vp]
    lib.chunkkv_workspace_bytes_hybrid.restype = C.c_size_t
    lib.chunkkv_workspace_bytes_hybrid.argtypes = [C.POINTER(_CProblem), C.c_int32, C.c_int32, i32p]
    lib.chunkkv_compress_stack_hybrid.restype = C.c_int
    lib.chunkkv_compress_stack_hybrid.argtypes = [C.POINTER(_CProblem), C.c_int32, C.c_int32, i32p, C.POINTER(vp),
                                                  C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp),
                                                  C.POINTER(vp), i32p, i32p, i32p, vp, C.c_size_t, vp]
    lib.chunkkv_jaccard.restype = C.c_int
    lib.chunkkv_jaccard.argtypes = [C.POINTER(_CProblem), C.c_int32, i32p, i32p, i32p, f32p, vp]
    lib.chunkkv_decode_workspace_bytes.restype = C.c_size_t
    lib.chunkkv_decode_workspace_bytes.argtypes = [C.POINTER(_CProblem), C.c_int32]
    lib.chunkkv_decode_attention.restype = C.c_int
    lib.chunkkv_decode_attention.argtypes = [C.POINTER(_CProblem), C.c_int32, i32p, vp, vp, vp, f32p, f32p, vp,
                                             C.c_size_t, vp]
    lib.chunkkv_quality_workspace_bytes.restype = C.c_size_t
    lib.chunkkv_quality_workspace_bytes.argtypes = [C.POINTER(_CProblem)]
    lib.chunkkv_quality_metrics.restype = C.c_int
    lib.chunkkv_quality_metrics.argtypes = [C.POINTER(_CProblem), i32p, vp, vp, vp, vp, vp, f32p, f32p, vp, C.c_size_t, vp]
    lib.chunkkv_paged_compact.restype = C.c_int
    lib.chunkkv_paged_compact.argtypes = [C.POINTER(_CProblem), C.POINTER(_CPages), C.c_int32, C.c_int32, vp, vp, i32p, i32p, i32p, vp, i32p, vp, vp,
                                          i32p, i32p, f32p, vp]
    lib.chunkkv_paged_append.restype = C.c_int
    lib.chunkkv_paged_append.argtypes = [C.POINTER(_CPages), i32p, vp, C.c_int64, vp, C.c_int64, vp, C.c_int64, i32p, vp, vp, C.c_float, f32p, C.c_int32,
                                         C.c_int32, vp, i32p, vp, vp, i32p, i32p, i32p, f32p, vp]
    lib.chunkkv_paged_decode_workspace_bytes.restype = C.c_size_t
    lib.chunkkv_paged_decode_workspace_bytes.argtypes = [C.POINTER(_CPages), C.c_int32]
    lib.chunkkv_paged_decode_attention.restype = C.c_int
    lib.chunkkv_paged_decode_attention.argtypes = [C.POINTER(_CPages), i32p, i32p, vp, vp, vp, f32p, f32p, f32p, vp, C.c_size_t, vp]
    lib.chunkkv_paged_evict_workspace_bytes.restype = C.c_size_t
    lib.chunkkv_paged_evict_workspace_bytes.argtypes = [C.POINTER(_CPages), C.c_int32, i32p]
    lib.chunkkv_paged_evict.restype = C.c_int
    lib.chunkkv_paged_evict.argtypes = [C.POINTER(_CPages), C.c_int32, i32p, C.c_int32, i32p, vp, vp, i32p, i32p, f32p, vp, C.c_size_t, vp]
    lib.chunkkv_decode_attention_static.restype = C.c_int
    lib.chunkkv_decode_attention_static.argtypes = [C.POINTER(_CProblem), C.c_int32, i32p, vp, vp, vp, f32p, f32p, vp]
    _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _bytes(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.nbytes


def _stream(stream, dev: Optional[int] = None):
    if stream is None:
        # the handle itself: building a torch.cuda.Stream object around it takes 2.7 us
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if dev is None else dev)
    return stream.cuda_stream


def _check(rc: int, where: str):
    if rc != 0:
        raise ChunkKVError(rc, where, load_library().chunkkv_status_string(rc).decode())


def chunkkv_status_string(status: int) -> str:
    return load_library().chunkkv_status_string(int(status)).decode()


def chunkkv_workspace_bytes(prob: Problem, n_layers: int = 1, reuse: int = 1) -> int:
    return int(load_library().chunkkv_workspace_bytes(prob._c(), n_layers, reuse))


def chunkkv_score(prob: Problem, q_obs, k, chunk_scores, token_importance, workspace, stream=None) -> None:
    cp = prob._c()
    _check(load_library().chunkkv_score(cp, _ptr(q_obs), _ptr(k), _ptr(chunk_scores),
                                        _ptr(token_importance), _ptr(workspace),
                                        _bytes(workspace),
                                        _stream(stream)), "chunkkv_score")


def chunkkv_chunk_topk(prob: Problem, chunk_scores, sel_chunk, sel_len, sel_count, workspace=None, stream=None) -> None:
    cp = prob._c()
    _check(load_library().chunkkv_chunk_topk(cp, _ptr(chunk_scores), _ptr(sel_chunk), _ptr(sel_len),
                                             _ptr(sel_count), _ptr(workspace),
                                             _bytes(workspace),
                                             _stream(stream)), "chunkkv_chunk_topk")


def chunkkv_compact(prob: Problem, k, v, sel_chunk, sel_len, sel_count, k_out, v_out, stream=None) -> None:
    cp = prob._c()
    _check(load_library().chunkkv_compact(cp, _ptr(k), _ptr(v), _ptr(sel_chunk), _ptr(sel_len),
                                          _ptr(sel_count), _ptr(k_out), _ptr(v_out), _stream(stream)),
           "chunkkv_compact")


def chunkkv_compress_stack(prob: Problem, reuse: int, q_obs: Sequence, k: Sequence, v: Sequence, k_out: Sequence,
                           v_out: Sequence, sel_chunk, sel_len, sel_count, workspace, stream=None) -> None:
    n = len(k)
    cp = prob._c()

    def table(ts):
        return (C.c_void_p * n)(*[None if t is None else t.data_ptr() for t in ts])

    _check(load_library().chunkkv_compress_stack(
        cp, n, reuse, table(q_obs), table(k), table(v), table(k_out), table(v_out), _ptr(sel_chunk),
        _ptr(sel_len), _ptr(sel_count), _ptr(workspace),
        _bytes(workspace), _stream(stream)),
        "chunkkv_compress_stack")


def chunkkv_score_lse(prob: Problem, q_obs, k, lse, chunk_scores, token_importance, workspace, stream=None) -> None:
    cp = prob._c()
    _check(load_library().chunkkv_score_lse(cp, _ptr(q_obs), _ptr(k), _ptr(lse), _ptr(chunk_scores),
                                            _ptr(token_importance), _ptr(workspace),
                                            _bytes(workspace),
                                            _stream(stream)), "chunkkv_score_lse")


def chunkkv_compress_stack_lse(prob: Problem, reuse: int, q_obs: Sequence, k: Sequence, v: Sequence, lse: Sequence,
                               k_out: Sequence, v_out: Sequence, sel_chunk, sel_len, sel_count, workspace,
                               stream=None) -> None:
    n = len(k)
    cp = prob._c()

    def table(ts):
        return (C.c_void_p * n)(*[None if t is None else t.data_ptr() for t in ts])

    _check(load_library().chunkkv_compress_stack_lse(
        cp, n, reuse, table(q_obs), table(k), table(v), table(lse), table(k_out), table(v_out),
        _ptr(sel_chunk), _ptr(sel_len), _ptr(sel_count), _ptr(workspace),
        _bytes(workspace), _stream(stream)),
        "chunkkv_compress_stack_lse")


def chunkkv_compress_layer(prob: Problem, layer: int, reuse: int, q_obs, lse, k, v, k_out, v_out, sel_chunk, sel_len,
                           sel_count, workspace, stream=None) -> None:
    cp = prob._c()
    _check(load_library().chunkkv_compress_layer(
        cp, layer, reuse, _ptr(q_obs), _ptr(lse), _ptr(k), _ptr(v), _ptr(k_out), _ptr(v_out),
        _ptr(sel_chunk), _ptr(sel_len), _ptr(sel_count), _ptr(workspace),
        _bytes(workspace), _stream(stream)),
        "chunkkv_compress_layer")


def _chunk_table(chunk_per_group):
    return None if chunk_per_group is None else (C.c_int32 * len(chunk_per_group))(*[int(c) for c in chunk_per_group])


def chunkkv_workspace_bytes_hybrid(prob: Problem, n_layers: int, reuse: int, chunk_per_group) -> int:
    return int(load_library().chunkkv_workspace_bytes_hybrid(prob._c(), n_layers, reuse,
                                                             _chunk_table(chunk_per_group)))


def chunkkv_compress_stack_hybrid(prob: Problem, reuse: int, chunk_per_group, q_obs: Sequence, k: Sequence,
                                  v: Sequence, lse, k_out: Sequence, v_out: Sequence, sel_chunk, sel_len, sel_count,
                                  workspace, stream=None) -> None:
    n = len(k)
    cp = prob._c()

    def table(ts):
        return None if ts is None else (C.c_void_p * n)(*[None if t is None else t.data_ptr() for t in ts])

    _check(load_library().chunkkv_compress_stack_hybrid(
        cp, n, reuse, _chunk_table(chunk_per_group), table(q_obs), table(k), table(v), table(lse),
        table(k_out), table(v_out), _ptr(sel_chunk), _ptr(sel_len), _ptr(sel_count), _ptr(workspace),
        _bytes(workspace), _stream(stream)),
        "chunkkv_compress_stack_hybrid")


def chunkkv_jaccard(prob: Problem, n_groups: int, sel_chunk, sel_len, sel_count, jaccard, stream=None) -> None:
    cp = prob._c()
    _check(load_library().chunkkv_jaccard(cp, n_groups, _ptr(sel_chunk), _ptr(sel_len), _ptr(sel_count),
                                          _ptr(jaccard), _stream(stream)), "chunkkv_jaccard")


def chunkkv_quality_workspace_bytes(prob: Problem) -> int:
    return int(load_library().chunkkv_quality_workspace_bytes(prob._c()))


def chunkkv_quality_metrics(prob: Problem, kv_len, q, k, v, k_out, v_out, l1_loss, attn_cos, workspace, stream=None) -> None:
    cp = prob._c()
    _check(load_library().chunkkv_quality_metrics(
        cp, _ptr(kv_len), _ptr(q), _ptr(k), _ptr(v), _ptr(k_out), _ptr(v_out), _ptr(l1_loss), _ptr(attn_cos),
        _ptr(workspace), _bytes(workspace), _stream(stream)),
        "chunkkv_quality_metrics")


def chunkkv_decode_workspace_bytes(prob: Problem, compacted: bool = True) -> int:
    return int(load_library().chunkkv_decode_workspace_bytes(prob._c(), 1 if compacted else 0))


def chunkkv_decode_attention(prob: Problem, compacted: bool, kv_len, q, k, v, out, lse, workspace, stream=None) -> None:
    cp = prob._c()
    _check(load_library().chunkkv_decode_attention(
        cp, 1 if compacted else 0, _ptr(kv_len), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
        _ptr(workspace), _bytes(workspace), _stream(stream)),
        "chunkkv_decode_attention")


def chunkkv_decode_attention_static(prob: Problem, compacted: bool, kv_len, q, k, v, out, lse, stream=None) -> None:
    cp = prob._c()
    _check(load_library().chunkkv_decode_attention_static(
        cp, 1 if compacted else 0, _ptr(kv_len), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
        _stream(stream)), "chunkkv_decode_attention_static")


# ---- caches in pages ----
# A wrong size here is a read or a write out of bounds on the device, so sizes, types and devices are compared with the
# handle's before a call.  A decoding step is 5 to 10 us on the device, so the comparisons are written to cost 0.2 us a tensor
# and 0.1 us a pool of a list.
_KINDS = {F32: torch.float32, BF16: torch.bfloat16, F16: torch.float16}
_I32, _F32 = torch.int32, torch.float32
# torch.cuda.current_device() without its look at whether the runtime has been started (0.5 us): a call's tensors have done that
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_get_device, _data_ptr, _is_contiguous = torch.Tensor.get_device, torch.Tensor.data_ptr, torch.Tensor.is_contiguous
_dtype, _nbytes = torch.Tensor.dtype.__get__, torch.Tensor.nbytes.__get__


def _refuse(where: str, dev: int, name: str, t, kind, elements: int):
    if t.dtype is not kind:
        raise ValueError(f"{where}: {name} is {t.dtype}, not {kind}")
    if t.get_device() != dev:
        raise ValueError(f"{where}: {name} is on device {t.get_device()}, the call runs on {dev}")
    raise ValueError(f"{where}: {name} has {t.numel()} elements{'' if t.is_contiguous() else ', not contiguous'}; {elements} are needed")


def _arrays(where: str, dev: int, *arrays):
    """Checks (name, tensor or None, type, elements) each; -> their addresses."""
    out = []
    for name, t, kind, elements in arrays:
        if t is None:
            out.append(None)
            continue
        if t.dtype is not kind or t.get_device() != dev or t.numel() < elements or not t.is_contiguous():
            _refuse(where, dev, name, t, kind, elements)
        out.append(t.data_ptr())
    return out


def _pool(where: str, dev: int, name: str, t: Optional[torch.Tensor], kind, elements: int) -> int:
    """Address of a pool, 0 without one: what has to be there is the library's to say."""
    if t is None:
        return 0
    if t.dtype is not kind or t.get_device() != dev or t.numel() < elements or not t.is_contiguous():
        # a view of something larger: what counts is the memory behind its first element
        room = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
        if t.dtype is not kind or t.get_device() != dev or room < elements:
            _refuse(where, dev, name, t, kind, elements)
    return t.data_ptr()


def _alike(dev: int, ts: Sequence, kind, elements: int) -> bool:
    """Are all of the type and on the device, contiguous and large enough; for a long list, at 0.03 us a tensor and property."""
    n = len(ts)
    try:
        return ([*map(_dtype, ts)].count(kind) == n and [*map(_get_device, ts)].count(dev) == n and min(map(_nbytes, ts)) >= elements * ts[0].element_size()
                and all(map(_is_contiguous, ts)))
    except TypeError:   # one is None
        return False


def _pools(where: str, dev: int, name: str, ts: Sequence, kind, elements: int):
    """Addresses of the pools of several layers, as an array whose own address the library reads them from."""
    if len(ts) <= 4 or not _alike(dev, ts, kind, elements):
        return array("Q", [_pool(where, dev, name, t, kind, elements) for t in ts])
    return array("Q", [*map(_data_ptr, ts)])


def _pool_pairs(where: str, dev: int, names: Sequence[str], a: Sequence, b: Sequence, kind, elements: int):
    """The same for two lists of as many pools, looked through as one; -> the array and where either's addresses begin."""
    ts = [*a, *b]
    if len(ts) <= 4 or not _alike(dev, ts, kind, elements):
        at = array("Q", [_pool(where, dev, name, t, kind, elements) for name, xs in zip(names, (a, b)) for t in xs])
    else:
        at = array("Q", [*map(_data_ptr, ts)])
    first = at.buffer_info()[0]
    return at, first, first + 8 * len(a)


def _scratch(where: str, dev: int, t: Optional[torch.Tensor]):
    """Address and bytes of a workspace of any type."""
    if t is None:
        return None, 0
    if t.get_device() != dev or not t.is_contiguous():
        _refuse(where, dev, "workspace", t, t.dtype, 0)
    return t.data_ptr(), t.nbytes


def _at(table) -> Optional[int]:
    return None if table is None else table.buffer_info()[0]


def _new_rows(where: str, dev: int, name: str, t: Optional[torch.Tensor], kind, tokens: int, heads: int, dim: int):
    """Address and token stride of [tokens][heads][dim] rows."""
    if t is None:
        return None, 0
    if t.dtype is not kind or t.get_device() != dev:
        _refuse(where, dev, name, t, kind, 0)
    strides = t.stride()
    if t.shape != (tokens, heads, dim) or (tokens and (strides[2] != 1 or (heads > 1 and strides[1] != dim))):
        raise ValueError(f"{where}: {name} is {tuple(t.shape)} with strides {strides}, not [{tokens}][{heads}][{dim}] with contiguous heads")
    return t.data_ptr(), strides[0] if tokens > 1 else heads * dim   # that of a single row can be anything


_last_ints = ((), None)   # the host array of the last call's numbers, found again by the numbers


def _ints(xs: Sequence[int]):
    global _last_ints
    key = tuple(xs)
    last = _last_ints
    if last[0] != key:
        key = tuple(map(int, key))
        host = (C.c_int32 * len(key))(*key)
        _fits("host array", host, key)
        last = _last_ints = (key, host)
    return last


def chunkkv_paged_compact(prob: Problem, pages: Pages, reuse: int, k: Sequence, v: Sequence, sel_chunk, sel_len, sel_count, token_importance,
                          page_table, k_pages: Sequence, v_pages: Sequence, kv_len, token_pos, token_weight, stream=None) -> None:
    where, n, dev = "chunkkv_paged_compact", len(k), _device()
    reuse = min(reuse, n)   # of all layers, at most
    heads, groups, cp, full = pages.batch * pages.n_kv_heads, -(-n // max(1, reuse)), pages._c(), prob._c()
    _, seen, _, reach = prob._kept   # of the struct just returned: sizes are the library's
    if not len(v) == len(k_pages) == len(v_pages) == n or (token_importance is not None and len(token_importance) != groups):
        raise ValueError(f"{where}: lists of {n}, {len(v)}, {len(k_pages)} and {len(v_pages)} layers")
    sel, slots, kind, room = groups * heads * seen.sel_cap, n * heads * pages.slot_pitch, _KINDS.get(pages.dtype), pages._pool_elements()
    chunks, lens, count, table, length, pos, weight = _arrays(
        where, dev, ("sel_chunk", sel_chunk, _I32, sel), ("sel_len", sel_len, _I32, sel), ("sel_count", sel_count, _I32, groups * heads),
        ("page_table", page_table, _I32, pages.batch * pages.table_pitch), ("kv_len", kv_len, _I32, n * heads), ("token_pos", token_pos, _I32, slots),
        ("token_weight", token_weight, _F32, slots))
    given = None if token_importance is None else _pools(where, dev, "token_importance", token_importance, _F32, heads * seen.score_cap * seen.chunk)
    caches, ks, vs = _pool_pairs(where, dev, ("k", "v"), k, v, kind, reach)   # caches, pools: hold the addresses until the call returns
    pools, kp, vp = _pool_pairs(where, dev, ("k_pages", "v_pages"), k_pages, v_pages, kind, room)
    _check(load_library().chunkkv_paged_compact(full, cp, n, reuse, ks, vs, chunks, lens, count, _at(given), table, kp, vp, length, pos, weight,
                                                _stream(stream, dev)), where)


def chunkkv_paged_append(pages: Pages, n_new: Sequence[int], q, k, v, positions, q_norm, k_norm, eps: float, inv_freq, interleaved: bool, q_out,
                         page_table, k_pages, v_pages, kv_len, kv_len_out, token_pos, token_weight, stream=None) -> None:
    """q, k, v: [tokens][heads][head_dim], views of a fused projection among them, None without tokens; rotary_dim is twice inv_freq's length."""
    where, dev, kind = "chunkkv_paged_append", _device(), _KINDS.get(pages.dtype)
    batch, hkv, d, cp = pages.batch, pages.n_kv_heads, pages.head_dim, pages._c()
    numbers, new = _ints(n_new)
    if len(numbers) != batch:
        raise ValueError(f"{where}: n_new has {len(numbers)} entries for {batch} sequences")
    tokens, heads = max(0, sum(numbers)), batch * hkv
    qp, q_tok = _new_rows(where, dev, "q", q, kind, tokens, pages.n_q_heads, d)
    kp, k_tok = _new_rows(where, dev, "k", k, kind, tokens, hkv, d)
    vp, v_tok = _new_rows(where, dev, "v", v, kind, tokens, hkv, d)
    at, qn, kn, out, table, length, after, freq, pos, weight = _arrays(
        where, dev, ("positions", positions, _I32, tokens), ("q_norm", q_norm, kind, d), ("k_norm", k_norm, kind, d),
        ("q_out", q_out, kind, tokens * pages.n_q_heads * d), ("page_table", page_table, _I32, batch * pages.table_pitch), ("kv_len", kv_len, _I32, heads),
        ("kv_len_out", kv_len_out, _I32, heads), ("inv_freq", inv_freq, _F32, 0), ("token_pos", token_pos, _I32, heads * pages.slot_pitch),
        ("token_weight", token_weight, _F32, heads * pages.slot_pitch))
    room = pages._pool_elements()
    _check(load_library().chunkkv_paged_append(
        cp, new, qp, q_tok, kp, k_tok, vp, v_tok, at, qn, kn, eps, freq,
        0 if inv_freq is None else 2 * inv_freq.numel(), 1 if interleaved else 0, out, table, _pool(where, dev, "k_pages", k_pages, kind, room),
        _pool(where, dev, "v_pages", v_pages, kind, room), length, after, pos, weight, _stream(stream, dev)), where)


def chunkkv_paged_decode_workspace_bytes(pages: Pages, with_weights: bool = False) -> int:
    return int(load_library().chunkkv_paged_decode_workspace_bytes(pages._c(), 1 if with_weights else 0))


def chunkkv_paged_decode_attention(pages: Pages, page_table, kv_len, q, k_pages, v_pages, out, lse, token_weight, workspace, stream=None) -> None:
    where, dev, kind = "chunkkv_paged_decode_attention", _device(), _KINDS.get(pages.dtype)
    cp, batch = pages._c(), pages.batch
    rows, heads, room = batch * pages.n_q_heads, batch * pages.n_kv_heads, pages._pool_elements()
    table, length, qp, op, lp, weight = _arrays(
        where, dev, ("page_table", page_table, _I32, batch * pages.table_pitch), ("kv_len", kv_len, _I32, heads), ("q", q, kind, rows * pages.head_dim),
        ("out", out, _F32, rows * pages.head_dim), ("lse", lse, _F32, rows), ("token_weight", token_weight, _F32, heads * pages.slot_pitch))
    _check(load_library().chunkkv_paged_decode_attention(
        cp, table, length, qp, _pool(where, dev, "k_pages", k_pages, kind, room), _pool(where, dev, "v_pages", v_pages, kind, room), op, lp, weight,
        *_scratch(where, dev, workspace), _stream(stream, dev)), where)


def _budgets(where: str, pages: Pages, budget: Sequence[int]):
    numbers, host = _ints(budget)
    if len(numbers) != pages.batch:
        raise ValueError(f"{where}: budget has {len(numbers)} entries for {pages.batch} sequences")
    return host


def chunkkv_paged_evict_workspace_bytes(pages: Pages, n_layers: int, budget: Sequence[int]) -> int:
    return int(load_library().chunkkv_paged_evict_workspace_bytes(pages._c(), n_layers, _budgets("chunkkv_paged_evict_workspace_bytes", pages, budget)))


def chunkkv_paged_evict(pages: Pages, budget: Sequence[int], recent: int, page_table, k_pages: Sequence, v_pages: Sequence, kv_len, token_pos,
                        token_weight, workspace, stream=None) -> None:
    where, n, dev, kind = "chunkkv_paged_evict", len(k_pages), _device(), _KINDS.get(pages.dtype)
    if len(v_pages) != n:
        raise ValueError(f"{where}: lists of {n} and {len(v_pages)} layers")
    cp, heads = pages._c(), n * pages.batch * pages.n_kv_heads
    room, slots = pages._pool_elements(), heads * pages.slot_pitch
    table, length, pos, weight = _arrays(where, dev, ("page_table", page_table, _I32, pages.batch * pages.table_pitch), ("kv_len", kv_len, _I32, heads),
                                         ("token_pos", token_pos, _I32, slots), ("token_weight", token_weight, _F32, slots))
    pools, kp, vp = _pool_pairs(where, dev, ("k_pages", "v_pages"), k_pages, v_pages, kind, room)   # pools: holds the addresses until the call returns
    _check(load_library().chunkkv_paged_evict(cp, n, _budgets(where, pages, budget), recent, table, kp, vp, length, pos, weight,
                                              *_scratch(where, dev, workspace), _stream(stream, dev)), where)


def chunkkv_timing_begin(max_records: int = 4096) -> None:
    lib = load_library()
    lib.chunkkv_timing_begin.restype = C.c_int
    lib.chunkkv_timing_begin.argtypes = [C.c_int32]
    _check(lib.chunkkv_timing_begin(max_records), "chunkkv_timing_begin")


def chunkkv_timing_end() -> dict:
    """-> {kind: (total milliseconds, launches)} for the kernels launched since chunkkv_timing_begin."""
    lib = load_library()
    n = len(TIMING_KINDS)
    ms, cnt = (C.c_double * n)(), (C.c_int64 * n)()
    lib.chunkkv_timing_end.restype = C.c_int
    lib.chunkkv_timing_end.argtypes = [C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    _check(lib.chunkkv_timing_end(ms, cnt), "chunkkv_timing_end")
    return {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(TIMING_KINDS)}
