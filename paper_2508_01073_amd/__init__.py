"""MI355X-native RDF2vec random-walk corpus extraction.

Python binding of ``librdf2v.so`` (HIP kernels for gfx950 behind the C ABI in
``include/rdf2v.h``). The functions carry the C names and only marshal
arguments: PyTorch supplies device memory and the stream, every step of the
computation runs in the library's kernels. There is no CPU fallback: every call
raises if the library has not been built (``python -m paper_2508_01073_amd.build``),
and calls fail if no GPU is present.

Walk extraction follows gpuRDF2vec (Boeckling & Paulheim, arXiv 2508.01073):
uniform random walks (Sec. 2) emitted as entity/predicate token rows padded
with -1 (Sec. 3.1), all walks of all start entities launched together
(Sec. 4.1), with walk depth, walks per entity and seed as in Sec. 3.3.
"""

from __future__ import annotations

import ctypes
import os
import warnings
from dataclasses import dataclass
from typing import NamedTuple

import torch
from torch.autograd import forward_ad

__all__ = [
    "Csr", "Rdf2vError", "RDF2V_MAX_DEPTH", "RDF2V_STATUS_ID_OUT_OF_RANGE", "RDF2V_STATUS_BAD_CSR",
    "RDF2V_TOKENS_TRIPLES", "RDF2V_TOKENS_ENTITIES", "RDF2V_TOKENS_PROPERTIES",
    "rdf2v_build_csr_workspace_size", "rdf2v_build_csr", "rdf2v_build_walk_edges",
    "rdf2v_walk_edges_recommended",
    "rdf2v_nonsink_starts_workspace_size",
    "rdf2v_nonsink_starts", "rdf2v_random_walks", "rdf2v_random_walks_tokens",
    "rdf2v_unique_walks_workspace_size", "rdf2v_unique_walks", "rdf2v_bfs_walks_workspace_size",
    "rdf2v_bfs_walks", "rdf2v_skipgram_pairs_workspace_size",
    "rdf2v_skipgram_pairs", "rdf2v_skipgram_pairs_noalloc", "RDF2V_NOALLOC_MAX_WALKS",
    "RDF2V_NOALLOC_SCRATCH_BYTES", "rdf2v_cbow_examples_workspace_size", "rdf2v_cbow_examples",
    "rdf2v_build_vocabulary_workspace_size", "rdf2v_build_vocabulary",
    "RDF2V_STATUS_BAD_VALUE", "RDF2V_MAX_HEAD_SIZE", "RDF2V_MAX_BEAMS", "RDF2V_MAX_TEACHER_TOP",
    "rdf2v_decay_attention_workspace_size", "rdf2v_decay_attention",
    "rdf2v_decay_attention_backward_workspace_size", "rdf2v_decay_attention_backward",
    "rdf2v_decay_attention_step", "rdf2v_beam_select_workspace_size", "rdf2v_beam_select", "rdf2v_beam_reorder",
    "rdf2v_distill_workspace_size", "rdf2v_distill_loss", "rdf2v_distill_loss_backward",
    "RDF2V_MAX_CONV_WIDTH", "RDF2V_MAX_SCAN_STATES", "RDF2V_MAX_NORM_CHANNELS",
    "rdf2v_causal_conv", "rdf2v_causal_conv_backward_workspace_size", "rdf2v_causal_conv_backward",
    "rdf2v_causal_conv_step", "rdf2v_selective_scan_workspace_size", "rdf2v_selective_scan",
    "rdf2v_selective_scan_backward_workspace_size", "rdf2v_selective_scan_backward", "ScanGradients",
    "rdf2v_selective_scan_step", "rdf2v_residual_norm", "rdf2v_residual_norm_backward_workspace_size",
    "rdf2v_residual_norm_backward", "NormGradients",
    "rdf2v_status_string", "check_device_status",
    "library_path",
]

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librdf2v.so")

RDF2V_OK = 0
RDF2V_ERR_INVALID_ARGUMENT = 1
RDF2V_ERR_ID_OUT_OF_RANGE = 2
RDF2V_ERR_TOO_LARGE = 3
RDF2V_ERR_WORKSPACE = 4
RDF2V_ERR_HIP = 5
RDF2V_STATUS_ID_OUT_OF_RANGE = 0x1
RDF2V_STATUS_BAD_CSR = 0x2
RDF2V_STATUS_BAD_LENGTH = 0x4
RDF2V_STATUS_CAPACITY = 0x8
RDF2V_STATUS_BAD_VALUE = 0x10
RDF2V_MAX_DEPTH = 64
RDF2V_TOKENS_TRIPLES = 0
RDF2V_TOKENS_ENTITIES = 1
RDF2V_TOKENS_PROPERTIES = 2
RDF2V_NOALLOC_MAX_WALKS = 1 << 22
RDF2V_NOALLOC_SCRATCH_BYTES = (32 << 20) + (64 << 10)
RDF2V_F32 = 0
RDF2V_BF16 = 1
RDF2V_MAX_HEAD_SIZE = 128
RDF2V_MAX_BEAMS = 64
RDF2V_MAX_TEACHER_TOP = 512
RDF2V_MAX_CONV_WIDTH = 8
RDF2V_MAX_SCAN_STATES = 64
RDF2V_MAX_NORM_CHANNELS = 16384

_lib = None


def library_path() -> str:
    return _LIB_PATH


class _CsrStruct(ctypes.Structure):
    _fields_ = [("num_entities", ctypes.c_int32), ("num_predicates", ctypes.c_int32),
                ("num_edges", ctypes.c_int64), ("row_ptr", ctypes.c_void_p),
                ("edges", ctypes.c_void_p), ("walk_edges", ctypes.c_void_p)]


class _AttentionStruct(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("length", ctypes.c_int64), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("dk", ctypes.c_int32), ("dv", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("log_decay", ctypes.c_void_p),
                ("len", ctypes.c_void_p)]


class _HeadsViewStruct(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class _TokensViewStruct(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64)]


class _ConvStruct(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("length", ctypes.c_int64), ("channels", ctypes.c_int32),
                ("width", ctypes.c_int32), ("dtype", ctypes.c_int32), ("silu", ctypes.c_int32),
                ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("len", ctypes.c_void_p)]


class _ScanStruct(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("length", ctypes.c_int64), ("channels", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("states", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("a", ctypes.c_void_p), ("dt_bias", ctypes.c_void_p), ("skip", ctypes.c_void_p),
                ("len", ctypes.c_void_p)]


class _ScanGradientsStruct(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("dx", "ddt", "db", "dc", "dgate", "da", "ddt_bias", "dskip",
                                                     "dstate")]


class _NormStruct(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("length", ctypes.c_int64), ("channels", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("residual_dtype", ctypes.c_int32), ("center", ctypes.c_int32),
                ("eps", ctypes.c_float), ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("scale", ctypes.c_void_p), ("drop", ctypes.c_double), ("seed", ctypes.c_uint64),
                ("seed_offset", ctypes.c_void_p), ("row_begin", ctypes.c_int64), ("len", ctypes.c_void_p)]


def _native():
    """The loaded librdf2v.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is not built; run `python -m paper_2508_01073_amd.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, u64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t
    csr_p = ctypes.POINTER(_CsrStruct)
    lib.rdf2v_build_csr_workspace_size.argtypes = [i64, i32]
    lib.rdf2v_build_csr_workspace_size.restype = sz
    lib.rdf2v_build_csr.argtypes = [vp, vp, vp, i64, i32, i32, vp, vp, vp, sz, vp, vp]
    lib.rdf2v_build_csr.restype = ctypes.c_int
    lib.rdf2v_build_walk_edges.argtypes = [csr_p, vp, vp, vp]
    lib.rdf2v_build_walk_edges.restype = ctypes.c_int
    lib.rdf2v_walk_edges_recommended.argtypes = [i32, i64]
    lib.rdf2v_walk_edges_recommended.restype = i32
    lib.rdf2v_nonsink_starts_workspace_size.argtypes = [i32]
    lib.rdf2v_nonsink_starts_workspace_size.restype = sz
    lib.rdf2v_nonsink_starts.argtypes = [csr_p, vp, vp, vp, sz, vp]
    lib.rdf2v_nonsink_starts.restype = ctypes.c_int
    lib.rdf2v_random_walks.argtypes = [csr_p, vp, i64, i32, i32, u64, i64, i64, vp, vp, vp, vp]
    lib.rdf2v_random_walks.restype = ctypes.c_int
    lib.rdf2v_random_walks_tokens.argtypes = [csr_p, vp, i64, i32, i32, u64, i64, i64, i32, vp, vp, vp, vp]
    lib.rdf2v_random_walks_tokens.restype = ctypes.c_int
    lib.rdf2v_unique_walks_workspace_size.argtypes = [i64]
    lib.rdf2v_unique_walks_workspace_size.restype = sz
    lib.rdf2v_unique_walks.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp, vp, sz, vp, vp]
    lib.rdf2v_unique_walks.restype = ctypes.c_int
    lib.rdf2v_bfs_walks_workspace_size.argtypes = [i32, i64]
    lib.rdf2v_bfs_walks_workspace_size.restype = sz
    lib.rdf2v_bfs_walks.argtypes = [csr_p, vp, i64, i32, i32, vp, vp, vp, vp, sz, vp, vp]
    lib.rdf2v_bfs_walks.restype = ctypes.c_int
    lib.rdf2v_bfs_fill_unused.argtypes = [vp, i64, i32, i32, vp, vp, vp]
    lib.rdf2v_bfs_fill_unused.restype = ctypes.c_int
    lib.rdf2v_skipgram_pairs_workspace_size.argtypes = [i64]
    lib.rdf2v_skipgram_pairs_workspace_size.restype = sz
    lib.rdf2v_skipgram_pairs.argtypes = [vp, vp, i64, i32, i32, vp, i64, vp, vp, sz, vp, vp]
    lib.rdf2v_skipgram_pairs.restype = ctypes.c_int
    lib.rdf2v_skipgram_pairs_noalloc.argtypes = [vp, vp, i64, i32, i32, vp, i64, vp, vp, vp]
    lib.rdf2v_skipgram_pairs_noalloc.restype = ctypes.c_int
    lib.rdf2v_cbow_examples_workspace_size.argtypes = [i64]
    lib.rdf2v_cbow_examples_workspace_size.restype = sz
    lib.rdf2v_cbow_examples.argtypes = [vp, vp, i64, i32, i32, vp, vp, i64, vp, vp, sz, vp, vp]
    lib.rdf2v_cbow_examples.restype = ctypes.c_int
    lib.rdf2v_build_vocabulary_workspace_size.argtypes = [i64, i64, i64]
    lib.rdf2v_build_vocabulary_workspace_size.restype = sz
    lib.rdf2v_build_vocabulary.argtypes = [vp, vp, i64] * 3 + [i64, i64, i64, vp, vp, vp, vp, vp, sz, vp, vp]
    lib.rdf2v_build_vocabulary.restype = ctypes.c_int
    att_p, view_p, f32 = ctypes.POINTER(_AttentionStruct), ctypes.POINTER(_HeadsViewStruct), ctypes.c_float
    lib.rdf2v_decay_attention_workspace_size.argtypes = [att_p]
    lib.rdf2v_decay_attention_workspace_size.restype = sz
    lib.rdf2v_decay_attention.argtypes = [att_p, view_p, view_p, view_p, vp, vp, vp, vp, sz, vp, vp]
    lib.rdf2v_decay_attention.restype = ctypes.c_int
    lib.rdf2v_decay_attention_backward_workspace_size.argtypes = [att_p]
    lib.rdf2v_decay_attention_backward_workspace_size.restype = sz
    lib.rdf2v_decay_attention_backward.argtypes = [att_p] + [view_p] * 4 + [vp] * 7 + [sz, vp, vp]
    lib.rdf2v_decay_attention_backward.restype = ctypes.c_int
    lib.rdf2v_decay_attention_step.argtypes = [att_p, view_p, view_p, view_p, vp, i64, vp, vp, vp, vp, vp]
    lib.rdf2v_decay_attention_step.restype = ctypes.c_int
    lib.rdf2v_beam_select_workspace_size.argtypes = [i64, i32, i64, i32]
    lib.rdf2v_beam_select_workspace_size.restype = sz
    lib.rdf2v_beam_select.argtypes = [vp, i64, i32, vp, vp, i64, i32, i64, i32, vp, vp, vp, vp, sz, vp, vp]
    lib.rdf2v_beam_select.restype = ctypes.c_int
    lib.rdf2v_beam_reorder.argtypes = [vp, i64, i64, vp, i64, vp, vp, vp]
    lib.rdf2v_beam_reorder.restype = ctypes.c_int
    lib.rdf2v_distill_workspace_size.argtypes = [i64, i64, i32, i32]
    lib.rdf2v_distill_workspace_size.restype = sz
    lib.rdf2v_distill_loss.argtypes = [vp, i64, i32, vp, vp, i64, i64, i32, f32, vp, vp, vp, vp, i64, vp, sz, vp, vp]
    lib.rdf2v_distill_loss.restype = ctypes.c_int
    lib.rdf2v_distill_loss_backward.argtypes = [vp, i64, i32, vp, vp, i64, i64, i32, f32, vp, vp, vp, i64, vp, sz,
                                                vp, vp]
    lib.rdf2v_distill_loss_backward.restype = ctypes.c_int
    conv_p, tok_p = ctypes.POINTER(_ConvStruct), ctypes.POINTER(_TokensViewStruct)
    scan_p, norm_p = ctypes.POINTER(_ScanStruct), ctypes.POINTER(_NormStruct)
    for name, args in (("causal_conv", [conv_p, tok_p] + [vp] * 5),
                       ("causal_conv_backward", [conv_p, tok_p, tok_p] + [vp] * 7 + [sz, vp, vp]),
                       ("causal_conv_step", [conv_p, tok_p, vp, i64] + [vp] * 5),
                       ("selective_scan", [scan_p, tok_p, tok_p, view_p, view_p, tok_p] + [vp] * 4 + [sz, vp, vp]),
                       ("selective_scan_backward", [scan_p, tok_p, tok_p, view_p, view_p, tok_p, tok_p, vp, vp,
                                                    ctypes.POINTER(_ScanGradientsStruct), vp, sz, vp, vp]),
                       ("selective_scan_step", [scan_p, tok_p, tok_p, view_p, view_p, tok_p, vp, i64] + [vp] * 5),
                       ("residual_norm", [norm_p, tok_p, tok_p] + [vp] * 5),
                       ("residual_norm_backward", [norm_p, tok_p, tok_p, vp, tok_p, tok_p] + [vp] * 6 + [sz, vp, vp])):
        call = getattr(lib, "rdf2v_" + name)
        call.argtypes, call.restype = args, ctypes.c_int
    for name, arg in (("causal_conv_backward", conv_p), ("selective_scan", scan_p), ("selective_scan_backward", scan_p),
                      ("residual_norm_backward", norm_p)):
        call = getattr(lib, f"rdf2v_{name}_workspace_size")
        call.argtypes, call.restype = [arg], sz
    lib.rdf2v_status_string.argtypes = [ctypes.c_int]
    lib.rdf2v_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


class Rdf2vError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {rdf2v_status_string(status)} ({status})")
        self.status = status


def rdf2v_status_string(status: int) -> str:
    return _native().rdf2v_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != RDF2V_OK:
        raise Rdf2vError(status, where)


def _dev_i32(t: torch.Tensor, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != torch.int32:
        raise TypeError(f"{name} must be int32, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _out(t: torch.Tensor, name: str, dtype: torch.dtype, min_numel: int, dev: torch.device) -> torch.Tensor:
    """A caller-supplied output: on the call's device, of the given dtype, contiguous, and large
    enough (the library writes through the raw pointer, so a short buffer would be overrun)."""
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda" or t.device != dev:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor on {dev}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() < min_numel:
        raise ValueError(f"{name} holds {t.numel()} elements; this call needs {min_numel}")
    return t


def _status(t: torch.Tensor | None, dev: torch.device) -> torch.Tensor | None:
    """The optional device status word (one int32 the kernels OR error bits into)."""
    return None if t is None else _out(t, "status", torch.int32, 1, dev)


def _same_device(dev: torch.device, **tensors) -> None:
    for name, t in tensors.items():
        if t is not None and t.device != dev:
            raise TypeError(f"{name} must be on {dev}, got {t.device}")


def _ws_bytes(t: torch.Tensor | None) -> int:
    """Size in bytes of a caller workspace (any dtype; contiguous device memory)."""
    if t is None:
        return 0
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda" or not t.is_contiguous():
        raise TypeError("workspace must be a contiguous CUDA (HIP) tensor")
    return t.numel() * t.element_size()


def _ptr(t: torch.Tensor | None):
    return None if t is None or t.numel() == 0 else t.data_ptr()


class _on_stream:
    """Makes the caller's stream current for the whole call and yields its handle.

    Everything the binding does for a call then happens on that stream: tensors it allocates
    (outputs, workspaces) belong to it in torch's caching allocator, so a workspace freed when
    the call returns is reused only by work ordered after the call's kernels, and a count read
    back with ``.item()`` waits for those kernels. ``stream`` is None (the device's current
    stream), a ``torch.cuda.Stream`` or a raw hipStream_t handle (int). The current stream of the
    current device is left as it is: switching to it costs a small call a third of its time."""

    __slots__ = ("_handle", "_switch")

    def __init__(self, device: torch.device, stream):
        if stream is None and device.index == torch.cuda.current_device():
            # the handle alone: a stream object would cost a small call a tenth of its time
            self._switch = None
            self._handle = torch._C._cuda_getCurrentRawStream(device.index)
            return
        if stream is None:
            s = torch.cuda.current_stream(device)
        elif isinstance(stream, torch.cuda.Stream):
            s = stream
        else:
            s = torch.cuda.ExternalStream(int(stream), device=device)
        if s.device != device:
            raise TypeError(f"stream is on {s.device}, the call's tensors on {device}")
        self._switch = torch.cuda.stream(s)
        self._handle = s.cuda_stream

    def __enter__(self) -> int:
        if self._switch is not None:
            self._switch.__enter__()
        return self._handle

    def __exit__(self, *exc) -> None:
        if self._switch is not None:
            self._switch.__exit__(*exc)


@dataclass
class Csr:
    """Subject-indexed CSR in device memory (see ``rdf2v_csr`` in rdf2v.h).

    row_ptr: int32 [num_entities + 1]; edges: int32 [num_edges, 2] = (predicate, object);
    walk_edges (optional): int32 [num_edges, 4] = (predicate, object, row lo, row hi) of the
    object, from rdf2v_build_walk_edges."""
    row_ptr: torch.Tensor
    edges: torch.Tensor
    num_entities: int
    num_predicates: int
    walk_edges: torch.Tensor | None = None

    @property
    def num_edges(self) -> int:
        return int(self.edges.shape[0])

    def _c(self) -> _CsrStruct:
        we = self.walk_edges
        return _CsrStruct(self.num_entities, self.num_predicates, self.num_edges,
                          self.row_ptr.data_ptr(), self.edges.data_ptr() if self.edges.numel() else None,
                          we.data_ptr() if we is not None and we.numel() else None)


def rdf2v_build_csr_workspace_size(num_triples: int, num_entities: int) -> int:
    return int(_native().rdf2v_build_csr_workspace_size(num_triples, num_entities))


def rdf2v_build_csr(subj: torch.Tensor, pred: torch.Tensor, obj: torch.Tensor, num_entities: int,
                    num_predicates: int, *, workspace: torch.Tensor | None = None,
                    status: torch.Tensor | None = None, stream=None,
                    row_ptr: torch.Tensor | None = None, edges: torch.Tensor | None = None) -> Csr:
    """Triples (device int32 [T] each) -> Csr. Rows keep the input order of their triples."""
    _dev_i32(subj, "subj"); _dev_i32(pred, "pred"); _dev_i32(obj, "obj")
    t = subj.shape[0]
    if pred.shape[0] != t or obj.shape[0] != t:
        raise ValueError("subj, pred and obj differ in length")
    dev = subj.device
    with _on_stream(dev, stream) as h:
        _same_device(dev, pred=pred, obj=obj)
        if row_ptr is None:
            row_ptr = torch.empty(num_entities + 1, dtype=torch.int32, device=dev)
        if edges is None:
            edges = torch.empty((t, 2), dtype=torch.int32, device=dev)
        _out(row_ptr, "row_ptr", torch.int32, num_entities + 1, dev)
        _out(edges, "edges", torch.int32, 2 * t, dev)
        _status(status, dev)
        need = rdf2v_build_csr_workspace_size(t, num_entities)
        if workspace is None and need > 0:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        ws_bytes = _ws_bytes(workspace)
        st = _native().rdf2v_build_csr(_ptr(subj), _ptr(pred), _ptr(obj), t, num_entities, num_predicates,
                                  _ptr(row_ptr), _ptr(edges), _ptr(workspace), ws_bytes, _ptr(status),
                                  h)
        _check(st, "rdf2v_build_csr")
        return Csr(row_ptr, edges, num_entities, num_predicates)


def rdf2v_build_walk_edges(csr: Csr, *, out: torch.Tensor | None = None,
                           status: torch.Tensor | None = None, stream=None) -> Csr:
    """Returns the Csr with walk_edges [num_edges, 4] = (predicate, object, row lo, row hi)
    of the object, so the walks read one 16-byte record per hop."""
    dev = csr.row_ptr.device
    with _on_stream(dev, stream) as h:
        if out is None:
            out = torch.empty((csr.num_edges, 4), dtype=torch.int32, device=dev)
        _same_device(dev, edges=csr.edges)
        _out(out, "out", torch.int32, 4 * csr.num_edges, dev)
        _status(status, dev)
        c = csr._c()
        st = _native().rdf2v_build_walk_edges(ctypes.byref(c), _ptr(out), _ptr(status), h)
        _check(st, "rdf2v_build_walk_edges")
        return Csr(csr.row_ptr, csr.edges, csr.num_entities, csr.num_predicates, out)


def rdf2v_walk_edges_recommended(num_entities: int, num_edges: int) -> bool:
    """Whether rdf2v_build_walk_edges' records are expected to speed up the walks on a CSR of
    this size (pure host call; the walks are the same either way)."""
    return bool(_native().rdf2v_walk_edges_recommended(num_entities, num_edges))


def rdf2v_nonsink_starts_workspace_size(num_entities: int) -> int:
    return int(_native().rdf2v_nonsink_starts_workspace_size(num_entities))


def rdf2v_nonsink_starts(csr: Csr, *, workspace: torch.Tensor | None = None, stream=None,
                         starts: torch.Tensor | None = None, count: torch.Tensor | None = None,
                         sync: bool = True):
    """Entities with out-degree >= 1, ascending. With sync=True returns the int32 tensor of
    start ids (one device-to-host read of the count); else (starts, count_device_int64)."""
    dev = csr.row_ptr.device
    with _on_stream(dev, stream) as h:
        if starts is None:
            starts = torch.empty(max(csr.num_entities, 1), dtype=torch.int32, device=dev)
        if count is None:
            count = torch.empty(1, dtype=torch.int64, device=dev)
        if workspace is None:
            workspace = torch.empty(rdf2v_nonsink_starts_workspace_size(csr.num_entities),
                                    dtype=torch.uint8, device=dev)
        _out(starts, "starts", torch.int32, csr.num_entities, dev)
        _out(count, "count", torch.int64, 1, dev)
        c = csr._c()
        st = _native().rdf2v_nonsink_starts(ctypes.byref(c), _ptr(starts), _ptr(count), _ptr(workspace),
                                       _ws_bytes(workspace), h)
        _check(st, "rdf2v_nonsink_starts")
        if not sync:
            return starts, count
        return starts[: int(count.item())]


def rdf2v_random_walks(csr: Csr, start_nodes: torch.Tensor, walks_per_node: int, depth: int,
                       seed: int, walk_begin: int = 0, walk_count: int | None = None, *,
                       tokens: torch.Tensor | None = None, lens: torch.Tensor | None = None,
                       status: torch.Tensor | None = None, stream=None):
    """Walks [walk_begin, walk_begin + walk_count) -> (tokens int32 [walk_count, 2*depth+1],
    lens int32 [walk_count]). Walk w starts at start_nodes[w // walks_per_node]."""
    return _walks(csr, start_nodes, walks_per_node, depth, seed, walk_begin, walk_count,
                  RDF2V_TOKENS_TRIPLES, tokens, lens, status, stream, "rdf2v_random_walks")


def rdf2v_random_walks_tokens(csr: Csr, start_nodes: torch.Tensor, walks_per_node: int, depth: int,
                              seed: int, walk_begin: int = 0, walk_count: int | None = None,
                              token_kind: int = RDF2V_TOKENS_TRIPLES, *,
                              tokens: torch.Tensor | None = None, lens: torch.Tensor | None = None,
                              status: torch.Tensor | None = None, stream=None):
    """Like rdf2v_random_walks with a choice of tokens: RDF2V_TOKENS_TRIPLES (2*depth+1 per row),
    RDF2V_TOKENS_ENTITIES or RDF2V_TOKENS_PROPERTIES (depth+1 per row)."""
    return _walks(csr, start_nodes, walks_per_node, depth, seed, walk_begin, walk_count, token_kind,
                  tokens, lens, status, stream, "rdf2v_random_walks_tokens")


def _walks(csr, start_nodes, walks_per_node, depth, seed, walk_begin, walk_count, token_kind,
           tokens, lens, status, stream, where):
    _dev_i32(start_nodes, "start_nodes")
    dev = start_nodes.device
    with _on_stream(dev, stream) as h:
        num_walks = start_nodes.shape[0] * walks_per_node
        if walk_count is None:
            walk_count = num_walks - walk_begin
        width = 2 * depth + 1 if token_kind == RDF2V_TOKENS_TRIPLES else depth + 1
        if tokens is None:
            tokens = torch.empty((max(walk_count, 0), max(width, 1)), dtype=torch.int32, device=dev)
        if lens is None:
            lens = torch.empty(max(walk_count, 0), dtype=torch.int32, device=dev)
        rows = max(walk_count, 0)
        _out(tokens, "tokens", torch.int32, rows * width, dev)
        _out(lens, "lens", torch.int32, rows, dev)
        _status(status, dev)
        _same_device(dev, row_ptr=csr.row_ptr, edges=csr.edges, walk_edges=csr.walk_edges)
        c = csr._c()
        st = _native().rdf2v_random_walks_tokens(ctypes.byref(c), _ptr(start_nodes), start_nodes.shape[0],
                                                 walks_per_node, depth, ctypes.c_uint64(seed & (2**64 - 1)),
                                                 walk_begin, walk_count, token_kind, _ptr(tokens), _ptr(lens),
                                                 _ptr(status), h)
        _check(st, where)
        return tokens, lens


def rdf2v_unique_walks_workspace_size(num_walks: int) -> int:
    return int(_native().rdf2v_unique_walks_workspace_size(num_walks))


def rdf2v_unique_walks(tokens: torch.Tensor, lens: torch.Tensor, group_size: int, *,
                       tokens_out: torch.Tensor | None = None, lens_out: torch.Tensor | None = None,
                       count: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                       status: torch.Tensor | None = None, stream=None, sync: bool = True):
    """Duplicate-free walks: within each group of group_size consecutive rows keep the first
    occurrence of each distinct walk. With sync=True returns the kept (tokens, lens) (one
    device-to-host read of the count); else (tokens_out, lens_out, count_device_int64)."""
    _dev_i32(tokens, "tokens"); _dev_i32(lens, "lens")
    dev = tokens.device
    with _on_stream(dev, stream) as h:
        n = int(lens.shape[0])
        width = int(tokens.shape[1]) if tokens.dim() == 2 else 1
        if tokens_out is None:
            tokens_out = torch.empty((n, width), dtype=torch.int32, device=dev)
        if lens_out is None:
            lens_out = torch.empty(n, dtype=torch.int32, device=dev)
        if count is None:
            count = torch.empty(1, dtype=torch.int64, device=dev)
        if workspace is None:
            workspace = torch.empty(max(rdf2v_unique_walks_workspace_size(n), 1), dtype=torch.uint8, device=dev)
        _same_device(dev, lens=lens)
        _out(tokens_out, "tokens_out", torch.int32, n * width, dev)
        _out(lens_out, "lens_out", torch.int32, n, dev)
        _out(count, "count", torch.int64, 1, dev)
        _status(status, dev)
        st = _native().rdf2v_unique_walks(_ptr(tokens), _ptr(lens), n, group_size, width, _ptr(tokens_out),
                                          _ptr(lens_out), _ptr(count), _ptr(workspace), _ws_bytes(workspace),
                                          _ptr(status), h)
        _check(st, "rdf2v_unique_walks")
        if not sync:
            return tokens_out, lens_out, count
        k = int(count.item())
        return tokens_out[:k], lens_out[:k]


def rdf2v_bfs_walks_workspace_size(num_entities: int, num_roots: int) -> int:
    return int(_native().rdf2v_bfs_walks_workspace_size(num_entities, num_roots))


def rdf2v_bfs_walks(csr: Csr, roots: torch.Tensor, depth: int, max_walks: int, *,
                    tokens: torch.Tensor | None = None, lens: torch.Tensor | None = None,
                    counts: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                    status: torch.Tensor | None = None, stream=None):
    """BFS walks per root -> (tokens [R, max_walks, 2*depth+1], lens [R, max_walks], counts [R]);
    rows past counts[r] are left as allocated (filled with -1 / 0 when allocated here)."""
    _dev_i32(roots, "roots")
    dev = roots.device
    with _on_stream(dev, stream) as h:
        R = int(roots.shape[0])
        width = 2 * depth + 1
        # the rows no walk takes are filled afterwards: filling both beforehand would write most twice
        fill = tokens is None and lens is None and max_walks > 0
        if tokens is None:
            tokens = (torch.empty((R, max_walks, width), dtype=torch.int32, device=dev) if fill else
                      torch.full((R, max_walks, width), -1, dtype=torch.int32, device=dev))
        if lens is None:
            lens = (torch.empty if fill else torch.zeros)((R, max_walks), dtype=torch.int32, device=dev)
        if counts is None:
            counts = torch.empty(R, dtype=torch.int32, device=dev)
        if workspace is None:
            workspace = torch.empty(max(rdf2v_bfs_walks_workspace_size(csr.num_entities, R), 1),
                                    dtype=torch.uint8, device=dev)
        _same_device(dev, row_ptr=csr.row_ptr, edges=csr.edges)
        _out(tokens, "tokens", torch.int32, R * max(max_walks, 0) * width, dev)
        _out(lens, "lens", torch.int32, R * max(max_walks, 0), dev)
        _out(counts, "counts", torch.int32, R, dev)
        _status(status, dev)
        c = csr._c()
        st = _native().rdf2v_bfs_walks(ctypes.byref(c), _ptr(roots), R, depth, max_walks, _ptr(tokens), _ptr(lens),
                                       _ptr(counts), _ptr(workspace), _ws_bytes(workspace), _ptr(status),
                                       h)
        _check(st, "rdf2v_bfs_walks")
        if fill:
            st = _native().rdf2v_bfs_fill_unused(_ptr(counts), R, max_walks, width, _ptr(tokens), _ptr(lens), h)
            _check(st, "rdf2v_bfs_fill_unused")
        return tokens, lens, counts


def rdf2v_skipgram_pairs_workspace_size(num_walks: int) -> int:
    return int(_native().rdf2v_skipgram_pairs_workspace_size(num_walks))


def rdf2v_skipgram_pairs(tokens: torch.Tensor, lens: torch.Tensor, window: int, *,
                         pairs: torch.Tensor | None = None, count: torch.Tensor | None = None,
                         workspace: torch.Tensor | None = None, status: torch.Tensor | None = None,
                         stream=None):
    """Walk rows tokens [W, width] + lens [W] -> (center, context) pairs [N, 2] int32.

    With `pairs` given, writes at most pairs.shape[0] pairs and returns (pairs, count) with the
    device int64 total (no host synchronisation). Without it, a first call counts, the host reads
    the count, and a second call fills a tensor of exactly that size, which is returned."""
    _dev_i32(tokens, "tokens"); _dev_i32(lens, "lens")
    dev = tokens.device
    with _on_stream(dev, stream) as h:
        w = int(lens.shape[0])
        width = int(tokens.shape[1]) if tokens.dim() == 2 else 1
        if workspace is None:
            workspace = torch.empty(max(rdf2v_skipgram_pairs_workspace_size(w), 1), dtype=torch.uint8, device=dev)
        if count is None:
            count = torch.empty(1, dtype=torch.int64, device=dev)
        _same_device(dev, lens=lens)
        _out(count, "count", torch.int64, 1, dev)
        _status(status, dev)

        def call(out, cap):
            st = _native().rdf2v_skipgram_pairs(_ptr(tokens), _ptr(lens), w, width, window, _ptr(out), cap,
                                              _ptr(count), _ptr(workspace), _ws_bytes(workspace), _ptr(status),
                                              h)
            _check(st, "rdf2v_skipgram_pairs")

        if pairs is not None:
            if pairs.dim() != 2 or pairs.shape[1] != 2:
                raise ValueError("pairs must have shape [capacity, 2]")
            _out(pairs, "pairs", torch.int32, 0, dev)
            call(pairs, int(pairs.shape[0]))
            return pairs, count
        call(None, 0)
        n = int(count.item())
        out = torch.empty((n, 2), dtype=torch.int32, device=dev)
        call(out, n)
        return out


def rdf2v_skipgram_pairs_noalloc(tokens: torch.Tensor, lens: torch.Tensor, window: int, *, pairs: torch.Tensor,
                                 count: torch.Tensor, status: torch.Tensor | None = None, stream=None):
    """rdf2v_skipgram_pairs without a workspace, for callers that cannot allocate: the library's
    fixed per-device scratch serves instead, so this binding allocates nothing either. The caller
    supplies `pairs` [capacity, 2] and `count` (device int64 [1]); at most
    RDF2V_NOALLOC_MAX_WALKS rows per call. Calls that overlap on one device race on the shared
    scratch. Returns (pairs, count) without synchronising."""
    _dev_i32(tokens, "tokens"); _dev_i32(lens, "lens")
    dev = tokens.device
    with _on_stream(dev, stream) as h:
        w = int(lens.shape[0])
        width = int(tokens.shape[1]) if tokens.dim() == 2 else 1
        _same_device(dev, lens=lens)
        if pairs.dim() != 2 or pairs.shape[1] != 2:
            raise ValueError("pairs must have shape [capacity, 2]")
        _out(pairs, "pairs", torch.int32, 0, dev)
        _out(count, "count", torch.int64, 1, dev)
        _status(status, dev)
        st = _native().rdf2v_skipgram_pairs_noalloc(_ptr(tokens), _ptr(lens), w, width, window, _ptr(pairs),
                                                    int(pairs.shape[0]), _ptr(count), _ptr(status), h)
        _check(st, "rdf2v_skipgram_pairs_noalloc")
        return pairs, count


def rdf2v_cbow_examples_workspace_size(num_walks: int) -> int:
    return int(_native().rdf2v_cbow_examples_workspace_size(num_walks))


def rdf2v_cbow_examples(tokens: torch.Tensor, lens: torch.Tensor, window: int, *,
                        centers: torch.Tensor | None = None, contexts: torch.Tensor | None = None,
                        count: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                        status: torch.Tensor | None = None, stream=None):
    """Walk rows tokens [W, width] + lens [W] -> CBOW examples: centers [N] int32 and contexts
    [N, 2*window] int32 (ascending, padded with -1), one example per valid token.

    With `centers` and `contexts` given (capacity = their rows), writes at most that many
    examples and returns (centers, contexts, count) with the device int64 total (no host
    synchronisation). Without them, a first call counts, the host reads the count, and a second
    call fills tensors of exactly that size, which are returned as (centers, contexts)."""
    _dev_i32(tokens, "tokens"); _dev_i32(lens, "lens")
    dev = tokens.device
    with _on_stream(dev, stream) as h:
        w = int(lens.shape[0])
        width = int(tokens.shape[1]) if tokens.dim() == 2 else 1
        if workspace is None:
            workspace = torch.empty(max(rdf2v_cbow_examples_workspace_size(w), 1), dtype=torch.uint8, device=dev)
        if count is None:
            count = torch.empty(1, dtype=torch.int64, device=dev)
        _same_device(dev, lens=lens)
        _out(count, "count", torch.int64, 1, dev)
        _status(status, dev)

        def call(c, x, cap):
            st = _native().rdf2v_cbow_examples(_ptr(tokens), _ptr(lens), w, width, window, _ptr(c), _ptr(x), cap,
                                               _ptr(count), _ptr(workspace), _ws_bytes(workspace), _ptr(status),
                                               h)
            _check(st, "rdf2v_cbow_examples")

        if (centers is None) != (contexts is None):
            raise ValueError("give both centers and contexts, or neither")
        if centers is not None:
            cap = int(centers.numel())
            _out(centers, "centers", torch.int32, 0, dev)
            _out(contexts, "contexts", torch.int32, cap * 2 * max(window, 0), dev)
            call(centers, contexts, cap)
            return centers, contexts, count
        call(None, None, 0)
        n = int(count.item())
        c = torch.empty(n, dtype=torch.int32, device=dev)
        x = torch.empty((n, 2 * window), dtype=torch.int32, device=dev)
        call(c, x, n)
        return c, x


def rdf2v_build_vocabulary_workspace_size(num_triples: int, max_entities: int, max_predicates: int) -> int:
    return int(_native().rdf2v_build_vocabulary_workspace_size(num_triples, max_entities, max_predicates))


def _string_column(col, name: str, n: int):
    chars, offsets = col
    for t, dt in ((chars, torch.uint8), (offsets, torch.int64)):
        if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
            raise TypeError(f"{name} must be CUDA (HIP) tensors")
        if t.dtype != dt or not t.is_contiguous():
            raise TypeError(f"{name}: chars must be contiguous uint8 and offsets contiguous int64")
    if offsets.shape[0] != n + 1:
        raise ValueError(f"{name}: offsets must hold num_triples + 1 entries")
    return [_ptr(chars), _ptr(offsets), int(chars.numel())]


def rdf2v_build_vocabulary(subj, pred, obj, max_entities: int, max_predicates: int, *,
                           ids: tuple | None = None, counts: torch.Tensor | None = None,
                           workspace: torch.Tensor | None = None, status: torch.Tensor | None = None,
                           stream=None):
    """String triples -> id triples. subj, pred, obj are (chars uint8, offsets int64) device
    tensor pairs, string t of a column being chars[offsets[t]:offsets[t+1]].

    Returns (subj_ids, pred_ids, obj_ids, counts): int32 [T] each and a device int64 [2] of
    (distinct entities, distinct predicates); no host synchronisation."""
    offsets = subj[1]
    dev = offsets.device
    with _on_stream(dev, stream) as h:
        n = int(offsets.shape[0]) - 1
        args = (_string_column(subj, "subj", n) + _string_column(pred, "pred", n) + _string_column(obj, "obj", n))
        if ids is None:
            ids = tuple(torch.empty(n, dtype=torch.int32, device=dev) for _ in range(3))
        for i, name in zip(ids, ("subj_ids", "pred_ids", "obj_ids")):
            _out(i, name, torch.int32, n, dev)
        if counts is None:
            counts = torch.empty(2, dtype=torch.int64, device=dev)
        _out(counts, "counts", torch.int64, 2, dev)
        _status(status, dev)
        if workspace is None:
            need = rdf2v_build_vocabulary_workspace_size(n, max_entities, max_predicates)
            workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
        st = _native().rdf2v_build_vocabulary(*args, n, max_entities, max_predicates, *[_ptr(i) for i in ids],
                                              _ptr(counts), _ptr(workspace), _ws_bytes(workspace), _ptr(status),
                                              h)
        _check(st, "rdf2v_build_vocabulary")
        return ids[0], ids[1], ids[2], counts


_DTYPES = {torch.float32: RDF2V_F32, torch.bfloat16: RDF2V_BF16}


def _float_dtype(t: torch.Tensor, name: str) -> int:
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype not in _DTYPES:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return _DTYPES[t.dtype]


def _heads_view(t: torch.Tensor, name: str, dtype: torch.dtype, dev: torch.device, shape) -> _HeadsViewStruct:
    """A [rows, tokens, heads, size] (or [rows, heads, size]) input in any layout whose last dimension
    is contiguous."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != dev:
        raise TypeError(f"{name} must be a {dtype} tensor on {dev}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}; this call needs {tuple(shape)}")
    stride = t.stride()
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return _HeadsViewStruct(t.data_ptr(), stride[0], stride[1] if len(stride) == 4 else 0, stride[-2])


def _exact(t: torch.Tensor, name: str, dtype: torch.dtype, shape, dev: torch.device) -> torch.Tensor:
    """A contiguous tensor of exactly this shape, type and device."""
    if isinstance(t, torch.Tensor) and t.shape == shape and t.dtype == dtype and t.device == dev and t.is_contiguous():
        return t
    _out(t, name, dtype, 0, dev)
    raise ValueError(f"{name} has shape {tuple(t.shape)}; this call needs {tuple(shape)}")


def _state(t: torch.Tensor | None, name: str, shape, dev: torch.device) -> torch.Tensor | None:
    """An optional float32 state tensor of exactly this shape."""
    return None if t is None else _exact(t, name, torch.float32, shape, dev)


class _Attention:
    """The checked arguments that the decay attention calls share."""

    __slots__ = ("c", "views", "dev")

    def __init__(self, q, k, v, log_decay, scale, lens, ndim):
        dtype = _float_dtype(q, "q")
        if not isinstance(v, torch.Tensor):
            raise TypeError("v must be a CUDA (HIP) tensor")
        shape, kind = q.shape, q.dtype
        if len(shape) != ndim or v.dim() != ndim:
            raise ValueError(f"q, k and v must have {ndim} dimensions")
        self.dev = dev = q.device
        heads, dk = shape[-2:]
        kv_heads, dv = v.shape[-2:]
        if kv_heads < 1 or heads % kv_heads:
            raise ValueError(f"{heads} query heads are no multiple of {kv_heads} key and value heads")
        if not 1 <= dk <= RDF2V_MAX_HEAD_SIZE or not 1 <= dv <= RDF2V_MAX_HEAD_SIZE:
            raise ValueError(f"head sizes {dk} and {dv}: 1 to {RDF2V_MAX_HEAD_SIZE} are supported")
        lead = shape[:-2]
        self.views = (_heads_view(q, "q", kind, dev, shape), _heads_view(k, "k", kind, dev, (*lead, kv_heads, dk)),
                      _heads_view(v, "v", kind, dev, (*lead, kv_heads, dv)))
        _exact(log_decay, "log_decay", torch.float32, (heads,), dev)
        if lens is not None:
            _exact(lens, "lens", torch.int32, (lead[0],), dev)
        self.c = _AttentionStruct(lead[0], lead[1] if ndim == 4 else 1, heads, kv_heads, dk, dv, dtype,
                                  dk ** -0.5 if scale is None else scale, log_decay.data_ptr(), _ptr(lens))


def _records(*tensors) -> bool:
    """Whether autograd records what is done with any of these (None: not there). Tangents, which no call carries on,
    are refused, as torch's own functions do that have no forward derivative."""
    if forward_ad._current_level >= 0:
        for t in tensors:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise NotImplementedError("the operators have no forward-mode derivatives: an input has a tangent")
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


def _no_gradient(call: str, names: str) -> None:
    """Said where a gradient is asked for that a call does not compute."""
    warnings.warn(f"{call} computes no gradient for {names}: autograd does not record it. Detach it, or call under "
                  "torch.no_grad()", stacklevel=3)


def _recorded(function, dev: torch.device, stream, *args):
    """function.apply(*args) with the call's stream current: autograd makes the backward call on the stream that is
    current here. What the forward call keeps for it belongs to that stream, is read in its order and given back in its
    order."""
    with _on_stream(dev, stream):
        return function.apply(*args)


def _saved(ctx):
    """What a recorded call has saved. On a stream that the call was given, inputs may belong to another one: their
    memory is not used anew before the backward call, which is the last that holds them, has read them."""
    saved = ctx.saved_tensors
    if ctx.moved:
        current = torch.cuda.current_stream(saved[0].device)
        for t in saved:
            if t is not None:
                t.record_stream(current)
    return saved


# Tells autograd that a call has written to these tensors, as an operation of torch in place does: gradients that would
# read what was there before raise an error. torch.autograd.graph.increment_version, at half of its time.
_written = torch._C._increment_version


def _written_of(*given) -> None:
    """The same of outputs that the caller may have given (None: a new one, which nothing has seen)."""
    for t in given:
        if t is not None:
            _written((t,))


class _DecayAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, state, scale, lens, want_state, workspace, status, stream):
        out, state_out = rdf2v_decay_attention(q, k, v, log_decay, scale=scale, lens=lens, state=state,
                                               want_state=want_state, workspace=workspace, status=status, stream=stream)
        ctx.moved = stream is not None
        ctx.save_for_backward(q, k, v, log_decay, state, lens)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return (out, state_out) if want_state else out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dstate_out=None):
        q, k, v, log_decay, state, lens = _saved(ctx)
        if dout is None:                                   # the states alone were used
            dout = q.new_zeros((*q.shape[:-1], v.shape[-1]))
        elif dout.stride(-1) != 1:
            dout = dout.contiguous()
        if dstate_out is not None:
            dstate_out = dstate_out.contiguous()
        dq, dk, dv, dstate = rdf2v_decay_attention_backward(q, k, v, log_decay, dout, scale=ctx.scale, lens=lens,
                                                            state=state, dstate_out=dstate_out)
        return dq, dk, dv, None, dstate, None, None, None, None, None, None


def rdf2v_decay_attention_workspace_size(rows: int, length: int, heads: int, kv_heads: int, dk: int, dv: int,
                                         dtype: torch.dtype = torch.float32) -> int:
    c = _AttentionStruct(rows, length, heads, kv_heads, dk, dv, _DTYPES.get(dtype, -1), 1.0, None, None)
    return int(_native().rdf2v_decay_attention_workspace_size(ctypes.byref(c)))


def rdf2v_decay_attention_backward_workspace_size(rows: int, length: int, heads: int, kv_heads: int, dk: int, dv: int,
                                                  dtype: torch.dtype = torch.float32) -> int:
    c = _AttentionStruct(rows, length, heads, kv_heads, dk, dv, _DTYPES.get(dtype, -1), 1.0, None, None)
    return int(_native().rdf2v_decay_attention_backward_workspace_size(ctypes.byref(c)))


def rdf2v_decay_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor, *,
                          scale: float | None = None, lens: torch.Tensor | None = None,
                          state: torch.Tensor | None = None, want_state: bool = False,
                          out: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                          workspace: torch.Tensor | None = None, status: torch.Tensor | None = None, stream=None):
    """Linear attention with a decay for each head over rows of tokens:
    S_t = exp(log_decay) S_{t-1} + k_t v_t^T, out_t = scale * S_t^T q_t.

    q [rows, length, heads, dk], k [rows, length, kv_heads, dk] and v [rows, length, kv_heads, dv] are
    float32 or bfloat16 in any layout whose last dimension is contiguous; query head h reads key and
    value head h // (heads // kv_heads). log_decay: float32 [heads], <= 0. scale defaults to dk ** -0.5.
    lens: int32 [rows], the tokens of each row that count (as the walk calls return them). state: float32
    [rows, heads, dk, dv] to begin from. Returns (out [rows, length, heads, dv], state_out), state_out
    being None unless it is given or want_state is set.

    Where q, k, v or state requires gradients, autograd records the call; out and state_out must then be left
    to it, as in torch's own functions."""
    a = _Attention(q, k, v, log_decay, scale, lens, 4)
    dev, c = a.dev, a.c
    if _records(log_decay):
        _no_gradient("rdf2v_decay_attention", "log_decay")
    if _records(q, k, v, state):
        if out is not None or state_out is not None:
            raise ValueError("out and state_out cannot be given where autograd records the call: an input requires "
                             "gradients")
        got = _recorded(_DecayAttention, dev, stream, q, k, v, log_decay, state, scale, lens, want_state, workspace,
                        status, stream)
        return got if want_state else (got, None)
    with _on_stream(dev, stream) as h:
        given = out, state_out
        shape = (c.rows, c.heads, c.dk, c.dv)
        if out is None:
            out = torch.empty((c.rows, c.length, c.heads, c.dv), dtype=q.dtype, device=dev)
        else:
            _exact(out, "out", q.dtype, (c.rows, c.length, c.heads, c.dv), dev)
        if state_out is None:
            if want_state:
                state_out = torch.empty(shape, dtype=torch.float32, device=dev)
        else:
            _state(state_out, "state_out", shape, dev)
        _state(state, "state", shape, dev)
        _status(status, dev)
        ref = ctypes.byref(c)
        if workspace is None:
            need = _native().rdf2v_decay_attention_workspace_size(ref)
            workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        vq, vk, vv = a.views
        st = _native().rdf2v_decay_attention(ref, vq, vk, vv, _ptr(state), _ptr(out), _ptr(state_out),
                                             _ptr(workspace), _ws_bytes(workspace), _ptr(status), h)
        _check(st, "rdf2v_decay_attention")
        _written_of(*given)
        return out, state_out


def rdf2v_decay_attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor,
                                   dout: torch.Tensor, *, scale: float | None = None,
                                   lens: torch.Tensor | None = None, state: torch.Tensor | None = None,
                                   dstate_out: torch.Tensor | None = None, dq: torch.Tensor | None = None,
                                   dk: torch.Tensor | None = None, dv: torch.Tensor | None = None,
                                   dstate: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                                   status: torch.Tensor | None = None, stream=None):
    """Gradients of rdf2v_decay_attention for its inputs, from dout (that of out) and dstate_out (that of
    state_out; None: zeros). Returns (dq, dk, dv, dstate) in the shapes of q, k, v and state; dstate is
    None unless state or dstate is given. log_decay is a constant and has no gradient."""
    a = _Attention(q, k, v, log_decay, scale, lens, 4)
    dev, c = a.dev, a.c
    with _on_stream(dev, stream) as h:
        given = dq, dk, dv, dstate
        shape = (c.rows, c.heads, c.dk, c.dv)
        view = _heads_view(dout, "dout", q.dtype, dev, (c.rows, c.length, c.heads, c.dv))
        grads = []
        for t, like, name in ((dq, q, "dq"), (dk, k, "dk"), (dv, v, "dv")):
            grads.append(torch.empty(like.shape, dtype=q.dtype, device=dev) if t is None else
                         _exact(t, name, q.dtype, like.shape, dev))
        dq, dk, dv = grads
        if dstate is None:
            if state is not None:
                dstate = torch.empty(shape, dtype=torch.float32, device=dev)
        else:
            _state(dstate, "dstate", shape, dev)
        _state(state, "state", shape, dev)
        _state(dstate_out, "dstate_out", shape, dev)
        _status(status, dev)
        ref = ctypes.byref(c)
        if workspace is None:
            need = _native().rdf2v_decay_attention_backward_workspace_size(ref)
            workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        vq, vk, vv = a.views
        st = _native().rdf2v_decay_attention_backward(ref, vq, vk, vv, view, _ptr(state), _ptr(dstate_out), _ptr(dq),
                                                      _ptr(dk), _ptr(dv), _ptr(dstate), _ptr(workspace),
                                                      _ws_bytes(workspace), _ptr(status), h)
        _check(st, "rdf2v_decay_attention_backward")
        _written_of(*given)
        return dq, dk, dv, dstate


def rdf2v_decay_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor,
                               state: torch.Tensor, *, scale: float | None = None,
                               parents: torch.Tensor | None = None, out: torch.Tensor | None = None,
                               state_out: torch.Tensor | None = None, status: torch.Tensor | None = None,
                               stream=None):
    """rdf2v_decay_attention for one more token of each row: q [rows, heads, dk], k [rows, kv_heads, dk],
    v [rows, kv_heads, dv], state float32 [num_states, heads, dk, dv]. Returns (out [rows, heads, dv],
    state_out [rows, heads, dk, dv]).

    With parents (int32, one per row), row r continues state parents[r], as rdf2v_beam_select numbers
    them, and state_out must not overlap state. Without, row r continues state r, and state is updated
    in place unless state_out is given. For answering: autograd does not record it."""
    a = _Attention(q, k, v, log_decay, scale, None, 3)
    dev, c = a.dev, a.c
    with _on_stream(dev, stream) as h:
        given = out
        shape = (c.rows, c.heads, c.dk, c.dv)
        num_states = c.rows
        if parents is not None:
            _out(parents, "parents", torch.int32, 0, dev)
            if parents.numel() != c.rows:
                raise ValueError(f"parents holds {parents.numel()} elements; this call needs {c.rows}")
            num_states = state.shape[0] if isinstance(state, torch.Tensor) and state.dim() == 4 else c.rows
        if state is None:
            raise TypeError("state must be a CUDA (HIP) tensor")
        _state(state, "state", (num_states,) + shape[1:], dev)
        if out is None:
            out = torch.empty((c.rows, c.heads, c.dv), dtype=q.dtype, device=dev)
        else:
            _exact(out, "out", q.dtype, (c.rows, c.heads, c.dv), dev)
        if state_out is None:
            state_out = state if parents is None else torch.empty(shape, dtype=torch.float32, device=dev)
        else:
            _state(state_out, "state_out", shape, dev)
        _status(status, dev)
        if _records(q, k, v, log_decay, state):
            _no_gradient("rdf2v_decay_attention_step", "its inputs")
        vq, vk, vv = a.views
        st = _native().rdf2v_decay_attention_step(ctypes.byref(c), vq, vk, vv, _ptr(state), num_states,
                                                  _ptr(parents), _ptr(out), _ptr(state_out), _ptr(status), h)
        _check(st, "rdf2v_decay_attention_step")
        _written((state_out,) if given is None else (given, state_out))
        return out, state_out


def rdf2v_beam_select_workspace_size(groups: int, beams: int, vocab: int, num_out: int) -> int:
    return int(_native().rdf2v_beam_select_workspace_size(groups, beams, vocab, num_out))


def rdf2v_beam_select(logits: torch.Tensor, scores: torch.Tensor, num_out: int, *,
                      finished: torch.Tensor | None = None, scores_out: torch.Tensor | None = None,
                      tokens: torch.Tensor | None = None, parents: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None, status: torch.Tensor | None = None, stream=None):
    """The num_out best continuations of each group's beams: logits [groups, beams, vocab] (float32 or
    bfloat16; beams contiguous up to a row stride), scores float32 [groups, beams]. Totals are
    scores + log_softmax(logits); a beam whose `finished` (int32 [groups, beams]) is nonzero has one
    candidate, token -1 at its score.

    Returns (scores, tokens, parents), each [groups, num_out]: totals in descending order, ties to the
    lowest (beam, token); parents are row numbers group * beams + beam, as rdf2v_beam_reorder and
    rdf2v_decay_attention_step take them. Places without a candidate hold -inf, -1 and the group's first
    row. For answering: autograd does not record it."""
    dtype = _float_dtype(logits, "logits")
    if logits.dim() != 3:
        raise ValueError("logits must have shape [groups, beams, vocab]")
    dev = logits.device
    with _on_stream(dev, stream) as h:
        given = scores_out, tokens, parents
        groups, beams, vocab = logits.shape
        gs, bs, vs = logits.stride()
        if (vs != 1 and vocab > 1) or (gs != beams * bs and groups > 1 and beams > 1):
            raise ValueError("logits must be rows of contiguous values at one row stride")
        row = bs if beams > 1 else gs if groups > 1 else vocab
        _exact(scores, "scores", torch.float32, (groups, beams), dev)
        if finished is not None:
            _exact(finished, "finished", torch.int32, (groups, beams), dev)
        shape = (groups, num_out)
        scores_out = (torch.empty(shape, dtype=torch.float32, device=dev) if scores_out is None else
                      _exact(scores_out, "scores_out", torch.float32, shape, dev))
        tokens = (torch.empty(shape, dtype=torch.int32, device=dev) if tokens is None else
                  _exact(tokens, "tokens", torch.int32, shape, dev))
        parents = (torch.empty(shape, dtype=torch.int32, device=dev) if parents is None else
                   _exact(parents, "parents", torch.int32, shape, dev))
        _status(status, dev)
        if _records(logits, scores):
            _no_gradient("rdf2v_beam_select", "logits and scores")
        lib = _native()
        if workspace is None:
            need = lib.rdf2v_beam_select_workspace_size(groups, beams, vocab, num_out)
            workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        st = lib.rdf2v_beam_select(_ptr(logits), row, dtype, _ptr(scores), _ptr(finished), groups, beams, vocab,
                                   num_out, _ptr(scores_out), _ptr(tokens), _ptr(parents), _ptr(workspace),
                                   _ws_bytes(workspace), _ptr(status), h)
        _check(st, "rdf2v_beam_select")
        _written_of(*given)
        return scores_out, tokens, parents


def rdf2v_beam_reorder(src: torch.Tensor, parents: torch.Tensor, *, out: torch.Tensor | None = None,
                       status: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Rows of src (any type, contiguous) in the order of parents (int32, any shape): out[r] =
    src[parents.flatten()[r]]. For answering: autograd does not record it."""
    _dev_i32(parents, "parents")
    dev = parents.device
    if not isinstance(src, torch.Tensor) or src.device != dev:
        raise TypeError(f"src must be a CUDA (HIP) tensor on {dev}")
    if src.dim() < 1 or not src.is_contiguous():
        raise ValueError("src must be contiguous rows")
    with _on_stream(dev, stream) as h:
        given = (out,)
        rows, shape = parents.numel(), src.shape[1:]
        if out is None:
            out = torch.empty((rows,) + shape, dtype=src.dtype, device=dev)
        else:
            _exact(out, "out", src.dtype, (rows,) + shape, dev)
        _status(status, dev)
        if _records(src):
            _no_gradient("rdf2v_beam_reorder", "src")
        row_bytes = src.element_size() * shape.numel()
        st = _native().rdf2v_beam_reorder(_ptr(src), src.shape[0], row_bytes, _ptr(parents), rows, _ptr(out),
                                          _ptr(status), h)
        _check(st, "rdf2v_beam_reorder")
        _written_of(*given)
        return out


def rdf2v_distill_workspace_size(rows: int, vocab: int, top: int, dtype: torch.dtype = torch.float32) -> int:
    return int(_native().rdf2v_distill_workspace_size(rows, vocab, top, _DTYPES.get(dtype, -1)))


def _rows(t: torch.Tensor, name: str, like: torch.Tensor) -> int:
    """Row stride of a [rows, vocab] tensor with contiguous rows."""
    if not isinstance(t, torch.Tensor) or t.device != like.device or t.dtype != like.dtype:
        raise TypeError(f"{name} must be a {like.dtype} tensor on {like.device}")
    if t.dim() != 2 or t.shape != like.shape:
        raise ValueError(f"{name} must have shape [rows, vocab]")
    rows, vocab = t.shape
    row, one = t.stride()
    if one != 1 and vocab > 1:
        raise ValueError(f"rows of {name} must be contiguous")
    if row < vocab and rows > 1:
        raise ValueError(f"rows of {name} must not overlap")
    return row if rows > 1 else max(row, vocab)


def _teacher(logits, ids, teacher):
    dtype = _float_dtype(logits, "logits")
    stride = _rows(logits, "logits", logits)
    dev = logits.device
    _dev_i32(ids, "ids")
    if ids.dim() != 2 or ids.shape[0] != logits.shape[0]:
        raise ValueError("ids must have shape [rows, top]")
    _same_device(dev, ids=ids)
    _exact(teacher, "teacher", torch.float32, ids.shape, dev)
    return dtype, stride, dev


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, teacher, temperature, workspace, status, stream):
        loss, lse = rdf2v_distill_loss(logits, ids, teacher, temperature=temperature, workspace=workspace,
                                       status=status, stream=stream)
        ctx.moved = stream is not None
        ctx.save_for_backward(logits, ids, teacher, lse)
        ctx.temperature = temperature
        ctx.mark_non_differentiable(lse)
        return loss, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss, _):
        logits, ids, teacher, lse = _saved(ctx)
        grad = rdf2v_distill_loss_backward(logits, ids, teacher, lse, dloss.contiguous(), temperature=ctx.temperature)
        return grad, None, None, None, None, None, None


def rdf2v_distill_loss(logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, *, temperature: float = 1.0,
                       dloss: torch.Tensor | None = None, loss: torch.Tensor | None = None,
                       lse: torch.Tensor | None = None, dlogits: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None, status: torch.Tensor | None = None, stream=None):
    """Distillation from a teacher's top logits: temperature^2 * KL(softmax of the teacher's entries /
    temperature || softmax(logits / temperature)) for each row.

    logits [rows, vocab] float32 or bfloat16, rows contiguous; ids int32 [rows, top] (negative: absent)
    and teacher float32 [rows, top]. Returns (loss, lse), float32 [rows]; with dloss (float32 [rows], the
    gradient of loss) the gradient of the logits is computed in the same pass and (loss, lse, dlogits) is
    returned. dlogits may be logits itself.

    Where logits requires gradients and dloss is not given, autograd records loss (not lse); loss and lse must
    then be left to the call, as in torch's own functions."""
    dtype, stride, dev = _teacher(logits, ids, teacher)
    if _records(teacher):
        _no_gradient("rdf2v_distill_loss", "teacher")
    if _records(logits) and dloss is None and dlogits is None:
        if loss is not None or lse is not None:
            raise ValueError("loss and lse cannot be given where autograd records the call: logits requires gradients")
        return _recorded(_DistillLoss, dev, stream, logits, ids, teacher, temperature, workspace, status, stream)
    with _on_stream(dev, stream) as h:
        given = loss, lse, dlogits
        rows, vocab = logits.shape
        loss = torch.empty(rows, dtype=torch.float32, device=dev) if loss is None else \
            _exact(loss, "loss", torch.float32, (rows,), dev)
        lse = torch.empty(rows, dtype=torch.float32, device=dev) if lse is None else \
            _exact(lse, "lse", torch.float32, (rows,), dev)
        dstride = vocab
        if dloss is not None:
            _exact(dloss, "dloss", torch.float32, (rows,), dev)
            if dlogits is None:
                dlogits = torch.empty((rows, vocab), dtype=logits.dtype, device=dev)
            else:
                dstride = _rows(dlogits, "dlogits", logits)
        elif dlogits is not None:
            raise ValueError("dlogits needs dloss")
        _status(status, dev)
        lib = _native()
        if workspace is None:
            need = lib.rdf2v_distill_workspace_size(rows, vocab, ids.shape[1], dtype)
            workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        st = lib.rdf2v_distill_loss(_ptr(logits), stride, dtype, _ptr(ids), _ptr(teacher), rows, vocab, ids.shape[1],
                                    temperature, _ptr(loss), _ptr(lse), _ptr(dloss), _ptr(dlogits), dstride,
                                    _ptr(workspace), _ws_bytes(workspace), _ptr(status), h)
        _check(st, "rdf2v_distill_loss")
        _written_of(*given)
        return (loss, lse) if dloss is None else (loss, lse, dlogits)


def rdf2v_distill_loss_backward(logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, lse: torch.Tensor,
                                dloss: torch.Tensor, *, temperature: float = 1.0, dlogits: torch.Tensor | None = None,
                                workspace: torch.Tensor | None = None, status: torch.Tensor | None = None,
                                stream=None) -> torch.Tensor:
    """The gradient of the logits alone, with the lse that rdf2v_distill_loss returned."""
    dtype, stride, dev = _teacher(logits, ids, teacher)
    with _on_stream(dev, stream) as h:
        given = (dlogits,)
        rows, vocab = logits.shape
        _exact(lse, "lse", torch.float32, (rows,), dev)
        _exact(dloss, "dloss", torch.float32, (rows,), dev)
        dstride = vocab
        if dlogits is None:
            dlogits = torch.empty((rows, vocab), dtype=logits.dtype, device=dev)
        else:
            dstride = _rows(dlogits, "dlogits", logits)
        _status(status, dev)
        lib = _native()
        if workspace is None:
            need = lib.rdf2v_distill_workspace_size(rows, vocab, ids.shape[1], dtype)
            workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        st = lib.rdf2v_distill_loss_backward(_ptr(logits), stride, dtype, _ptr(ids), _ptr(teacher), rows, vocab,
                                             ids.shape[1], temperature, _ptr(lse), _ptr(dloss), _ptr(dlogits),
                                             dstride, _ptr(workspace), _ws_bytes(workspace), _ptr(status), h)
        _check(st, "rdf2v_distill_loss_backward")
        _written_of(*given)
        return dlogits


def _tokens_view(t: torch.Tensor, name: str, dtype: torch.dtype, dev: torch.device, shape) -> _TokensViewStruct:
    """A [rows, tokens, channels] (or [rows, channels]) input in any layout whose last dimension is contiguous."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != dev:
        raise TypeError(f"{name} must be a {dtype} tensor on {dev}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}; this call needs {tuple(shape)}")
    stride = t.stride()
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return _TokensViewStruct(t.data_ptr(), stride[0], stride[1] if len(stride) == 3 else 0)


def _parameter(t: torch.Tensor | None, name: str, shape, dev: torch.device):
    """Pointer of an optional float32 parameter of exactly this shape."""
    return None if t is None else _exact(t, name, torch.float32, shape, dev).data_ptr()


def _new(t: torch.Tensor | None, name: str, dtype: torch.dtype, shape, dev: torch.device) -> torch.Tensor:
    """An output of exactly this shape: the caller's, or a new one."""
    return torch.empty(tuple(shape), dtype=dtype, device=dev) if t is None else _exact(t, name, dtype, shape, dev)


def _new_like(t: torch.Tensor | None, name: str, like: torch.Tensor, dtype: torch.dtype | None = None) -> torch.Tensor:
    """The same in an input's shape, and type unless another is given; half of _new's time."""
    if t is not None:
        return _exact(t, name, dtype or like.dtype, like.shape, like.device)
    return torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)


def _workspace(need: int, dev: torch.device) -> torch.Tensor | None:
    return torch.empty(need, dtype=torch.uint8, device=dev) if need else None


def _gradient(t: torch.Tensor | None, like) -> torch.Tensor:
    """What autograd hands a backward call for an output, as the calls take it; zeros for an output that was not used."""
    if t is None:
        return torch.zeros(like[0], dtype=like[1], device=like[2])
    return t if t.stride(-1) == 1 or t.shape[-1] <= 1 else t.contiguous()


def _lens(t: torch.Tensor | None, rows: int, dev: torch.device):
    return None if t is None else _ptr(_exact(t, "lens", torch.int32, (rows,), dev))


def _parents_and_states(parents, state, rows: int, tail, dtype: torch.dtype, dev: torch.device) -> int:
    """Checks a step's parents and states; returns how many states there are."""
    num_states = rows
    if parents is not None:
        _out(parents, "parents", torch.int32, 0, dev)
        if parents.numel() != rows:
            raise ValueError(f"parents holds {parents.numel()} elements; this call needs {rows}")
        if isinstance(state, torch.Tensor) and state.dim() == len(tail) + 1:
            num_states = state.shape[0]
    if state is None:
        raise TypeError("state must be a CUDA (HIP) tensor")
    _exact(state, "state", dtype, (num_states, *tail), dev)
    return num_states


class _Conv:
    """The checked arguments that the causal convolution calls share."""

    __slots__ = ("c", "view", "dev", "dtype", "shape", "states")

    def __init__(self, x, weight, bias, silu, lens, ndim):
        dtype = _float_dtype(x, "x")
        shape = self.shape = x.shape
        if len(shape) != ndim:
            raise ValueError(f"x must have {ndim} dimensions")
        dev, self.dtype = x.device, x.dtype
        self.dev = dev
        rows, channels = shape[0], shape[-1]
        if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
            raise ValueError("weight must have shape [channels, width]")
        width = weight.shape[1]
        if not 1 <= width <= RDF2V_MAX_CONV_WIDTH:
            raise ValueError(f"width {width}: 1 to {RDF2V_MAX_CONV_WIDTH} are supported")
        if channels < 1:
            raise ValueError("x must have channels")
        self.view = _tokens_view(x, "x", x.dtype, dev, shape)
        self.states = (rows, width - 1, channels)
        self.c = _ConvStruct(rows, shape[1] if ndim == 3 else 1, channels, width, dtype, bool(silu),
                             _parameter(weight, "weight", (channels, width), dev),
                             _parameter(bias, "bias", (channels,), dev), _lens(lens, rows, dev))


class _CausalConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, state, silu, lens, want_state, status, stream):
        out, state_out = rdf2v_causal_conv(x, weight, bias, silu=silu, lens=lens, state=state, want_state=want_state,
                                           status=status, stream=stream)
        ctx.moved = stream is not None
        ctx.save_for_backward(x, weight, bias, state, lens)
        ctx.silu = silu
        ctx.set_materialize_grads(False)
        return (out, state_out) if want_state else out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dstate_out=None):
        x, weight, bias, state, lens = _saved(ctx)
        if dstate_out is not None:
            dstate_out = dstate_out.contiguous()
        dx, dweight, dbias, dstate = rdf2v_causal_conv_backward(
            x, weight, bias, _gradient(dout, (x.shape, x.dtype, x.device)), silu=ctx.silu, lens=lens, state=state,
            dstate_out=dstate_out)
        return dx, dweight, dbias, dstate, None, None, None, None, None


def rdf2v_causal_conv(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, *, silu: bool = True,
                      lens: torch.Tensor | None = None, state: torch.Tensor | None = None, want_state: bool = False,
                      out: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                      status: torch.Tensor | None = None, stream=None):
    """Causal convolution of each channel by itself: u_t = bias + sum_j weight[:, j] x_{t - width + 1 + j}, out_t = u_t
    sigmoid(u_t), or u_t where silu is False.

    x [rows, length, channels] is float32 or bfloat16 in any layout whose last dimension is contiguous; weight
    [channels, width] and bias [channels] are float32. lens: int32 [rows], the tokens of each row that count. state
    [rows, width - 1, channels] in x's type: the inputs before the row's first (None: zeros). Returns (out, state_out),
    state_out (the last width - 1 inputs) being None unless it is given or want_state is set.

    Where x, weight, bias or state requires gradients, autograd records the call; out and state_out must then be left
    to it, as in torch's own functions."""
    a = _Conv(x, weight, bias, silu, lens, 3)
    dev, c = a.dev, a.c
    if _records(x, weight, bias, state):
        if out is not None or state_out is not None:
            raise ValueError("out and state_out cannot be given where autograd records the call: an input requires "
                             "gradients")
        got = _recorded(_CausalConv, dev, stream, x, weight, bias, state, silu, lens, want_state, status, stream)
        return got if want_state else (got, None)
    with _on_stream(dev, stream) as h:
        given = out, state_out
        out = _new_like(out, "out", x)
        if want_state or state_out is not None:
            state_out = _new(state_out, "state_out", a.dtype, a.states, dev)
        if state is not None:
            _exact(state, "state", a.dtype, a.states, dev)
        _status(status, dev)
        st = _native().rdf2v_causal_conv(c, a.view, _ptr(state), _ptr(out), _ptr(state_out), _ptr(status), h)
        _check(st, "rdf2v_causal_conv")
        _written_of(*given)
        return out, state_out


def rdf2v_causal_conv_backward_workspace_size(rows: int, length: int, channels: int, width: int,
                                              dtype: torch.dtype = torch.float32) -> int:
    c = _ConvStruct(rows, length, channels, width, _DTYPES.get(dtype, -1), 1, None, None, None)
    return int(_native().rdf2v_causal_conv_backward_workspace_size(c))


def rdf2v_causal_conv_backward(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None, dout: torch.Tensor, *,
                               silu: bool = True, lens: torch.Tensor | None = None, state: torch.Tensor | None = None,
                               dstate_out: torch.Tensor | None = None, dx: torch.Tensor | None = None,
                               dweight: torch.Tensor | None = None, dbias: torch.Tensor | None = None,
                               dstate: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                               status: torch.Tensor | None = None, stream=None):
    """Gradients of rdf2v_causal_conv for its inputs, from dout (that of out) and dstate_out (that of state_out; None:
    zeros). Returns (dx, dweight, dbias, dstate); dbias is None unless bias or dbias is given, dstate unless state or
    dstate is."""
    a = _Conv(x, weight, bias, silu, lens, 3)
    dev, c = a.dev, a.c
    with _on_stream(dev, stream) as h:
        given = dx, dweight, dbias, dstate
        view = _tokens_view(dout, "dout", a.dtype, dev, a.shape)
        dx = _new_like(dx, "dx", x)
        dweight = _new(dweight, "dweight", torch.float32, weight.shape, dev)
        if bias is not None or dbias is not None:
            dbias = _new(dbias, "dbias", torch.float32, (c.channels,), dev)
        if state is not None or dstate is not None:
            dstate = _new(dstate, "dstate", a.dtype, a.states, dev)
        for t, name in ((state, "state"), (dstate_out, "dstate_out")):
            if t is not None:
                _exact(t, name, a.dtype, a.states, dev)
        _status(status, dev)
        lib = _native()
        if workspace is None:
            workspace = _workspace(lib.rdf2v_causal_conv_backward_workspace_size(c), dev)
        st = lib.rdf2v_causal_conv_backward(c, a.view, view, _ptr(state), _ptr(dstate_out), _ptr(dx), _ptr(dweight),
                                            _ptr(dbias), _ptr(dstate), _ptr(workspace), _ws_bytes(workspace),
                                            _ptr(status), h)
        _check(st, "rdf2v_causal_conv_backward")
        _written_of(*given)
        return dx, dweight, dbias, dstate


def rdf2v_causal_conv_step(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None, state: torch.Tensor, *,
                           silu: bool = True, parents: torch.Tensor | None = None, out: torch.Tensor | None = None,
                           state_out: torch.Tensor | None = None, status: torch.Tensor | None = None, stream=None):
    """rdf2v_causal_conv for one more token of each row: x [rows, channels], state [num_states, width - 1, channels] in
    x's type. Returns (out [rows, channels], state_out [rows, width - 1, channels]). parents and state_out are as in
    rdf2v_decay_attention_step. For answering: autograd does not record it."""
    a = _Conv(x, weight, bias, silu, None, 2)
    dev, c = a.dev, a.c
    with _on_stream(dev, stream) as h:
        given = out
        num_states = _parents_and_states(parents, state, c.rows, a.states[1:], a.dtype, dev)
        out = _new_like(out, "out", x)
        if state_out is None and parents is None:
            state_out = state
        state_out = _new(state_out, "state_out", a.dtype, a.states, dev)
        _status(status, dev)
        if _records(x, weight, bias, state):
            _no_gradient("rdf2v_causal_conv_step", "its inputs")
        st = _native().rdf2v_causal_conv_step(c, a.view, _ptr(state), num_states, _ptr(parents), _ptr(out),
                                              _ptr(state_out), _ptr(status), h)
        _check(st, "rdf2v_causal_conv_step")
        _written((state_out,) if given is None else (given, state_out))
        return out, state_out


class ScanGradients(NamedTuple):
    """Gradients of rdf2v_selective_scan's inputs; None for an input that was not given."""

    dx: torch.Tensor
    ddt: torch.Tensor
    da: torch.Tensor
    db: torch.Tensor
    dc: torch.Tensor
    ddt_bias: torch.Tensor | None
    dskip: torch.Tensor | None
    dgate: torch.Tensor | None
    dstate: torch.Tensor | None


class _Scan:
    """The checked arguments that the selective scan calls share."""

    __slots__ = ("c", "views", "dev", "dtype", "shape", "heads", "states")

    def __init__(self, x, dt, a, b, c, dt_bias, skip, gate, lens, ndim):
        dtype = _float_dtype(x, "x")
        shape = self.shape = x.shape
        if len(shape) != ndim:
            raise ValueError(f"x must have {ndim} dimensions")
        dev, kind = x.device, x.dtype
        self.dev, self.dtype = dev, kind
        rows, channels = shape[0], shape[-1]
        if not isinstance(b, torch.Tensor) or b.dim() != ndim + 1:
            raise ValueError(f"b and c must have {ndim + 1} dimensions")
        groups, states = b.shape[-2:]
        if channels < 1 or groups < 1 or channels % groups:
            raise ValueError(f"{channels} channels are no multiple of {groups} groups")
        if not 1 <= states <= RDF2V_MAX_SCAN_STATES:
            raise ValueError(f"{states} states: 1 to {RDF2V_MAX_SCAN_STATES} are supported")
        self.heads = (*shape[:-1], groups, states)
        self.states = (rows, channels, states)
        self.views = (_tokens_view(x, "x", kind, dev, shape), _tokens_view(dt, "dt", kind, dev, shape),
                      _heads_view(b, "b", kind, dev, self.heads), _heads_view(c, "c", kind, dev, self.heads),
                      None if gate is None else _tokens_view(gate, "gate", kind, dev, shape))
        if a is None:
            raise TypeError("a must be a CUDA (HIP) tensor")
        self.c = _ScanStruct(rows, shape[1] if ndim == 3 else 1, channels, groups, states, dtype,
                             _parameter(a, "a", (channels, states), dev),
                             _parameter(dt_bias, "dt_bias", (channels,), dev),
                             _parameter(skip, "skip", (channels,), dev), _lens(lens, rows, dev))


class _SelectiveScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, dt, a, b, c, dt_bias, skip, gate, state, lens, want_state, workspace, status, stream):
        out, state_out = rdf2v_selective_scan(x, dt, a, b, c, dt_bias=dt_bias, skip=skip, gate=gate, lens=lens,
                                              state=state, want_state=want_state, workspace=workspace, status=status,
                                              stream=stream)
        ctx.moved = stream is not None
        ctx.save_for_backward(x, dt, a, b, c, dt_bias, skip, gate, state, lens)
        ctx.set_materialize_grads(False)
        return (out, state_out) if want_state else out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dstate_out=None):
        x, dt, a, b, c, dt_bias, skip, gate, state, lens = _saved(ctx)
        if dstate_out is not None:
            dstate_out = dstate_out.contiguous()
        g = rdf2v_selective_scan_backward(x, dt, a, b, c, _gradient(dout, (x.shape, x.dtype, x.device)),
                                          dt_bias=dt_bias, skip=skip, gate=gate, lens=lens, state=state,
                                          dstate_out=dstate_out)
        return g.dx, g.ddt, g.da, g.db, g.dc, g.ddt_bias, g.dskip, g.dgate, g.dstate, None, None, None, None, None


def rdf2v_selective_scan_workspace_size(rows: int, length: int, channels: int, groups: int, states: int,
                                        dtype: torch.dtype = torch.float32) -> int:
    c = _ScanStruct(rows, length, channels, groups, states, _DTYPES.get(dtype, -1), None, None, None, None)
    return int(_native().rdf2v_selective_scan_workspace_size(c))


def rdf2v_selective_scan_backward_workspace_size(rows: int, length: int, channels: int, groups: int, states: int,
                                                 dtype: torch.dtype = torch.float32) -> int:
    c = _ScanStruct(rows, length, channels, groups, states, _DTYPES.get(dtype, -1), None, None, None, None)
    return int(_native().rdf2v_selective_scan_backward_workspace_size(c))


def rdf2v_selective_scan(x: torch.Tensor, dt: torch.Tensor, a: torch.Tensor, b: torch.Tensor, c: torch.Tensor, *,
                         dt_bias: torch.Tensor | None = None, skip: torch.Tensor | None = None,
                         gate: torch.Tensor | None = None, lens: torch.Tensor | None = None,
                         state: torch.Tensor | None = None, want_state: bool = False, out: torch.Tensor | None = None,
                         state_out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                         status: torch.Tensor | None = None, stream=None):
    """Selective scan over rows of tokens, channel by channel: delta_t = softplus(dt_t + dt_bias), h_t = exp(delta_t a)
    h_{t-1} + delta_t x_t b_t, y_t = c_t . h_t + skip x_t, out_t = y_t gate_t sigmoid(gate_t) (y_t without a gate).

    x, dt and gate [rows, length, channels] and b and c [rows, length, groups, states] are float32 or bfloat16 in any
    layout whose last dimension is contiguous; channel d reads group d // (channels // groups). a [channels, states]
    (finite, <= 0; below -2^95 it counts as that), dt_bias and skip [channels] are float32. lens: int32 [rows], the
    tokens of each row that count.
    state: float32 [rows, channels, states] to begin from. Returns (out, state_out), state_out being None unless it is
    given or want_state is set.

    Where an input requires gradients, autograd records the call; out and state_out must then be left to it, as in
    torch's own functions."""
    s = _Scan(x, dt, a, b, c, dt_bias, skip, gate, lens, 3)
    dev = s.dev
    if _records(x, dt, a, b, c, dt_bias, skip, gate, state):
        if out is not None or state_out is not None:
            raise ValueError("out and state_out cannot be given where autograd records the call: an input requires "
                             "gradients")
        got = _recorded(_SelectiveScan, dev, stream, x, dt, a, b, c, dt_bias, skip, gate, state, lens, want_state,
                        workspace, status, stream)
        return got if want_state else (got, None)
    with _on_stream(dev, stream) as h:
        given = out, state_out
        out = _new_like(out, "out", x)
        if want_state or state_out is not None:
            state_out = _new(state_out, "state_out", torch.float32, s.states, dev)
        _state(state, "state", s.states, dev)
        _status(status, dev)
        lib = _native()
        if workspace is None:
            workspace = _workspace(lib.rdf2v_selective_scan_workspace_size(s.c), dev)
        st = lib.rdf2v_selective_scan(s.c, *s.views, _ptr(state), _ptr(out), _ptr(state_out), _ptr(workspace),
                                      _ws_bytes(workspace), _ptr(status), h)
        _check(st, "rdf2v_selective_scan")
        _written_of(*given)
        return out, state_out


def rdf2v_selective_scan_backward(x: torch.Tensor, dt: torch.Tensor, a: torch.Tensor, b: torch.Tensor, c: torch.Tensor,
                                  dout: torch.Tensor, *, dt_bias: torch.Tensor | None = None,
                                  skip: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                                  lens: torch.Tensor | None = None, state: torch.Tensor | None = None,
                                  dstate_out: torch.Tensor | None = None, out: ScanGradients | None = None,
                                  workspace: torch.Tensor | None = None, status: torch.Tensor | None = None,
                                  stream=None) -> ScanGradients:
    """Gradients of rdf2v_selective_scan for its inputs, from dout (that of out) and dstate_out (that of state_out;
    None: zeros), each in its input's shape and type. `out`: tensors to write them to, with None for those of inputs
    that are not given (dstate may be there without a state)."""
    s = _Scan(x, dt, a, b, c, dt_bias, skip, gate, lens, 3)
    dev, kind, f32 = s.dev, s.dtype, torch.float32
    with _on_stream(dev, stream) as h:
        view = _tokens_view(dout, "dout", kind, dev, s.shape)
        given = (None,) * 9 if out is None else out
        channels = (s.c.channels,)
        wanted = ((True, kind, s.shape), (True, kind, s.shape), (True, f32, a.shape), (True, kind, s.heads),
                  (True, kind, s.heads), (dt_bias is not None, f32, channels), (skip is not None, f32, channels),
                  (gate is not None, kind, s.shape), (state is not None, f32, s.states))
        g = ScanGradients(*[_new(t, name, type_, shape, dev) if want or t is not None else None
                            for t, name, (want, type_, shape) in zip(given, ScanGradients._fields, wanted)])
        _state(state, "state", s.states, dev)
        _state(dstate_out, "dstate_out", s.states, dev)
        _status(status, dev)
        lib = _native()
        if workspace is None:
            workspace = _workspace(lib.rdf2v_selective_scan_backward_workspace_size(s.c), dev)
        to = _ScanGradientsStruct(_ptr(g.dx), _ptr(g.ddt), _ptr(g.db), _ptr(g.dc), _ptr(g.dgate), _ptr(g.da),
                                  _ptr(g.ddt_bias), _ptr(g.dskip), _ptr(g.dstate))
        st = lib.rdf2v_selective_scan_backward(s.c, *s.views, view, _ptr(state), _ptr(dstate_out), to,
                                               _ptr(workspace), _ws_bytes(workspace), _ptr(status), h)
        _check(st, "rdf2v_selective_scan_backward")
        _written_of(*given)
        return g


def rdf2v_selective_scan_step(x: torch.Tensor, dt: torch.Tensor, a: torch.Tensor, b: torch.Tensor, c: torch.Tensor,
                              state: torch.Tensor, *, dt_bias: torch.Tensor | None = None,
                              skip: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                              parents: torch.Tensor | None = None, out: torch.Tensor | None = None,
                              state_out: torch.Tensor | None = None, status: torch.Tensor | None = None, stream=None):
    """rdf2v_selective_scan for one more token of each row: x, dt, gate [rows, channels], b, c [rows, groups, states],
    state float32 [num_states, channels, states]. Returns (out [rows, channels], state_out [rows, channels, states]).
    parents and state_out are as in rdf2v_decay_attention_step. For answering: autograd does not record it."""
    s = _Scan(x, dt, a, b, c, dt_bias, skip, gate, None, 2)
    dev = s.dev
    with _on_stream(dev, stream) as h:
        given = out
        num_states = _parents_and_states(parents, state, s.c.rows, s.states[1:], torch.float32, dev)
        out = _new_like(out, "out", x)
        if state_out is None and parents is None:
            state_out = state
        state_out = _new(state_out, "state_out", torch.float32, s.states, dev)
        _status(status, dev)
        if _records(x, dt, a, b, c, dt_bias, skip, gate, state):
            _no_gradient("rdf2v_selective_scan_step", "its inputs")
        st = _native().rdf2v_selective_scan_step(s.c, *s.views, _ptr(state), num_states, _ptr(parents), _ptr(out),
                                                 _ptr(state_out), _ptr(status), h)
        _check(st, "rdf2v_selective_scan_step")
        _written((state_out,) if given is None else (given, state_out))
        return out, state_out


class NormGradients(NamedTuple):
    """Gradients of rdf2v_residual_norm's inputs; None for an input that was not given."""

    dx: torch.Tensor
    dresidual: torch.Tensor | None
    dweight: torch.Tensor
    dbias: torch.Tensor | None
    dscale: torch.Tensor | None


class _Norm:
    """The checked arguments that the residual norm calls share."""

    __slots__ = ("c", "views", "dev", "dtype", "shape", "hidden_dtype", "stats")

    def __init__(self, x, residual, weight, bias, scale, drop, seed, seed_offset, row_begin, center, eps, lens,
                 hidden_dtype):
        dtype = _float_dtype(x, "x")
        shape = self.shape = x.shape
        if len(shape) not in (2, 3):
            raise ValueError("x must have shape [rows, length, channels] or [rows, channels]")
        dev, self.dtype = x.device, x.dtype
        self.dev = dev
        rows, channels = shape[0], shape[-1]
        if not 1 <= channels <= RDF2V_MAX_NORM_CHANNELS:
            raise ValueError(f"{channels} channels: 1 to {RDF2V_MAX_NORM_CHANNELS} are supported")
        if residual is not None:
            hidden_dtype = residual.dtype if isinstance(residual, torch.Tensor) else None
        elif hidden_dtype is None:
            hidden_dtype = x.dtype
        if hidden_dtype not in (x.dtype, torch.float32):
            raise TypeError(f"residual must be {x.dtype} or float32, got {hidden_dtype}")
        if not 0.0 <= drop < 1.0 - 2.0 ** -32:
            raise ValueError(f"drop must be in [0, 1), got {drop}")
        if not 0 <= row_begin < 1 << 63:
            raise ValueError("row_begin must be in [0, 2^63)")
        self.hidden_dtype = hidden_dtype
        self.views = (_tokens_view(x, "x", x.dtype, dev, shape),
                      None if residual is None else _tokens_view(residual, "residual", hidden_dtype, dev, shape))
        self.stats = (*shape[:-1], 2)
        if weight is None:
            raise TypeError("weight must be a CUDA (HIP) tensor")
        if seed_offset is not None:
            seed_offset = _out(seed_offset, "seed_offset", torch.int64, 1, dev).data_ptr()
        each = (channels,)
        self.c = _NormStruct(rows, shape[1] if len(shape) == 3 else 1, channels, dtype, _DTYPES[hidden_dtype],
                             bool(center), eps, _parameter(weight, "weight", each, dev),
                             _parameter(bias, "bias", each, dev), _parameter(scale, "scale", each, dev), drop,
                             seed & 0xFFFFFFFFFFFFFFFF, seed_offset, row_begin, _lens(lens, rows, dev))


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, bias, scale, seed_offset, lens, given, status, stream):
        out, hidden, stats = rdf2v_residual_norm(x, residual, weight, bias, scale=scale, seed_offset=seed_offset,
                                                 lens=lens, status=status, stream=stream, **given)
        ctx.moved = stream is not None
        ctx.save_for_backward(x, residual, weight, bias, scale, seed_offset, lens, stats)
        ctx.given = given
        ctx.hidden_dtype = hidden.dtype
        ctx.mark_non_differentiable(stats)
        ctx.set_materialize_grads(False)
        return out, hidden, stats

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dhidden, _):
        x, residual, weight, bias, scale, seed_offset, lens, stats = _saved(ctx)
        if dhidden is not None:
            dhidden = _gradient(dhidden, None)
        g = rdf2v_residual_norm_backward(x, residual, weight, bias, stats, _gradient(dout, (x.shape, x.dtype, x.device)),
                                         dhidden=dhidden, scale=scale, seed_offset=seed_offset, lens=lens, **ctx.given)
        return g.dx, g.dresidual, g.dweight, g.dbias, g.dscale, None, None, None, None, None


def rdf2v_residual_norm(x: torch.Tensor, residual: torch.Tensor | None, weight: torch.Tensor,
                        bias: torch.Tensor | None = None, *, scale: torch.Tensor | None = None, drop: float = 0.0,
                        seed: int = 0, seed_offset: torch.Tensor | None = None, row_begin: int = 0,
                        center: bool = False, eps: float = 1e-5, lens: torch.Tensor | None = None,
                        hidden_dtype: torch.dtype | None = None, out: torch.Tensor | None = None,
                        hidden: torch.Tensor | None = None, stats: torch.Tensor | None = None,
                        status: torch.Tensor | None = None, stream=None):
    """Residual connection and norm of each token: hidden = residual + scale * dropout(x), out = weight * (hidden -
    mean) / sqrt(mean of (hidden - mean)^2 + eps) + bias, the mean being taken off only where center is set.

    x [rows, length, channels] (or [rows, channels]) is float32 or bfloat16, residual the same or float32, in any layout
    whose last dimension is contiguous; None stands for zeros, and hidden is of residual's type (hidden_dtype, or x's,
    without one). weight, bias and scale [channels] are float32. lens: int32 [rows], the tokens of each row that count.
    Returns (out, hidden, stats): stats, float32 [..., 2], is for the backward call.

    A share `drop` of x's values is dropped, by random words of (seed + seed_offset; row_begin + row, token, channel)
    that are made where they are needed: nothing is stored, and the backward call, given the same, drops the same.
    seed_offset: int64 [1] on the device, read by the kernels, so that a captured graph draws new masks when it is
    changed.

    Where an input requires gradients, autograd records out and hidden; they must then be left to the call, as in
    torch's own functions."""
    n = _Norm(x, residual, weight, bias, scale, drop, seed, seed_offset, row_begin, center, eps, lens, hidden_dtype)
    dev = n.dev
    if _records(x, residual, weight, bias, scale):
        if out is not None or hidden is not None or stats is not None:
            raise ValueError("out, hidden and stats cannot be given where autograd records the call: an input requires "
                             "gradients")
        given = dict(drop=drop, seed=seed, row_begin=row_begin, center=center, eps=eps, hidden_dtype=hidden_dtype)
        return _recorded(_ResidualNorm, dev, stream, x, residual, weight, bias, scale, seed_offset, lens, given, status,
                         stream)
    with _on_stream(dev, stream) as h:
        given = out, hidden, stats
        out = _new_like(out, "out", x)
        hidden = _new_like(hidden, "hidden", x, n.hidden_dtype)
        stats = _new(stats, "stats", torch.float32, n.stats, dev)
        _status(status, dev)
        st = _native().rdf2v_residual_norm(n.c, *n.views, _ptr(out), _ptr(hidden), _ptr(stats), _ptr(status), h)
        _check(st, "rdf2v_residual_norm")
        _written_of(*given)
        return out, hidden, stats


def rdf2v_residual_norm_backward_workspace_size(rows: int, length: int, channels: int,
                                                dtype: torch.dtype = torch.float32,
                                                hidden_dtype: torch.dtype | None = None) -> int:
    c = _NormStruct(rows, length, channels, _DTYPES.get(dtype, -1), _DTYPES.get(hidden_dtype or dtype, -1))
    return int(_native().rdf2v_residual_norm_backward_workspace_size(c))


def rdf2v_residual_norm_backward(x: torch.Tensor, residual: torch.Tensor | None, weight: torch.Tensor,
                                 bias: torch.Tensor | None, stats: torch.Tensor, dout: torch.Tensor, *,
                                 dhidden: torch.Tensor | None = None, scale: torch.Tensor | None = None,
                                 drop: float = 0.0, seed: int = 0, seed_offset: torch.Tensor | None = None,
                                 row_begin: int = 0, center: bool = False, eps: float = 1e-5,
                                 lens: torch.Tensor | None = None, hidden_dtype: torch.dtype | None = None,
                                 out: NormGradients | None = None, workspace: torch.Tensor | None = None,
                                 status: torch.Tensor | None = None, stream=None) -> NormGradients:
    """Gradients of rdf2v_residual_norm for its inputs, from dout (that of out), dhidden (that of hidden; None: zeros)
    and the stats that it returned; the other arguments as there. `out`: tensors to write them to, with None for those
    of inputs that are not given."""
    n = _Norm(x, residual, weight, bias, scale, drop, seed, seed_offset, row_begin, center, eps, lens, hidden_dtype)
    dev, f32, each = n.dev, torch.float32, weight.shape
    with _on_stream(dev, stream) as h:
        views = (_tokens_view(dout, "dout", n.dtype, dev, n.shape),
                 None if dhidden is None else _tokens_view(dhidden, "dhidden", n.hidden_dtype, dev, n.shape))
        _exact(stats, "stats", f32, n.stats, dev)
        given = (None,) * 5 if out is None else out
        wanted = ((True, n.dtype, n.shape), (residual is not None, n.hidden_dtype, n.shape), (True, f32, each),
                  (bias is not None, f32, each), (scale is not None, f32, each))
        g = NormGradients(*[_new(t, name, type_, shape, dev) if want or t is not None else None
                            for t, name, (want, type_, shape) in zip(given, NormGradients._fields, wanted)])
        _status(status, dev)
        lib = _native()
        if workspace is None:
            workspace = _workspace(lib.rdf2v_residual_norm_backward_workspace_size(n.c), dev)
        st = lib.rdf2v_residual_norm_backward(n.c, *n.views, _ptr(stats), *views, _ptr(g.dx), _ptr(g.dresidual),
                                              _ptr(g.dweight), _ptr(g.dbias), _ptr(g.dscale), _ptr(workspace),
                                              _ws_bytes(workspace), _ptr(status), h)
        _check(st, "rdf2v_residual_norm_backward")
        _written_of(*given)
        return g


def check_device_status(status: torch.Tensor, where: str = "device", stream=None) -> None:
    """Raise if a device status word (zeroed before the calls) has any bit set. The word is read
    on `stream` (default: the current stream), so pass the stream the calls were made on."""
    with _on_stream(status.device, stream):
        v = int(status.item())
    if v != 0:
        bits = [n for b, n in [(RDF2V_STATUS_ID_OUT_OF_RANGE, "ID_OUT_OF_RANGE"),
                               (RDF2V_STATUS_BAD_CSR, "BAD_CSR"), (RDF2V_STATUS_BAD_LENGTH, "BAD_LENGTH"),
                               (RDF2V_STATUS_CAPACITY, "CAPACITY"), (RDF2V_STATUS_BAD_VALUE, "BAD_VALUE")]
                if v & b]
        raise Rdf2vError(RDF2V_ERR_ID_OUT_OF_RANGE, f"{where}: status bits {'|'.join(bits) or v}")
