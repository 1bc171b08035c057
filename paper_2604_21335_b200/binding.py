"""ctypes binding of libstc.so: argument marshalling only.

Every function takes CUDA tensors, checks dtype / contiguity / device, and
passes ``data_ptr()`` plus the current stream to the C-ABI call of the same
name.  No step of the method runs in Python, and there is no CPU fallback: if
the shared library is missing the import of the library fails loudly.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import struct
import sysconfig
from dataclasses import dataclass
from pathlib import Path
from typing import Optional

import torch

_PKG = Path(__file__).resolve().parent
_LIB_PATH = _PKG / "libstc.so"

OP_QUEST_SELECT, OP_ROUTE_PACK, OP_DECODE_ATTN, OP_PREFIX_ATTN, OP_TREE_ATTN = 1, 2, 3, 4, 5
MODE_GLOBAL, MODE_PER_TOKEN = 0, 1
CLS_DROP, CLS_ROUTED, CLS_FULL = 0, 1, 2
ROPE_NONE, ROPE_LINEAR, ROPE_BANDS, ROPE_YARN = 0, 1, 2, 3
STC_OK = 0
STATIC_SCRATCH_BYTES = 8 << 20

EXPORTS = (
    "stc_status_string", "stc_version", "stc_workspace_bytes", "stc_build_page_meta",
    "stc_quest_select", "stc_route_pack", "stc_decode_attn", "stc_cache_bytes",
    "stc_pass_host_arena_bytes", "stc_pass_host", "stc_quest_select_static", "stc_route_mask", "stc_pack_values", "stc_append_tokens", "stc_router_logits", "stc_query_bias", "stc_quest_select_window", "stc_pages_to_class", "stc_route_new_pages", "stc_decode_step", "stc_decode_step_host_arena_bytes", "stc_decode_step_host",
    "stc_rope_frequencies", "stc_rope_write", "stc_decode_attn_scored", "stc_prefix_attn",
    "stc_tree_attn", "stc_tree_accept", "stc_tree_commit", "stc_cache_fork", "stc_cache_compact",
)


class StcError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = load_library().stc_status_string(code).decode()
        super().__init__(f"{where}: {msg} (status {code})")


class _Shape(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("page_size", C.c_int32), ("n_groups", C.c_int32),
                ("t_cap", C.c_int32), ("reserved", C.c_int32), ("seq_len", C.c_void_p)]


class _Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("kmin", C.c_void_p), ("kmax", C.c_void_p),
                ("v_packed", C.c_void_p), ("v_mask", C.c_void_p), ("v_offs", C.c_void_p),
                ("cap_groups", C.c_int64)]


class _Score(C.Structure):
    _fields_ = [("softcap", C.c_float), ("window", C.c_int32), ("slopes", C.c_void_p), ("q_pos", C.c_void_p),
                ("tok_doc", C.c_void_p), ("q_doc", C.c_void_p)]


class _Rope(C.Structure):
    _fields_ = [("inv_freq", C.c_void_p), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("scale", C.c_float),
                ("reserved", C.c_int32)]


_lib = None


def load_library():
    """Load libstc.so (built in-tree by ``paper_2604_21335_b200.build``)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise ImportError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2604_21335_b200.build` "
                "(nvcc, sm_100a).  There is no fallback implementation.")
        lib = C.CDLL(str(_LIB_PATH))
        lib.stc_status_string.restype = C.c_char_p
        lib.stc_status_string.argtypes = [C.c_int32]
        lib.stc_version.restype = C.c_int32
        for name in EXPORTS[2:]:
            getattr(lib, name).restype = C.c_int32
        lib.stc_workspace_bytes.argtypes = [C.POINTER(_Shape), C.c_int32, C.c_int64, C.POINTER(C.c_size_t)]
        lib.stc_build_page_meta.argtypes = [C.POINTER(_Shape), C.POINTER(_Cache), C.c_int32, C.c_int32, C.c_void_p]
        lib.stc_quest_select.argtypes = [C.POINTER(_Shape), C.POINTER(_Cache), C.c_void_p, C.c_int32, C.c_int32,
                                         C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.stc_quest_select_window.argtypes = [C.POINTER(_Shape), C.POINTER(_Cache), C.c_void_p, C.c_int32, C.c_int32,
                                                C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                                C.c_void_p]
        lib.stc_quest_select_static.argtypes = [C.POINTER(_Shape), C.POINTER(_Cache), C.c_void_p, C.c_int32,
                                                C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.stc_pages_to_class.argtypes = [C.POINTER(_Shape), C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                           C.c_void_p]
        lib.stc_route_pack.argtypes = [C.POINTER(_Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64,
                                       C.c_int32, C.c_int32, C.c_int32, C.POINTER(_Cache), C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.stc_route_mask.argtypes = [C.POINTER(_Shape), C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_int32,
                                       C.c_int32, C.POINTER(_Cache), C.c_void_p, C.c_size_t, C.c_void_p]
        lib.stc_pack_values.argtypes = [C.POINTER(_Shape), C.c_void_p, C.c_int32, C.POINTER(_Cache), C.c_void_p,
                                        C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.stc_append_tokens.argtypes = [C.POINTER(_Shape), C.POINTER(_Cache), C.c_void_p, C.c_void_p, C.c_int32,
                                          C.c_void_p, C.c_void_p, C.c_void_p]
        lib.stc_route_new_pages.argtypes = [C.POINTER(_Shape), C.POINTER(_Cache), C.c_void_p, C.c_void_p, C.c_int32,
                                            C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.stc_query_bias.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.stc_router_logits.argtypes = [C.POINTER(_Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                          C.c_void_p, C.c_void_p, C.c_void_p]
        lib.stc_decode_attn.argtypes = [C.POINTER(_Shape), C.POINTER(_Cache), C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_int32, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                        C.c_void_p]
        # (structures of these calls: C.byref of the ctypes ones, or their bytes)
        lib.stc_decode_attn_scored.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                               C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                               C.c_void_p]
        lib.stc_prefix_attn.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                        C.c_void_p]
        lib.stc_tree_attn.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                      C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                      C.c_void_p]
        lib.stc_tree_accept.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.stc_tree_commit.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_void_p]
        lib.stc_cache_fork.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.stc_cache_compact.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.stc_rope_frequencies.argtypes = [C.c_int32, C.c_double, C.c_int32, C.c_double, C.c_double, C.c_double,
                                             C.c_double, C.c_void_p, C.c_void_p]
        lib.stc_rope_write.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                       C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                       C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.stc_decode_step.argtypes = [C.POINTER(_Shape), C.POINTER(_Cache), C.c_void_p, C.c_int32, C.c_int32,
                                        C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_size_t, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.stc_cache_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        lib.stc_pass_host_arena_bytes.argtypes = [C.POINTER(_Shape), C.c_int64, C.c_int32, C.POINTER(C.c_size_t)]
        lib.stc_pass_host.argtypes = [C.POINTER(_Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_int64,
                                      C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.stc_decode_step_host_arena_bytes.argtypes = [C.POINTER(_Shape), C.c_int32, C.POINTER(C.c_size_t)]
        lib.stc_decode_step_host.argtypes = [C.POINTER(_Shape), C.POINTER(_Cache), C.c_void_p, C.c_int32, C.c_float,
                                             C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p]
        _lib = lib
        if _native_addresses is None:            # built since the import
            _take_native()
    return _lib


def _ptr(t: Optional[torch.Tensor], dtype=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream() -> int:
    return _raw_stream(_current_device())


# The current device and its current stream without the objects torch.cuda wraps around them: a decode step's calls
# take a few microseconds on the device, and the host's share of them is this module.
# (the tensors of a call have initialised CUDA)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)


def _at(t: Optional[torch.Tensor], dtype, device: int, name: str) -> int:
    """Address of a contiguous tensor of `dtype` on CUDA device `device`; 0 for None."""
    if t is None:
        return 0
    if t.get_device() == device and t.dtype is dtype and t.is_contiguous():
        return t.data_ptr()
    if t.is_cuda and t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, but the current device is cuda:{device}")
    return _ptr(t, dtype, name)


def args_library() -> Path:
    """Where the native argument check stands: it reads tensors by torch's own headers, so its name holds the versions of the torch
    and the Python it was built for, and another one's is not found."""
    return _PKG / f"_tensor_args.torch-{torch.__version__}{sysconfig.get_config_var('EXT_SUFFIX')}"


def _native_module():
    """The argument check built for this torch and this Python, or None: the same checks in Python."""
    path = args_library()
    if not path.exists():
        return None
    spec = importlib.util.spec_from_file_location(__package__ + "._tensor_args", path)
    try:
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError:
        return None
    return module


def _take_native() -> None:
    global _native_addresses, _sizes_are, _native_token_rows
    m = _native_module()
    _native_addresses, _sizes_are, _native_token_rows = (m.addresses, m.sizes_are, m.token_rows) if m else (None, None, None)


_take_native()
_CODES = {"b": torch.bfloat16, "f": torch.float32, "d": torch.float64, "i": torch.int32, "l": torch.int64, "u": torch.uint8}


def _addresses(device: int, codes: str, names: tuple, *tensors) -> tuple:
    """Address of each tensor (0 for None), checked to be a contiguous one of type codes[i] ('*': any) on CUDA `device`."""
    got = _native_addresses(device, codes, *tensors) if _native_addresses is not None else None
    if got is None:                              # something is wrong: find it and say what
        got = tuple(_at(t, _CODES[c] if c != "*" else None if t is None else t.dtype, device, n)
                    for t, c, n in zip(tensors, codes, names))
    return got


# Structures as the bytes the library reads (native layout of stc_shape, stc_cache, stc_score, stc_rope, stc_tree).
_PACK_SHAPE = struct.Struct("8iP").pack
_PACK_CACHE = struct.Struct("6Pq").pack
_PACK_SCORE = struct.Struct("fi4P").pack
_PACK_ROPE = struct.Struct("Piifi").pack
_PACK_TREE = struct.Struct("4Pii").pack


@dataclass
class Shape:
    batch: int
    n_q_heads: int
    n_kv_heads: int
    n_groups: int
    t_cap: int
    seq_len: Optional[torch.Tensor] = None   # int32 [batch] on the device, or None
    head_dim: int = 128
    page_size: int = 16

    @property
    def n_pages(self) -> int:
        return (self.t_cap + self.page_size - 1) // self.page_size

    @property
    def n_problems(self) -> int:
        return self.batch * self.n_kv_heads

    def c(self) -> _Shape:
        sl = _ptr(self.seq_len, torch.int32, "seq_len")
        return _Shape(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.page_size,
                      self.n_groups, self.t_cap, 0, sl)


@dataclass
class Cache:
    k: Optional[torch.Tensor] = None          # bf16 [B,Hkv,T,128]
    kmin: Optional[torch.Tensor] = None       # bf16 [B,Hkv,P,128]
    kmax: Optional[torch.Tensor] = None
    v_packed: Optional[torch.Tensor] = None   # bf16 [B,Hkv,cap_groups,128/S]
    v_mask: Optional[torch.Tensor] = None     # int16/uint16 [B,Hkv,T]
    v_offs: Optional[torch.Tensor] = None     # int32/uint32 [B,Hkv,T+1]
    cap_groups: int = 0

    def c(self) -> _Cache:
        return _Cache(_ptr(self.k, torch.bfloat16, "k"), _ptr(self.kmin, torch.bfloat16, "kmin"),
                      _ptr(self.kmax, torch.bfloat16, "kmax"), _ptr(self.v_packed, torch.bfloat16, "v_packed"),
                      _ptr(self.v_mask, None, "v_mask"), _ptr(self.v_offs, None, "v_offs"), self.cap_groups)

    @staticmethod
    def allocate(shape: Shape, k: torch.Tensor, cap_groups: int) -> "Cache":
        """Device buffers for the metadata and the packed store (torch owns the memory)."""
        dev = k.device
        B, H, T, P = shape.batch, shape.n_kv_heads, shape.t_cap, shape.n_pages
        g = shape.head_dim // shape.n_groups
        return Cache(
            k=k,
            kmin=torch.empty(B, H, P, shape.head_dim, dtype=torch.bfloat16, device=dev),
            kmax=torch.empty(B, H, P, shape.head_dim, dtype=torch.bfloat16, device=dev),
            v_packed=torch.empty(B, H, max(cap_groups, 1), g, dtype=torch.bfloat16, device=dev),
            v_mask=torch.zeros(B, H, T, dtype=torch.int16, device=dev),
            v_offs=torch.zeros(B, H, T + 1, dtype=torch.int32, device=dev),
            cap_groups=cap_groups)


@dataclass
class Score:
    """Options on the scores of decode_attn (stc_score): cap, window, distance slopes, document mask."""
    softcap: float = 0.0
    slopes: Optional[torch.Tensor] = None     # f32 [Hq]
    q_pos: Optional[torch.Tensor] = None      # i32, one per query row
    window: int = 0
    tok_doc: Optional[torch.Tensor] = None    # i32 [B, T]
    q_doc: Optional[torch.Tensor] = None      # i32, one per query row

    def check(self, shape: Shape, rows: int) -> None:
        _sizes(("slopes", "q_pos", "tok_doc", "q_doc"), self.slopes, (shape.n_q_heads,), self.q_pos, (rows,), self.tok_doc,
               (shape.batch, shape.t_cap), self.q_doc, (rows,))


@dataclass
class Rope:
    """Rotary table (stc_rope): inv_freq f64 [rot_dim/2] on the device, radians per position."""
    inv_freq: torch.Tensor
    interleaved: bool = False
    scale: float = 1.0


@dataclass
class Tree:
    """Drafted tokens (stc_tree): their keys and values, and the node each continues (None: a chain)."""
    k: torch.Tensor                           # bf16 [B,Hkv,n,128]
    v: torch.Tensor
    parent: Optional[torch.Tensor] = None     # i32 [B,n], parent[i] < i, -1 = the cached sequence
    n_nodes: Optional[torch.Tensor] = None    # i32 [B], None = n for all


def _sizes(names: tuple, *pairs) -> None:
    """Checks tensor, size, tensor, size, ..."""
    if _sizes_are is not None and _sizes_are(*pairs):
        return
    for i, name in enumerate(names):
        _sized(pairs[2 * i], pairs[2 * i + 1], name)


def _sized(t: Optional[torch.Tensor], size: tuple, name: str) -> None:
    if t is not None and t.shape != size:
        raise ValueError(f"{name} must have shape {size}, got {tuple(t.shape)}")


def _token_rows(t: Optional[torch.Tensor], B: int, n: int, heads: int, dim: int, device: int, name: str):
    """(address, elements from token to token) of rows [B, n, heads, dim] that may be a slice of wider token rows."""
    if t is None:
        return 0, 0
    got = _native_token_rows(device, t, B, n, heads, dim) if _native_token_rows is not None else None
    if got is not None:
        return got
    if t.get_device() != device or t.dtype is not torch.bfloat16:
        raise ValueError(f"{name} must be a tensor of torch.bfloat16 on cuda:{device}, got {t.dtype} on {t.device}")
    if t.shape != (B, n, heads, dim):
        raise ValueError(f"{name} must have shape {(B, n, heads, dim)}, got {tuple(t.shape)}")
    at, width = t.data_ptr(), heads * dim
    if B == 0 or n == 0:
        return at, width
    sb, sn, sh, sd = t.stride()
    step = sn if n > 1 else sb if B > 1 else width
    if sd != 1 or (heads > 1 and sh != dim) or (B > 1 and sb != n * step):
        raise ValueError(f"{name}: a token's rows must be contiguous and tokens equally spaced, got strides {t.stride()}")
    return at, step


def _check(rc: int, where: str):
    if rc != STC_OK:
        raise StcError(rc, where)


def workspace_bytes(shape: Shape, op: int, arg: int = 0) -> int:
    out = C.c_size_t(0)
    cs = shape.c()
    _check(load_library().stc_workspace_bytes(C.byref(cs), op, arg, C.byref(out)), "stc_workspace_bytes")
    return int(out.value)


def new_workspace(shape: Shape, op: int, arg: int = 0, device="cuda") -> torch.Tensor:
    n = workspace_bytes(shape, op, arg)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def build_page_meta(shape: Shape, cache: Cache, page_begin: int = 0, page_end: int = -1) -> None:
    cs, cc = shape.c(), cache.c()
    _check(load_library().stc_build_page_meta(C.byref(cs), C.byref(cc), page_begin, page_end, _stream()),
           "stc_build_page_meta")


def quest_select(shape: Shape, cache: Cache, q: torch.Tensor, token_budget: int, page_ids: torch.Tensor,
                 n_pages: torch.Tensor, ws: torch.Tensor, scores: Optional[torch.Tensor] = None,
                 n_recent_pages: int = 0) -> None:
    """n_recent_pages > 0 keeps that many most recent pages unconditionally (stc_quest_select_window)."""
    cs, cc = shape.c(), cache.c()
    if n_recent_pages:
        _check(load_library().stc_quest_select_window(
            C.byref(cs), C.byref(cc), _ptr(q, torch.bfloat16, "q"), token_budget, n_recent_pages,
            page_ids.shape[-1], _ptr(page_ids, torch.int32, "page_ids"), _ptr(n_pages, torch.int32, "n_pages"),
            _ptr(scores, torch.float32, "scores"), _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream()),
            "stc_quest_select_window")
        return
    _check(load_library().stc_quest_select(
        C.byref(cs), C.byref(cc), _ptr(q, torch.bfloat16, "q"), token_budget, page_ids.shape[-1],
        _ptr(page_ids, torch.int32, "page_ids"), _ptr(n_pages, torch.int32, "n_pages"),
        _ptr(scores, torch.float32, "scores"), _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream()),
        "stc_quest_select")


def quest_select_static(shape: Shape, cache: Cache, q: torch.Tensor, token_budget: int, page_ids: torch.Tensor,
                        n_pages: torch.Tensor, scores: Optional[torch.Tensor] = None) -> None:
    """stc_quest_select without a workspace argument: for callers that cannot
    allocate device memory where they select pages.  The scratch space is an array
    inside the library (STATIC_SCRATCH_BYTES per GPU); larger shapes raise StcError
    with code 8.  Calls must not overlap on the device."""
    cs, cc = shape.c(), cache.c()
    _check(load_library().stc_quest_select_static(
        C.byref(cs), C.byref(cc), _ptr(q, torch.bfloat16, "q"), token_budget, page_ids.shape[-1],
        _ptr(page_ids, torch.int32, "page_ids"), _ptr(n_pages, torch.int32, "n_pages"),
        _ptr(scores, torch.float32, "scores"), _stream()), "stc_quest_select_static")


def pages_to_class(shape: Shape, page_ids: torch.Tensor, n_pages: torch.Tensor, tok_class: torch.Tensor) -> None:
    """tok_class u8 [B,Hkv,T] <- ROUTED for the valid tokens of the listed pages, DROP elsewhere."""
    cs = shape.c()
    _check(load_library().stc_pages_to_class(
        C.byref(cs), _ptr(page_ids, torch.int32, "page_ids"), _ptr(n_pages, torch.int32, "n_pages"),
        page_ids.shape[-1], _ptr(tok_class, torch.uint8, "tok_class"), _stream()), "stc_pages_to_class")


def route_pack(shape: Shape, v: torch.Tensor, scores: torch.Tensor, tok_class: Optional[torch.Tensor],
               k_nominal: int, cache: Cache, total_groups: torch.Tensor, status: torch.Tensor,
               ws: torch.Tensor, min_per_token: int = 1, mode: int = MODE_GLOBAL) -> None:
    stride = 0
    if tok_class is not None and tok_class.dim() == 3:
        stride = shape.t_cap
    cs, cc = shape.c(), cache.c()
    _check(load_library().stc_route_pack(
        C.byref(cs), _ptr(v, torch.bfloat16, "v"), _ptr(scores, torch.float32, "scores"),
        _ptr(tok_class, torch.uint8, "tok_class"), stride, k_nominal, min_per_token, mode, C.byref(cc),
        _ptr(total_groups, torch.int64, "total_groups"), _ptr(status, torch.int32, "status"),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream()), "stc_route_pack")


def route_mask(shape: Shape, scores: torch.Tensor, tok_class: Optional[torch.Tensor], k_nominal: int,
               cache: Cache, ws: torch.Tensor, min_per_token: int = 1, mode: int = MODE_GLOBAL) -> None:
    """First half of route_pack: the routing masks (ties at the threshold are left in `ws`)."""
    stride = shape.t_cap if (tok_class is not None and tok_class.dim() == 3) else 0
    cs, cc = shape.c(), cache.c()
    _check(load_library().stc_route_mask(
        C.byref(cs), _ptr(scores, torch.float32, "scores"), _ptr(tok_class, torch.uint8, "tok_class"), stride,
        k_nominal, min_per_token, mode, C.byref(cc), _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream()),
        "stc_route_mask")


def pack_values(shape: Shape, v: torch.Tensor, cache: Cache, total_groups: torch.Tensor, status: torch.Tensor,
                ws: torch.Tensor, mode: int = MODE_GLOBAL) -> None:
    """Second half of route_pack: final masks, offsets and the packed value store."""
    cs, cc = shape.c(), cache.c()
    _check(load_library().stc_pack_values(
        C.byref(cs), _ptr(v, torch.bfloat16, "v"), mode, C.byref(cc),
        _ptr(total_groups, torch.int64, "total_groups"), _ptr(status, torch.int32, "status"),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream()), "stc_pack_values")


def append_tokens(shape: Shape, cache: Cache, v: torch.Tensor, old_len: torch.Tensor, max_new: int,
                  total_groups: torch.Tensor, status: torch.Tensor) -> None:
    """Tokens old_len[b] .. shape.seq_len[b] were just added: store their values in full, refresh page metadata."""
    cs, cc = shape.c(), cache.c()
    _check(load_library().stc_append_tokens(
        C.byref(cs), C.byref(cc), _ptr(v, torch.bfloat16, "v"), _ptr(old_len, torch.int32, "old_len"), max_new,
        _ptr(total_groups, torch.int64, "total_groups"), _ptr(status, torch.int32, "status"), _stream()),
        "stc_append_tokens")


def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: int = ROPE_NONE, factor: float = 1.0,
                     original_len: float = 0.0, low: float = 1.0, high: float = 0.0):
    """(inv_freq f64 [rot_dim/2] on the host, scale) of a rotary table; high 0 = 4 for ROPE_BANDS, 32 for ROPE_YARN."""
    if not high:
        high = 32.0 if scaling == ROPE_YARN else 4.0
    inv_freq = torch.zeros(max(rot_dim, 0) // 2, dtype=torch.float64)
    scale = C.c_float(1.0)
    _check(load_library().stc_rope_frequencies(rot_dim, base, scaling, factor, original_len, low, high,
                                               C.c_void_p(inv_freq.data_ptr() or 1), C.byref(scale)),
           "stc_rope_frequencies")
    return inv_freq, float(scale.value)


_ROPE_NAMES = ("seq_len", "inv_freq", "old_len", "positions", "q_out", "k", "v", "status")


def rope_write(shape: Shape, rope: Rope, old_len: torch.Tensor, status: torch.Tensor,
               q_in: Optional[torch.Tensor] = None, k_in: Optional[torch.Tensor] = None,
               v_in: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
               positions: Optional[torch.Tensor] = None) -> None:
    """Rotates q and k of the tokens old_len[b] .. shape.seq_len[b] and writes them, and v, where the cache wants them.

    q_in / k_in / v_in [B, n, heads, 128] (slices of one fused projection allowed) -> q_out [B, n, Hq, 128],
    k, v [B, Hkv, T, 128]; n is the most new tokens of a sequence; positions i32 [B, n] or None (= cache index)."""
    B, T, D, Hq, Hkv = shape.batch, shape.t_cap, shape.head_dim, shape.n_q_heads, shape.n_kv_heads
    first = q_in if q_in is not None else k_in if k_in is not None else v_in
    if first is None:
        raise ValueError("rope_write needs at least one of q_in, k_in, v_in")
    n, dev = first.shape[1], _current_device()
    qp, qs = _token_rows(q_in, B, n, Hq, D, dev, "q_in")
    kp, ks = _token_rows(k_in, B, n, Hkv, D, dev, "k_in")
    vp, vs = _token_rows(v_in, B, n, Hkv, D, dev, "v_in")
    cache, per_seq = (B, Hkv, T, D), (B,)
    _sizes(("q_out", "k", "v", "positions", "old_len", "status"), q_out, (B, n, Hq, D), k, cache, v, cache, positions, (B, n),
           old_len, per_seq, status, per_seq)
    lp, fp, op, pp, qo, ko, vo, sp = _addresses(dev, "idiibbbi", _ROPE_NAMES, shape.seq_len, rope.inv_freq, old_len,
                                                positions, q_out, k, v, status)
    rc = load_library().stc_rope_write(
        _PACK_SHAPE(B, Hq, Hkv, D, shape.page_size, shape.n_groups, T, 0, lp),
        _PACK_ROPE(fp, 2 * rope.inv_freq.numel(), int(rope.interleaved), rope.scale, 0), op, n, pp, qp, qs, kp, ks, vp, vs,
        qo, ko, vo, sp, _raw_stream(dev))
    if rc:
        raise StcError(rc, "stc_rope_write")


def route_new_pages(shape: Shape, cache: Cache, scores: torch.Tensor, first_page: torch.Tensor, k_nominal: int,
                    total_groups: torch.Tensor, status: torch.Tensor, min_per_token: int = 1,
                    mode: int = MODE_GLOBAL) -> None:
    """Routes, page by page, the complete pages from first_page[b] on (stored at full width by append_tokens)."""
    cs, cc = shape.c(), cache.c()
    _check(load_library().stc_route_new_pages(
        C.byref(cs), C.byref(cc), _ptr(scores, torch.float32, "scores"), _ptr(first_page, torch.int32, "first_page"),
        k_nominal, min_per_token, mode, _ptr(total_groups, torch.int64, "total_groups"),
        _ptr(status, torch.int32, "status"), _stream()), "stc_route_new_pages")


def router_logits(shape: Shape, h: torch.Tensor, w: torch.Tensor, scores: torch.Tensor, status_word: torch.Tensor,
                  bias: Optional[torch.Tensor] = None) -> None:
    """scores[b,hk,t,j] = h[b,t,:] . w[hk*S+j,:] (+ bias[b,hk*S+j]); h bf16 [B,T,d_model], w bf16 [Hkv*S,d_model]."""
    cs = shape.c()
    _check(load_library().stc_router_logits(
        C.byref(cs), _ptr(h, torch.bfloat16, "h"), _ptr(w, torch.bfloat16, "w"), _ptr(bias, torch.float32, "bias"),
        h.shape[-1], _ptr(scores, torch.float32, "scores"), _ptr(status_word, torch.int32, "status_word"),
        _stream()), "stc_router_logits")


def query_bias(h_q: torch.Tensor, w_q: torch.Tensor, s_q: torch.Tensor, bias: torch.Tensor,
               q_len: Optional[torch.Tensor] = None) -> None:
    """s_q[b,:] = mean of h_q[b,:q_len[b],:]; bias[b,n] = s_q[b,:] . w_q[n,:]; h_q bf16 [B,Lq,d_model], w_q bf16 [N,d_model]."""
    B, Lq, dm = h_q.shape
    _check(load_library().stc_query_bias(
        B, Lq, dm, w_q.shape[0], _ptr(h_q, torch.bfloat16, "h_q"), _ptr(q_len, torch.int32, "q_len"),
        _ptr(w_q, torch.bfloat16, "w_q"), _ptr(s_q, torch.float32, "s_q"), _ptr(bias, torch.float32, "bias"),
        _stream()), "stc_query_bias")


def _list_address(page_ids: Optional[torch.Tensor], address, other):
    """Address of the page lists for the attention calls, where NULL means every page.  Lists of no pages are an empty tensor,
    which has no address: `other` (that of any tensor) stands for it, nothing is read there."""
    return other if page_ids is not None and not address else address


_SCORED_NAMES = ("seq_len", "k", "v_packed", "v_mask", "v_offs", "slopes", "q_pos", "tok_doc", "q_doc", "q", "page_ids",
                 "n_pages", "out", "lse", "ws")


def decode_attn(shape: Shape, cache: Cache, q: torch.Tensor, page_ids: Optional[torch.Tensor],
                n_pages: Optional[torch.Tensor], sm_scale: float, out: torch.Tensor, ws: torch.Tensor,
                lse: Optional[torch.Tensor] = None, score: Optional[Score] = None) -> None:
    """score: capped / biased / windowed / per-document scores (stc_decode_attn_scored)."""
    max_pages = page_ids.shape[-1] if page_ids is not None else shape.n_pages
    if score is not None:
        dev, B, Hq, Hkv = _current_device(), shape.batch, shape.n_q_heads, shape.n_kv_heads
        rows = (B, Hq, shape.head_dim)
        _sizes(("q", "out", "lse", "page_ids", "n_pages"), q, rows, out, rows, lse, (B, Hq), page_ids, (B, Hkv, max_pages),
               n_pages, (B, Hkv))
        score.check(shape, B)
        lp, kp, vp, mp, op, slp, pop, tdp, qdp, qp, ip, np_, outp, lsep, wsp = _addresses(
            dev, "ibb**fiiibiiffu", _SCORED_NAMES, shape.seq_len, cache.k, cache.v_packed, cache.v_mask, cache.v_offs,
            score.slopes, score.q_pos, score.tok_doc, score.q_doc, q, page_ids, n_pages, out, lse, ws)
        ip = _list_address(page_ids, ip, qp)
        rc = load_library().stc_decode_attn_scored(
            _PACK_SHAPE(shape.batch, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.page_size, shape.n_groups,
                        shape.t_cap, 0, lp),
            _PACK_CACHE(kp, 0, 0, vp, mp, op, cache.cap_groups), qp, ip, np_, max_pages, sm_scale,
            _PACK_SCORE(score.softcap, score.window, slp, pop, tdp, qdp), outp, lsep, wsp, ws.numel(), _raw_stream(dev))
        if rc:
            raise StcError(rc, "stc_decode_attn_scored")
        return
    cs, cc = shape.c(), cache.c()
    qp = _ptr(q, torch.bfloat16, "q")
    _check(load_library().stc_decode_attn(
        C.byref(cs), C.byref(cc), qp, _list_address(page_ids, _ptr(page_ids, torch.int32, "page_ids"), qp),
        _ptr(n_pages, torch.int32, "n_pages"), max_pages, sm_scale, _ptr(out, torch.float32, "out"),
        _ptr(lse, torch.float32, "lse"), _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream()),
        "stc_decode_attn")


_PREFIX_NAMES = ("seq_len", "k", "v_packed", "v_mask", "v_offs", "slopes", "q_pos", "tok_doc", "q_doc", "q", "row_start",
                 "own_out", "own_lse", "out", "lse", "ws")
_PLAIN = Score()


def prefix_attn(shape: Shape, cache: Cache, q: torch.Tensor, row_start: torch.Tensor, sm_scale: float, out: torch.Tensor,
                ws: torch.Tensor, lse: Optional[torch.Tensor] = None, score: Optional[Score] = None,
                own_out: Optional[torch.Tensor] = None, own_lse: Optional[torch.Tensor] = None) -> None:
    """Rows row_start[g] .. row_start[g+1] of q [n_rows, Hq, 128] attend prefix g (sequence g of shape / cache), read
    once for all of them; own_out / own_lse (the rows' results over their own tokens) are joined by log-sum-exp."""
    n, Hq, dev = q.shape[0], shape.n_q_heads, _current_device()
    rows, heads = (n, Hq, shape.head_dim), (n, Hq)
    _sizes(("q", "row_start", "out", "lse", "own_out", "own_lse"), q, rows, row_start, (shape.batch + 1,), out, rows, lse, heads,
           own_out, rows, own_lse, heads)
    co = score if score is not None else _PLAIN
    co.check(shape, n)
    lp, kp, vp, mp, op, slp, pop, tdp, qdp, qp, sp, oop, olp, outp, lsep, wsp = _addresses(
        dev, "ibb**fiiibiffffu", _PREFIX_NAMES, shape.seq_len, cache.k, cache.v_packed, cache.v_mask, cache.v_offs,
        co.slopes, co.q_pos, co.tok_doc, co.q_doc, q, row_start, own_out, own_lse, out, lse, ws)
    rc = load_library().stc_prefix_attn(
        _PACK_SHAPE(shape.batch, Hq, shape.n_kv_heads, shape.head_dim, shape.page_size, shape.n_groups, shape.t_cap, 0, lp),
        _PACK_CACHE(kp, 0, 0, vp, mp, op, cache.cap_groups), n, qp, sp, sm_scale,
        _PACK_SCORE(co.softcap, co.window, slp, pop, tdp, qdp), oop, olp, outp, lsep, wsp, ws.numel(), _raw_stream(dev))
    if rc:
        raise StcError(rc, "stc_prefix_attn")


def _shape_bytes(shape: Shape, seq_len: int) -> bytes:
    return _PACK_SHAPE(shape.batch, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.page_size, shape.n_groups,
                       shape.t_cap, 0, seq_len)


_CACHE_NAMES = ("k", "kmin", "kmax", "v_packed", "v_mask", "v_offs")
_TREE_NAMES = ("seq_len", "k", "v_packed", "v_mask", "v_offs", "tree.k", "tree.v", "tree.parent", "tree.n_nodes", "slopes", "q_pos",
               "tok_doc", "q_doc", "q", "page_ids", "n_pages", "out", "lse", "status", "ws")


def _check_cache(shape: Shape, cache: Cache, what: str = "") -> None:
    """Sizes of a cache's buffers against its shape."""
    B, H, T, P, D = shape.batch, shape.n_kv_heads, shape.t_cap, shape.n_pages, shape.head_dim
    names = _CACHE_NAMES if not what else tuple(f"{what}.{n}" for n in _CACHE_NAMES)
    store = (B, H, cache.cap_groups, D // shape.n_groups)
    if cache.v_packed is not None and cache.cap_groups == 0:          # (allocate() gives an empty store one row)
        store = tuple(cache.v_packed.shape)
    _sizes(names, cache.k, (B, H, T, D), cache.kmin, (B, H, P, D), cache.kmax, (B, H, P, D), cache.v_packed, store,
           cache.v_mask, (B, H, T), cache.v_offs, (B, H, T + 1))
    if cache.v_mask is not None and cache.v_mask.element_size() != 2 or cache.v_offs is not None and cache.v_offs.element_size() != 4:
        raise ValueError("v_mask must hold 16-bit and v_offs 32-bit integers")


def _check_room(what: str, *shapes: Shape) -> None:
    """The library does nothing for a cache of t_cap 0, and says STC_OK: outputs that a caller reads next would be left as they were."""
    if any(s.t_cap == 0 and s.batch > 0 for s in shapes):
        raise ValueError(f"{what} needs caches with room for tokens, got t_cap 0")


def _check_tree(shape: Shape, tree: Tree) -> int:
    n = tree.k.shape[2] if tree.k.dim() == 4 else -1
    rows = (shape.batch, shape.n_kv_heads, n, shape.head_dim)
    _sizes(("tree.k", "tree.v", "tree.parent", "tree.n_nodes"), tree.k, rows, tree.v, rows, tree.parent, (shape.batch, n),
           tree.n_nodes, (shape.batch,))
    return n


def tree_attn(shape: Shape, cache: Cache, tree: Tree, q: torch.Tensor, page_ids: Optional[torch.Tensor],
              n_pages: Optional[torch.Tensor], sm_scale: float, out: torch.Tensor, status: torch.Tensor, ws: torch.Tensor,
              lse: Optional[torch.Tensor] = None, score: Optional[Score] = None) -> None:
    """Every node of every sequence's tree attends the listed pages (None: all) of the sequence and its own ancestors.

    q [B, n, Hq, 128] -> out f32 [B, n, Hq, 128], lse f32 [B, n, Hq]; score.q_pos i32 [B, n] or None (cache length + depth),
    score.q_doc i32 [B]; status i32 [B]."""
    dev, B, Hq, Hkv = _current_device(), shape.batch, shape.n_q_heads, shape.n_kv_heads
    n = _check_tree(shape, tree)
    max_pages = page_ids.shape[-1] if page_ids is not None else shape.n_pages
    rows = (B, n, Hq, shape.head_dim)
    _sizes(("q", "out", "lse", "page_ids", "n_pages", "status"), q, rows, out, rows, lse, (B, n, Hq), page_ids, (B, Hkv, max_pages),
           n_pages, (B, Hkv), status, (B,))
    co = score if score is not None else _PLAIN
    _sizes(("slopes", "q_pos", "tok_doc", "q_doc"), co.slopes, (Hq,), co.q_pos, (B, n), co.tok_doc, (B, shape.t_cap), co.q_doc, (B,))
    lp, kp, vp, mp, op, tkp, tvp, tpp, tnp, slp, pop, tdp, qdp, qp, ip, np_, outp, lsep, stp, wsp = _addresses(
        dev, "ibb**bbiifiiibiiffiu", _TREE_NAMES, shape.seq_len, cache.k, cache.v_packed, cache.v_mask, cache.v_offs, tree.k, tree.v,
        tree.parent, tree.n_nodes, co.slopes, co.q_pos, co.tok_doc, co.q_doc, q, page_ids, n_pages, out, lse, status, ws)
    ip = _list_address(page_ids, ip, qp)
    rc = load_library().stc_tree_attn(
        _shape_bytes(shape, lp), _PACK_CACHE(kp, 0, 0, vp, mp, op, cache.cap_groups), _PACK_TREE(tkp, tvp, tpp, tnp, n, 0), qp, ip, np_,
        max_pages, sm_scale, _PACK_SCORE(co.softcap, co.window, slp, pop, tdp, qdp), outp, lsep, stp, wsp, ws.numel(),
        _raw_stream(dev))
    if rc:
        raise StcError(rc, "stc_tree_attn")


_ACCEPT_NAMES = ("tokens", "parent", "n_nodes", "path", "n_accepted", "next_token")


def tree_accept(logits: torch.Tensor, tokens: torch.Tensor, path: torch.Tensor, n_accepted: torch.Tensor,
                next_token: torch.Tensor, parent: Optional[torch.Tensor] = None, n_nodes: Optional[torch.Tensor] = None) -> None:
    """Greedy verification: follows argmax(logits) from node 0 through the tree while a child holds the chosen token.

    logits bf16 or f32 [B, n, vocab] (a slice of wider rows allowed); tokens, parent, path i32 [B, n]; n_nodes, n_accepted,
    next_token i32 [B]."""
    if logits.dim() != 3 or logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"logits must be bfloat16 or float32 [B, n, vocab], got {logits.dtype} {tuple(logits.shape)}")
    dev, (B, n, V) = _current_device(), logits.shape
    if logits.get_device() != dev:
        raise ValueError(f"logits is on {logits.device}, but the current device is cuda:{dev}")
    sb, sn, sv = logits.stride()
    step = sn if n > 1 else sb if B > 1 else V
    if (V > 1 and sv != 1) or (B > 1 and sb != n * step):
        raise ValueError(f"logits: a row must be contiguous and rows equally spaced, got strides {logits.stride()}")
    _sizes(_ACCEPT_NAMES, tokens, (B, n), parent, (B, n), n_nodes, (B,), path, (B, n), n_accepted, (B,), next_token, (B,))
    tp, pp, np_, hp, ap, xp = _addresses(dev, "iiiiii", _ACCEPT_NAMES, tokens, parent, n_nodes, path, n_accepted, next_token)
    rc = load_library().stc_tree_accept(B, n, V, logits.data_ptr(), int(logits.dtype is torch.float32), step, tp, pp, np_, hp, ap, xp,
                                        _raw_stream(dev))
    if rc:
        raise StcError(rc, "stc_tree_accept")


_COMMIT_NAMES = ("seq_len", *_CACHE_NAMES, "tree.k", "tree.v", "tree.n_nodes", "path", "n_accepted", "new_len", "total_groups", "status")


def tree_commit(shape: Shape, cache: Cache, tree: Tree, path: torch.Tensor, n_accepted: torch.Tensor, new_len: torch.Tensor,
                total_groups: torch.Tensor, status: torch.Tensor) -> None:
    """The accepted nodes path[b, :n_accepted[b]] become the tokens behind shape.seq_len[b] (the lengths before the call), at full
    width, in cache.k and the packed store; new_len i32 [B] receives the lengths.  A cache of t_cap 0 is refused."""
    dev, B, H = _current_device(), shape.batch, shape.n_kv_heads
    n = _check_tree(shape, tree)
    _check_room("tree_commit", shape)
    _check_cache(shape, cache)
    _sizes(("path", "n_accepted", "new_len", "total_groups", "status"), path, (B, n), n_accepted, (B,), new_len, (B,), total_groups,
           (B, H), status, (B, H))
    lp, kp, lo, hi, vp, mp, op, tkp, tvp, tnp, pp, ap, np_, tp, sp = _addresses(
        dev, "ibbbb**bbiiiili", _COMMIT_NAMES, shape.seq_len, cache.k, cache.kmin, cache.kmax, cache.v_packed, cache.v_mask, cache.v_offs,
        tree.k, tree.v, tree.n_nodes, path, n_accepted, new_len, total_groups, status)
    rc = load_library().stc_tree_commit(
        _shape_bytes(shape, lp), _PACK_CACHE(kp, lo, hi, vp, mp, op, cache.cap_groups), _PACK_TREE(tkp, tvp, 0, tnp, n, 0), pp, ap, np_,
        tp, sp, _raw_stream(dev))
    if rc:
        raise StcError(rc, "stc_tree_commit")


_FORK_NAMES = ("seq_len", *("src." + n for n in _CACHE_NAMES), *("dst." + n for n in _CACHE_NAMES), "src_row", "dst_row", "new_len",
               "total_groups", "status")


def cache_fork(src_shape: Shape, src: Cache, dst_shape: Shape, dst: Cache, src_row: torch.Tensor, dst_row: torch.Tensor,
               new_len: torch.Tensor, total_groups: torch.Tensor, status: torch.Tensor) -> None:
    """Copies the sequences src_row[i] of src to the rows dst_row[i] of dst (which may be src); pairs of one source next to each
    other share its reading.  new_len i32 [dst batch], total_groups i64 [dst batch, Hkv], status i32 [pairs, Hkv].  Caches of t_cap 0
    are refused."""
    dev, n, B, H = _current_device(), src_row.shape[0], dst_shape.batch, dst_shape.n_kv_heads
    if n > 0:
        _check_room("cache_fork", src_shape, dst_shape)
    _check_cache(src_shape, src, "src")
    _check_cache(dst_shape, dst, "dst")
    _sizes(("src_row", "dst_row", "new_len", "total_groups", "status"), src_row, (n,), dst_row, (n,), new_len, (B,), total_groups, (B, H),
           status, (n, H))
    at = _addresses(dev, "ibbbb**bbbb**iiili", _FORK_NAMES, src_shape.seq_len, src.k, src.kmin, src.kmax, src.v_packed, src.v_mask,
                    src.v_offs, dst.k, dst.kmin, dst.kmax, dst.v_packed, dst.v_mask, dst.v_offs, src_row, dst_row, new_len, total_groups,
                    status)
    rc = load_library().stc_cache_fork(_shape_bytes(src_shape, at[0]), _PACK_CACHE(*at[1:7], src.cap_groups), _shape_bytes(dst_shape, 0),
                                       _PACK_CACHE(*at[7:13], dst.cap_groups), n, *at[13:], _raw_stream(dev))
    if rc:
        raise StcError(rc, "stc_cache_fork")


_COMPACT_NAMES = ("seq_len", *("src." + n for n in _CACHE_NAMES), *("dst." + n for n in _CACHE_NAMES), "page_ids", "n_pages", "new_len",
                  "total_groups", "status")


def cache_compact(shape: Shape, cache: Cache, page_ids: torch.Tensor, n_pages: torch.Tensor, new_len: torch.Tensor,
                  total_groups: torch.Tensor, status: torch.Tensor, dst_shape: Optional[Shape] = None, dst: Optional[Cache] = None) -> None:
    """Keeps the listed pages of every KV head, closed up, in dst (None: in place).  page_ids i32 [B, Hkv, max], ascending, n_pages
    i32 [B, Hkv], new_len i32 [B], total_groups i64 [B, Hkv], status i32 [B, Hkv].  Caches of t_cap 0 are refused."""
    if (dst is None) != (dst_shape is None):
        raise ValueError("cache_compact needs both dst_shape and dst, or neither")
    to_shape, to = (shape, cache) if dst is None else (dst_shape, dst)
    dev, B, H, most = _current_device(), shape.batch, shape.n_kv_heads, page_ids.shape[-1]
    _check_room("cache_compact", shape, to_shape)
    _check_cache(shape, cache)
    if dst is not None:
        _check_cache(dst_shape, dst, "dst")
    _sizes(("page_ids", "n_pages", "new_len", "total_groups", "status"), page_ids, (B, H, most), n_pages, (B, H), new_len, (B,),
           total_groups, (B, H), status, (B, H))
    at = _addresses(dev, "ibbbb**bbbb**iiili", _COMPACT_NAMES, shape.seq_len, cache.k, cache.kmin, cache.kmax, cache.v_packed, cache.v_mask,
                    cache.v_offs, to.k, to.kmin, to.kmax, to.v_packed, to.v_mask, to.v_offs, page_ids, n_pages, new_len, total_groups,
                    status)
    rc = load_library().stc_cache_compact(_shape_bytes(shape, at[0]), _PACK_CACHE(*at[1:7], cache.cap_groups), at[13], at[14], most,
                                          _shape_bytes(to_shape, 0), _PACK_CACHE(*at[7:13], to.cap_groups), *at[15:], _raw_stream(dev))
    if rc:
        raise StcError(rc, "stc_cache_compact")


def decode_step(shape: Shape, cache: Cache, q: torch.Tensor, token_budget: int, page_ids: torch.Tensor,
                n_pages: torch.Tensor, sm_scale: float, out: torch.Tensor, ws_select: torch.Tensor,
                ws_attn: torch.Tensor, lse: Optional[torch.Tensor] = None) -> None:
    """quest_select + decode_attn as one call (both workspaces cleared up front, the kernels back to back)."""
    cs, cc = shape.c(), cache.c()
    _check(load_library().stc_decode_step(
        C.byref(cs), C.byref(cc), _ptr(q, torch.bfloat16, "q"), token_budget, page_ids.shape[-1],
        _ptr(page_ids, torch.int32, "page_ids"), _ptr(n_pages, torch.int32, "n_pages"), sm_scale,
        _ptr(out, torch.float32, "out"), _ptr(lse, torch.float32, "lse"), _ptr(ws_select, torch.uint8, "ws_select"),
        ws_select.numel(), _ptr(ws_attn, torch.uint8, "ws_attn"), ws_attn.numel(), _stream()), "stc_decode_step")


def cache_bytes(n_tokens_retained: int, n_groups_kept: int, n_groups: int):
    """(key + packed value bytes, mask + offset + page-metadata bytes) of the compressed cache."""
    kv, idx = C.c_int64(0), C.c_int64(0)
    _check(load_library().stc_cache_bytes(n_tokens_retained, n_groups_kept, n_groups, C.byref(kv), C.byref(idx)),
           "stc_cache_bytes")
    return int(kv.value), int(idx.value)


def _hptr(t: Optional[torch.Tensor], dtype, name):
    if t is None:
        return None
    if t.is_cuda or not t.is_contiguous() or t.dtype != dtype:
        raise ValueError(f"{name} must be a contiguous host tensor of {dtype}")
    return C.c_void_p(t.data_ptr())


def pass_host_arena_bytes(shape: Shape, cap_groups: int, token_budget: Optional[int]) -> int:
    out = C.c_size_t(0)
    cs = shape.c()
    _check(load_library().stc_pass_host_arena_bytes(C.byref(cs), cap_groups,
                                                    -1 if token_budget is None else token_budget,
                                                    C.byref(out)), "stc_pass_host_arena_bytes")
    return int(out.value)


def pass_host(shape: Shape, k: torch.Tensor, v: torch.Tensor, scores: torch.Tensor,
              tok_class: Optional[torch.Tensor], q: torch.Tensor, token_budget: Optional[int],
              k_nominal: int, sm_scale: float, cap_groups: int, arena: torch.Tensor, out: torch.Tensor,
              total_groups: torch.Tensor, status: torch.Tensor, min_per_token: int = 1,
              mode: int = MODE_GLOBAL) -> None:
    """Whole pass from (pinned) host tensors; results land in host tensors after a stream sync."""
    cs = shape.c()
    _check(load_library().stc_pass_host(
        C.byref(cs), _hptr(k, torch.bfloat16, "k"), _hptr(v, torch.bfloat16, "v"),
        _hptr(scores, torch.float32, "scores"), _hptr(tok_class, torch.uint8, "tok_class"),
        _hptr(q, torch.bfloat16, "q"), -1 if token_budget is None else token_budget, k_nominal,
        min_per_token, mode, sm_scale, cap_groups, _ptr(arena, torch.uint8, "arena"), arena.numel(),
        _hptr(out, torch.float32, "out"), _hptr(total_groups, torch.int64, "total_groups"),
        _hptr(status, torch.int32, "status"), _stream()), "stc_pass_host")


def decode_step_host_arena_bytes(shape: Shape, token_budget: Optional[int]) -> int:
    out = C.c_size_t(0)
    cs = shape.c()
    _check(load_library().stc_decode_step_host_arena_bytes(
        C.byref(cs), -1 if token_budget is None else token_budget, C.byref(out)), "stc_decode_step_host_arena_bytes")
    return int(out.value)


def decode_step_host(shape: Shape, cache: Cache, q: torch.Tensor, token_budget: Optional[int], sm_scale: float,
                     arena: torch.Tensor, out: torch.Tensor, status: torch.Tensor) -> None:
    """One decode step (page selection + routed attention) on a device-resident cache, query and result in
    (pinned) host tensors; the results are valid after a stream sync."""
    cs, cc = shape.c(), cache.c()
    _check(load_library().stc_decode_step_host(
        C.byref(cs), C.byref(cc), _hptr(q, torch.bfloat16, "q"), -1 if token_budget is None else token_budget,
        sm_scale, _ptr(arena, torch.uint8, "arena"), arena.numel(), _hptr(out, torch.float32, "out"),
        _hptr(status, torch.int32, "status"), _stream()), "stc_decode_step_host")
