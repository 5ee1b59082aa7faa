"""HeadGuard head-masked low-bit image-KV quantizer on MI355X (gfx950).

A thin ctypes binding over libheadguard.so (include/headguard.h): the entry
points keep their C names and only marshal arguments; every step of the
quantizer runs in the library's HIP kernels.  torch is used for device memory
and streams.  There is no fallback: if the library is missing or fails to load
the import raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Dict, Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# HG_LIBRARY may name another build of the same ABI; default: the in-tree build.
LIB_PATH = os.environ.get("HG_LIBRARY") or os.path.join(_HERE, "libheadguard.so")

HG_BASE_MINMAX, HG_BASE_KIVI, HG_BASE_AKVQ = 0, 1, 2
BASES = {"minmax": HG_BASE_MINMAX, "kivi": HG_BASE_KIVI, "akvq": HG_BASE_AKVQ}
STATUS = ("HG_OK", "HG_ERR_NULL", "HG_ERR_SHAPE", "HG_ERR_SPAN", "HG_ERR_BITS", "HG_ERR_BASE",
          "HG_ERR_HEADDIM", "HG_ERR_ALIGN", "HG_ERR_MASK", "HG_ERR_NO_DEVICE", "HG_ERR_HIP",
          "HG_ERR_POINTER", "HG_ERR_VALUE")
for _i, _n in enumerate(STATUS):
    globals()[_n] = _i
HG_MAX_HEADS = 8192  # largest L*H the routing holds (headguard.h)
BUFFERS = ("codes_k", "meta_k", "side_k", "codes_v", "meta_v", "side_v",
           "norm_k", "ret_idx", "ret_k", "ret_v")  # the packed outputs
PACKED = BUFFERS + ("workspace",)  # the fields of hg_packed


class hg_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("L", "B", "H", "T", "D", "img_start", "img_len", "bits", "base",
                 "keys_only", "kivi_group", "retain_permille")]


class hg_sizes(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in BUFFERS] + [("workspace", C.c_uint64),
                                                     ("fake_workspace", C.c_uint64)] + [
        ("n_protected", C.c_int32), ("n_unprot_k", C.c_int32), ("n_unprot_v", C.c_int32),
        ("retain_count", C.c_int32)]


class hg_packed(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in PACKED]


def _struct(name, fields):
    """A ctypes structure of "type: names" lines; hg_rows members are flat
    (data, token stride, head stride)."""
    kinds = {"i32": C.c_int32, "i64": C.c_int64, "u64": C.c_uint64, "f32": C.c_float, "ptr": C.c_void_p}
    out = []
    for f in fields:
        kind, names = f.split(": ")
        for n in names.split():
            if kind == "rows":
                out += [(n, C.c_void_p), (n + "_token_stride", C.c_int64), (n + "_head_stride", C.c_int64)]
            else:
                out.append((n, kinds[kind]))
    return type(name, (C.Structure,), {"_fields_": out})


hg_paged_cache = _struct("hg_paged_cache", ["i32: B H D page_size num_pages max_pages",
                                            "i64: page_stride head_stride token_stride", "ptr: K V block_table"])
hg_rotation = _struct("hg_rotation", ["ptr: cos sin", "i32: max_pos rot_dim interleaved section0 section1 section2"])
hg_append = _struct("hg_append", ["i32: N Hq", "rows: q k v q_out k_out", "ptr: lens cu_new positions"])
hg_prefill = _struct("hg_prefill", ["i32: B Hq H D Nq Nk causal", "f32: scale", "rows: q k v out", "ptr: lse cu_q cu_k"])
hg_decode = _struct("hg_decode", ["i32: Hq", "f32: scale", "rows: q out", "ptr: lse lens starts workspace",
                                  "u64: workspace_bytes"])
hg_cache8 = _struct("hg_cache8", ["i32: B H D page_size num_pages max_pages block_size",
                                  "i64: page_stride head_stride token_stride", "ptr: K V k_scale v_scale bounds block_table"])
hg_decode8 = _struct("hg_decode8", ["i32: Hq", "f32: scale", "rows: q out", "ptr: lse lens starts workspace",
                                    "u64: workspace_bytes", "ptr: blocks", "i32: budget"])
hg_select = _struct("hg_select", ["i32: Hq", "rows: q", "ptr: lens starts blocks", "i32: budget first last", "ptr: workspace",
                                  "u64: workspace_bytes"])
hg_page_pool = _struct("hg_page_pool", ["i32: B page_size num_pages max_pages", "ptr: block_table lens free_pages n_free"])
hg_resize = _struct("hg_resize", ["i32: N", "ptr: targets cu_new slots positions result"])


class HeadGuardError(RuntimeError):
    def __init__(self, status: int, detail: str):
        name = STATUS[status] if 0 <= status < len(STATUS) else f"status {status}"
        super().__init__(f"{name}: {detail}")
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'` "
            "or `python paper_2609_35800_amd/build.py`")
    lib = C.CDLL(LIB_PATH)
    P = C.c_void_p
    lib.hg_packed_sizes.argtypes = [C.POINTER(hg_config), P, C.POINTER(hg_sizes)]
    lib.hg_quantize.argtypes = [C.POINTER(hg_config), P, P, P, C.POINTER(hg_packed), P]
    lib.hg_dequantize.argtypes = [C.POINTER(hg_config), P, C.POINTER(hg_packed), P, P, P]
    lib.hg_select_heads.argtypes = [P, P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, P]
    lib.hg_fake_quantize.argtypes = [C.POINTER(hg_config), P, P, P, P, P, P, C.c_uint64, P]
    lib.hg_head_budget.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
    lib.hg_fake_quantize_noalloc.argtypes = [C.POINTER(hg_config), P, P, P, P, P, P]
    lib.hg_append_kv.argtypes = [C.POINTER(hg_paged_cache), C.POINTER(hg_rotation), C.POINTER(hg_append), P]
    lib.hg_prefill_attention.argtypes = [C.POINTER(hg_prefill), P]
    lib.hg_decode_workspace.argtypes = [C.POINTER(hg_paged_cache), C.c_int32, C.POINTER(C.c_uint64)]
    lib.hg_decode_attention.argtypes = [C.POINTER(hg_paged_cache), C.POINTER(hg_decode), P]
    lib.hg_append_kv8.argtypes = [C.POINTER(hg_cache8), C.POINTER(hg_rotation), C.POINTER(hg_append), P]
    lib.hg_append_kv8_from.argtypes = [C.POINTER(hg_cache8), C.POINTER(hg_rotation), C.POINTER(hg_append), P, P]
    lib.hg_decode8_workspace.argtypes = [C.POINTER(hg_cache8), C.c_int32, C.POINTER(C.c_uint64)]
    lib.hg_decode_attention8.argtypes = [C.POINTER(hg_cache8), C.POINTER(hg_decode8), P]
    lib.hg_select_workspace.argtypes = [C.POINTER(hg_cache8), C.POINTER(C.c_uint64)]
    lib.hg_select_blocks.argtypes = [C.POINTER(hg_cache8), C.POINTER(hg_select), P]
    lib.hg_resize_rows.argtypes = [C.POINTER(hg_page_pool), C.POINTER(hg_resize), P]
    for f in ("hg_append_kv", "hg_prefill_attention", "hg_decode_workspace", "hg_decode_attention", "hg_append_kv8",
              "hg_append_kv8_from", "hg_decode8_workspace", "hg_decode_attention8", "hg_select_workspace", "hg_select_blocks",
              "hg_resize_rows"):
        getattr(lib, f).restype = C.c_int
    for f in ("hg_packed_sizes", "hg_quantize", "hg_dequantize", "hg_select_heads",
              "hg_fake_quantize", "hg_head_budget", "hg_fake_quantize_noalloc"):
        getattr(lib, f).restype = C.c_int
    lib.hg_status_string.argtypes = [C.c_int]
    lib.hg_status_string.restype = C.c_char_p
    lib.hg_last_error.argtypes = []
    lib.hg_last_error.restype = C.c_char_p
    return lib


_lib = _load()


def _packed_call(name: str, before: int, layout: str):
    """A C call whose argument structure is packed into bytes (0.4 us; a ctypes
    structure of 25 fields 1.5): the function, taking addresses, and the packer."""
    f = _lib[name]  # a function object of its own
    f.argtypes, f.restype = [C.c_void_p] * (before + 2), C.c_int
    return f, struct.Struct("@" + layout).pack


# hg_append, hg_prefill and hg_decode; rows are an address and two strides (Pqq)
_append_call, _append_args = _packed_call("hg_append_kv", 2, "ii" + 5 * "Pqq" + "PPP")
_prefill_call, _prefill_args = _packed_call("hg_prefill_attention", 0, "7if" + 4 * "Pqq" + "PPP")
_decode_call, _decode_args = _packed_call("hg_decode_attention", 1, "if" + 2 * "Pqq" + "PPPPQ")
_append8_call, _ = _packed_call("hg_append_kv8_from", 3, "")
_decode8_call, _decode8_args = _packed_call("hg_decode_attention8", 1, "if" + 2 * "Pqq" + "PPPPQPi0P")
_select_call, _select_args = _packed_call("hg_select_blocks", 1, "iPqqPPPiiiPQ")
_resize_call, _resize_args = _packed_call("hg_resize_rows", 1, "iPPPPP")


def library() -> C.CDLL:
    return _lib


# ------------------------------------------------------------ raw C entry points

def hg_status_string(status: int) -> str:
    return _lib.hg_status_string(int(status)).decode()


def hg_last_error() -> str:
    return _lib.hg_last_error().decode()


def _check(status: int) -> None:
    if status != 0:
        raise HeadGuardError(status, hg_last_error())


# Marshalling is what bounds the calls of one layer (its kernels run 4-8 us):
# the mask goes as the address of a bytes copy (0.3 us; ctypes views of the
# array 2.7), the descriptor's fields by position, and the stream as the raw
# handle torch keeps (a Stream object costs four times as much).  Calls of one
# layer: quantize 10.8 -> 6.8 us (4 heads, 1360 tokens), dequantize 14.4 -> 10.4
# (8 heads, 3456 tokens, rotated keys, retention).

def _mask_arg(mask) -> bytes:
    return np.asarray(mask, dtype=np.uint8).tobytes()


def _ptr(t) -> Optional[int]:
    if t is None or isinstance(t, int):
        return t
    return t.data_ptr()  # 0 for a tensor without elements


def _stream(stream) -> Optional[int]:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_config(L, B, H, T, D, img_start, img_len, bits, base, keys_only, kivi_group=32,
                retain_permille=0) -> hg_config:
    if isinstance(base, str):
        base = BASES[base]
    return hg_config(L=L, B=B, H=H, T=T, D=D, img_start=img_start, img_len=img_len, bits=bits,
                     base=base, keys_only=keys_only, kivi_group=kivi_group,
                     retain_permille=retain_permille)


def hg_packed_sizes(cfg: hg_config, protect_mask) -> Dict[str, int]:
    m = _mask_arg(protect_mask)
    out = hg_sizes()
    _check(_lib.hg_packed_sizes(C.byref(cfg), m, C.byref(out)))
    return {n: getattr(out, n) for n, _ in hg_sizes._fields_}


def _packed_struct(packed: Dict[str, torch.Tensor]) -> hg_packed:
    return hg_packed(*map(_ptr, map(packed.get, PACKED)))


def hg_quantize(cfg: hg_config, K: torch.Tensor, V: torch.Tensor, protect_mask,
                packed: Dict[str, torch.Tensor], stream=None) -> None:
    """Enqueue quantize+pack of the image KV of K, V into `packed` buffers."""
    m = _mask_arg(protect_mask)
    pk = _packed_struct(packed)
    _check(_lib.hg_quantize(C.byref(cfg), _ptr(K), _ptr(V), m,
                            C.byref(pk), _stream(stream)))


def hg_dequantize(cfg: hg_config, protect_mask, packed: Dict[str, torch.Tensor],
                  K_out: torch.Tensor, V_out: torch.Tensor, stream=None) -> None:
    """Enqueue reconstruction of the image rows of K_out, V_out."""
    m = _mask_arg(protect_mask)
    pk = _packed_struct(packed)
    _check(_lib.hg_dequantize(C.byref(cfg), m, C.byref(pk),
                              _ptr(K_out), _ptr(V_out), _stream(stream)))


def hg_fake_quantize(cfg: hg_config, K: torch.Tensor, V: torch.Tensor, protect_mask,
                     K_out: torch.Tensor, V_out: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """Enqueue the one-pass quantize-and-reconstruct of the image rows of K, V
    into K_out, V_out (which may be K, V themselves).  `workspace`: a device
    buffer of at least hg_packed_sizes(...)["fake_workspace"] bytes, needed
    with token retention and with whole-sequence KIVI keys longer than one
    workgroup holds (see alloc_fake_workspace)."""
    m = _mask_arg(protect_mask)
    ws = _ptr(workspace)
    nbytes = workspace.numel() * workspace.element_size() if ws is not None else 0
    _check(_lib.hg_fake_quantize(C.byref(cfg), _ptr(K), _ptr(V), m,
                                 _ptr(K_out), _ptr(V_out), ws, nbytes, _stream(stream)))


def hg_fake_quantize_noalloc(cfg: hg_config, K: torch.Tensor, V: torch.Tensor, protect_mask,
                             K_out: torch.Tensor, V_out: torch.Tensor, stream=None) -> None:
    """hg_fake_quantize with its workspace (retention lists, or the
    whole-sequence key exchange area) taken from the library's own device
    array (HG_NOALLOC_SCRATCH_BYTES per GPU): nothing is allocated;
    overlapping calls on one GPU race on that array."""
    m = _mask_arg(protect_mask)
    _check(_lib.hg_fake_quantize_noalloc(C.byref(cfg), _ptr(K), _ptr(V), m,
                                         _ptr(K_out), _ptr(V_out), _stream(stream)))


HG_NOALLOC_SCRATCH_BYTES = 96 << 20  # headguard.h


# ------------------------------------------------------------ allocation helper

def alloc_packed(cfg: hg_config, protect_mask, device="cuda") -> Dict[str, torch.Tensor]:
    """Device buffers of the sizes hg_packed_sizes reports (uint8 tensors),
    the quantize call's workspace included."""
    sz = hg_packed_sizes(cfg, protect_mask)
    return {n: torch.empty(sz[n], dtype=torch.uint8, device=device) for n in PACKED}


def alloc_fake_workspace(cfg: hg_config, protect_mask, device="cuda") -> Optional[torch.Tensor]:
    """The one-pass call's workspace (uint8 tensor), or None when it needs none."""
    n = hg_packed_sizes(cfg, protect_mask)["fake_workspace"]
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


# ------------------------------------------------------------ head selection

def hg_select_heads(g, o, Hkv: int, K: int) -> np.ndarray:
    """Protection mask uint8 [L*Hkv] from per-query-head scores g, o [L][Hq]."""
    g = np.ascontiguousarray(g, dtype=np.float64)
    o = np.ascontiguousarray(o, dtype=np.float64)
    if g.shape != o.shape or g.ndim != 2:
        raise ValueError("g and o must both be [L, Hq]")
    L, Hq = g.shape
    mask = np.zeros(L * Hkv, dtype=np.uint8)
    _check(_lib.hg_select_heads(g.ctypes.data_as(C.c_void_p), o.ctypes.data_as(C.c_void_p),
                                L, Hq, Hkv, int(K), mask.ctypes.data_as(C.c_void_p)))
    return mask


def head_budget(n_kv: int, num: int = 1, den: int = 8) -> int:
    """hg_head_budget: K = round(n_kv * num / den), halves rounded up."""
    out = C.c_int32()
    _check(_lib.hg_head_budget(int(n_kv), int(num), int(den), C.byref(out)))
    return out.value


# ------------------------------------------------------------ attention over the cache
#
# One layer a call.  Operands are BF16 tensors whose last dimension is
# contiguous, any other strides (views of a fused projection); lengths, offsets,
# positions and the block table int32, contiguous, on the GPU.  Shapes and
# types are checked here, since the C calls see addresses only; sizes, strides,
# alignment and overlaps there.

def _rows(t: torch.Tensor, name: str, n: int, heads: int, D: int):
    """data, token stride and head stride of an [n, heads, D] tensor."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{name} is {t.dtype}, not bfloat16")
    if t.shape != (n, heads, D):
        raise ValueError(f"{name} is {tuple(t.shape)}, not {(n, heads, D)}")
    ts, hs, ds = t.stride()
    if ds != 1:
        raise ValueError(f"the channels of {name} are not contiguous")
    return t.data_ptr(), ts, hs


def _array(t: Optional[torch.Tensor], name: str, shape, dtype=torch.int32) -> int:
    """Address of a contiguous tensor; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype:
        raise TypeError(f"{name} is {t.dtype}, not {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} is {tuple(t.shape)}, not {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} is not contiguous")
    return t.data_ptr()


def make_paged_cache(K: torch.Tensor, V: torch.Tensor, block_table: torch.Tensor) -> hg_paged_cache:
    """Descriptor of one layer's pages: K, V [pages, H, page_size, D] (a
    transposed view where tokens come before heads in memory), block_table
    [B, max_pages].  It holds their addresses and keeps them alive.  A layer
    K[l] of the quantizer's cache is B pages of T tokens: its block table is
    arange(B) as a column."""
    if K.dim() != 4 or K.shape != V.shape or any(n != 1 and a != b for n, a, b in zip(K.shape, K.stride(), V.stride())):
        raise ValueError("K and V must both be [pages, H, page_size, D] with the same strides")
    if K.dtype is not torch.bfloat16 or V.dtype is not torch.bfloat16:
        raise TypeError("K and V must be bfloat16")
    if K.stride(3) != 1:
        raise ValueError("the channels of K and V are not contiguous")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    pages, H, page_size, D = K.shape
    table = _array(block_table, "block_table", block_table.shape)
    cache = hg_paged_cache(block_table.shape[0], H, D, page_size, pages, block_table.shape[1], K.stride(0), K.stride(1),
                           K.stride(2), K.data_ptr(), V.data_ptr(), table)
    cache.tensors = (K, V, block_table)
    return cache


def _kind(cache, kind) -> None:
    """The calls read the descriptor's memory as one kind of cache."""
    if not isinstance(cache, kind):
        raise TypeError(f"{type(cache).__name__} in the place of a {kind.__name__}")


def make_rotation(cos: torch.Tensor, sin: torch.Tensor, interleaved=False, sections=None) -> hg_rotation:
    """Descriptor of a position rotation: fp32 tables [max_pos, rot_dim / 2];
    sections: pairs per position axis, three numbers."""
    if cos.dim() != 2:
        raise ValueError("cos and sin must be [max_pos, rot_dim / 2]")
    c = _array(cos, "cos", cos.shape, torch.float32)
    s = _array(sin, "sin", cos.shape, torch.float32)
    rot = hg_rotation(c, s, cos.shape[0], 2 * cos.shape[1], int(interleaved), *(sections or (0, 0, 0)))
    rot.tensors = (cos, sin)
    return rot


_NO_ROWS = (0, 0, 0)
_address = C.addressof


def _append_operands(cache, rotation, q, k, v, lens, q_out, cu_new, positions, k_out) -> bytes:
    """The packed hg_append of an append call."""
    B, D, H = cache.B, cache.D, cache.H
    N = k.shape[0]
    Hq, q_rows, out_rows, k_rows = 0, _NO_ROWS, _NO_ROWS, _NO_ROWS
    if q is not None:
        Hq = q.shape[1]
        q_rows, out_rows = _rows(q, "q", N, Hq, D), _rows(q_out, "q_out", N, Hq, D)
    if k_out is not None:
        k_rows = _rows(k_out, "k_out", N, H, D)
    p = 0
    if positions is not None:
        axes = rotation is not None and (rotation.section0 or rotation.section1 or rotation.section2)
        p = _array(positions, "positions", (3, N) if axes else (N,))
    return _append_args(N, Hq, *q_rows, *_rows(k, "k", N, H, D), *_rows(v, "v", N, H, D), *out_rows, *k_rows,
                        _array(lens, "lens", (B,)), 0 if cu_new is None else _array(cu_new, "cu_new", (B + 1,)), p)


def hg_append_kv(cache: hg_paged_cache, rotation: Optional[hg_rotation], q: Optional[torch.Tensor], k: torch.Tensor,
                 v: torch.Tensor, lens: torch.Tensor, q_out: Optional[torch.Tensor] = None,
                 cu_new: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                 k_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue the rotation of the new tokens' keys (and queries: q [N, Hq, D]
    into q_out, which may be q) and the store of keys and values [N, H, D] into
    the cache.  lens [B]: tokens of each row with the new ones; cu_new [B + 1]:
    offsets of the rows' new tokens (None: one token a row); positions [N], or
    [3, N] with sections (None: a token's index in the cache); k_out: packed
    rotated keys, for the prompts' attention."""
    _kind(cache, hg_paged_cache)
    args = _append_operands(cache, rotation, q, k, v, lens, q_out, cu_new, positions, k_out)
    status = _append_call(_address(cache), None if rotation is None else _address(rotation), args, _stream(stream))
    if status:
        _check(status)


def hg_prefill_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, out: torch.Tensor,
                         cu_k: Optional[torch.Tensor] = None, causal: bool = True, scale: Optional[float] = None,
                         lse: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue the attention of packed prompts: q, out [Nq, Hq, D], k, v
    [Nk, H, D], cu_q, cu_k (None: cu_q) [B + 1] the rows' offsets; lse fp32
    [Nq, Hq] or None; scale None: 1/sqrt(D)."""
    Nq, Hq, D = q.shape
    Nk, H, _ = k.shape
    B = cu_q.shape[0] - 1
    args = _prefill_args(B, Hq, H, D, Nq, Nk, int(causal), D ** -0.5 if scale is None else scale,
                         *_rows(q, "q", Nq, Hq, D), *_rows(k, "k", Nk, H, D), *_rows(v, "v", Nk, H, D),
                         *_rows(out, "out", Nq, Hq, D), _array(lse, "lse", (Nq, Hq), torch.float32),
                         _array(cu_q, "cu_q", (B + 1,)), _array(cu_k, "cu_k", (B + 1,)))
    status = _prefill_call(args, _stream(stream))
    if status:
        _check(status)


def hg_decode_workspace(cache: hg_paged_cache, Hq: int) -> int:
    """Bytes of the decode call's workspace."""
    out = C.c_uint64()
    _check(_lib.hg_decode_workspace(cache, int(Hq), C.byref(out)))
    return out.value


def alloc_decode_workspace(cache: hg_paged_cache, Hq: int, device="cuda") -> torch.Tensor:
    """A zeroed workspace (uint8) for hg_decode_attention; every call leaves it
    ready for the next, whatever that one's number of rows and heads.  Calls that
    may overlap need one each."""
    return torch.zeros(hg_decode_workspace(cache, Hq), dtype=torch.uint8, device=device)


def hg_decode_attention(cache: hg_paged_cache, q: torch.Tensor, lens: torch.Tensor, out: torch.Tensor,
                        workspace: torch.Tensor, starts: Optional[torch.Tensor] = None,
                        lse: Optional[torch.Tensor] = None, scale: Optional[float] = None, stream=None) -> None:
    """Enqueue the attention of one new token per row, q, out [B, Hq, D], over
    the row's cached tokens [starts[b], lens[b]) (starts None: 0); lse fp32
    [B, Hq] or None; scale None: 1/sqrt(D)."""
    _kind(cache, hg_paged_cache)
    if workspace is None or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor")
    B, D = cache.B, cache.D
    Hq = q.shape[1]
    args = _decode_args(Hq, D ** -0.5 if scale is None else scale, *_rows(q, "q", B, Hq, D), *_rows(out, "out", B, Hq, D),
                        0 if lse is None else _array(lse, "lse", (B, Hq), torch.float32), _array(lens, "lens", (B,)),
                        0 if starts is None else _array(starts, "starts", (B,)), workspace.data_ptr(),
                        workspace.numel() * workspace.element_size())
    status = _decode_call(_address(cache), args, _stream(stream))
    if status:
        _check(status)


# ------------------------------------------------------------ the cache in 8 bits

def make_cache8(K: torch.Tensor, V: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, block_table: torch.Tensor,
                bounds: Optional[torch.Tensor] = None) -> hg_cache8:
    """Descriptor of one layer's pages in 8 bits: K, V [pages, H, page_size, D]
    codes (uint8 or float8_e4m3fn; a transposed view where tokens come before
    heads in memory), k_scale, v_scale fp32 [pages, H, page_size / block_size],
    which say the block size, bounds bfloat16 [pages, H, page_size / block_size,
    2, D] or None (needed by hg_select_blocks), block_table [B, max_pages].  It
    holds their addresses and keeps them alive."""
    if K.dim() != 4 or K.shape != V.shape or any(n != 1 and a != b for n, a, b in zip(K.shape, K.stride(), V.stride())):
        raise ValueError("K and V must both be [pages, H, page_size, D] with the same strides")
    if K.dtype not in (torch.uint8, torch.float8_e4m3fn) or V.dtype is not K.dtype:
        raise TypeError("K and V must both be uint8 or float8_e4m3fn")
    if K.stride(3) != 1:
        raise ValueError("the channels of K and V are not contiguous")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    pages, H, page_size, D = K.shape
    if k_scale.dim() != 3 or k_scale.shape[2] == 0 or page_size % k_scale.shape[2]:
        raise ValueError("k_scale must be [pages, H, page_size / block_size]")
    n = k_scale.shape[2]
    cache = hg_cache8(block_table.shape[0], H, D, page_size, pages, block_table.shape[1], page_size // n, K.stride(0), K.stride(1),
                      K.stride(2), K.data_ptr(), V.data_ptr(), _array(k_scale, "k_scale", (pages, H, n), torch.float32),
                      _array(v_scale, "v_scale", (pages, H, n), torch.float32),
                      _array(bounds, "bounds", (pages, H, n, 2, D), torch.bfloat16),
                      _array(block_table, "block_table", block_table.shape))
    cache.tensors = (K, V, k_scale, v_scale, bounds, block_table)
    return cache


def alloc_cache8(num_pages: int, H: int, page_size: int, D: int, block_table: torch.Tensor, block_size: int = 64, bounds: bool = True,
                 device="cuda") -> hg_cache8:
    """A zeroed 8-bit cache; its tensors (K, V, k_scale, v_scale, bounds,
    block_table) are cache.tensors."""
    if page_size % block_size:
        raise ValueError(f"page_size {page_size} is not a multiple of block_size {block_size}")
    n = page_size // block_size
    codes = [torch.zeros((num_pages, H, page_size, D), dtype=torch.uint8, device=device) for _ in range(2)]
    scales = [torch.ones((num_pages, H, n), dtype=torch.float32, device=device) for _ in range(2)]
    limits = torch.zeros((num_pages, H, n, 2, D), dtype=torch.bfloat16, device=device) if bounds else None
    return make_cache8(*codes, *scales, block_table, limits)


def hg_append_kv8(cache: hg_cache8, rotation: Optional[hg_rotation], q: Optional[torch.Tensor], k: torch.Tensor,
                  v: torch.Tensor, lens: torch.Tensor, q_out: Optional[torch.Tensor] = None,
                  cu_new: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                  k_out: Optional[torch.Tensor] = None, stream=None, starts: Optional[torch.Tensor] = None) -> None:
    """hg_append_kv into an 8-bit cache: the new keys and values become codes, the
    scales of the blocks that they lie in and their bounds are brought up to date.
    starts [B]: the rows' first tokens, as in the attention (hg_append_kv8_from; None:
    0); what a block held before its row's first token does not matter."""
    _kind(cache, hg_cache8)
    args = _append_operands(cache, rotation, q, k, v, lens, q_out, cu_new, positions, k_out)
    status = _append8_call(_address(cache), None if rotation is None else _address(rotation), args,
                           0 if starts is None else _array(starts, "starts", (cache.B,)), _stream(stream))
    if status:
        _check(status)


def _workspace(t: torch.Tensor, name: str):
    """Address and bytes of a workspace."""
    if t is None or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor")
    return t.data_ptr(), t.numel() * t.element_size()


def hg_decode8_workspace(cache: hg_cache8, Hq: int) -> int:
    """Bytes of hg_decode_attention8's workspace."""
    out = C.c_uint64()
    _check(_lib.hg_decode8_workspace(cache, int(Hq), C.byref(out)))
    return out.value


def alloc_decode8_workspace(cache: hg_cache8, Hq: int, device="cuda") -> torch.Tensor:
    """A zeroed workspace (uint8) for hg_decode_attention8, as alloc_decode_workspace's."""
    return torch.zeros(hg_decode8_workspace(cache, Hq), dtype=torch.uint8, device=device)


def hg_decode_attention8(cache: hg_cache8, q: torch.Tensor, lens: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor,
                         starts: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         scale: Optional[float] = None, blocks: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue the attention of one new token per row, q, out [B, Hq, D], over
    the row's tokens [starts[b], lens[b]) in an 8-bit cache, or over those of
    them that lie in the blocks listed: blocks int32 [B, H, budget], as
    hg_select_blocks writes them; lse fp32 [B, Hq] or None; scale None: 1/sqrt(D)."""
    _kind(cache, hg_cache8)
    B, D, H = cache.B, cache.D, cache.H
    Hq = q.shape[1]
    listed, budget = 0, 0
    if blocks is not None:
        if blocks.dim() != 3:
            raise ValueError("blocks must be [B, H, budget]")
        budget = blocks.shape[2]
        listed = _array(blocks, "blocks", (B, H, budget))
    args = _decode8_args(Hq, D ** -0.5 if scale is None else scale, *_rows(q, "q", B, Hq, D), *_rows(out, "out", B, Hq, D),
                         0 if lse is None else _array(lse, "lse", (B, Hq), torch.float32), _array(lens, "lens", (B,)),
                         0 if starts is None else _array(starts, "starts", (B,)), *_workspace(workspace, "workspace"),
                         listed, budget)
    status = _decode8_call(_address(cache), args, _stream(stream))
    if status:
        _check(status)


def hg_select_workspace(cache: hg_cache8) -> int:
    """Bytes of hg_select_blocks' workspace."""
    out = C.c_uint64()
    _check(_lib.hg_select_workspace(cache, C.byref(out)))
    return out.value


def alloc_select_workspace(cache: hg_cache8, device="cuda") -> torch.Tensor:
    """A workspace (uint8) for hg_select_blocks; calls that may overlap need one each."""
    return torch.empty(hg_select_workspace(cache), dtype=torch.uint8, device=device)


def hg_select_blocks(cache: hg_cache8, q: torch.Tensor, lens: torch.Tensor, blocks: torch.Tensor, workspace: torch.Tensor,
                     starts: Optional[torch.Tensor] = None, first: int = 1, last: int = 2, stream=None) -> None:
    """Enqueue the choice of each row's and key/value head's blocks for its
    queries q [B, Hq, D]: blocks int32 [B, H, budget] gets the numbers of the
    `first` first and `last` last blocks of the row's tokens [starts[b], lens[b])
    and of the highest bounds between, ascending, then -1."""
    _kind(cache, hg_cache8)
    B, D, H = cache.B, cache.D, cache.H
    Hq = q.shape[1]
    if blocks.dim() != 3:
        raise ValueError("blocks must be [B, H, budget]")
    budget = blocks.shape[2]
    args = _select_args(Hq, *_rows(q, "q", B, Hq, D), _array(lens, "lens", (B,)),
                        0 if starts is None else _array(starts, "starts", (B,)), _array(blocks, "blocks", (B, H, budget)),
                        budget, first, last, *_workspace(workspace, "workspace"))
    status = _select_call(_address(cache), args, _stream(stream))
    if status:
        _check(status)


# ------------------------------------------------------------ pages of rows

def make_page_pool(block_table: torch.Tensor, lens: torch.Tensor, free_pages: torch.Tensor, n_free: torch.Tensor,
                   page_size: int) -> hg_page_pool:
    """Descriptor of the pages of a cache's rows: block_table [B, max_pages] and
    lens [B], which the append and attention calls take too, free_pages
    [num_pages], whose first n_free [1] entries are the free pages."""
    if block_table.dim() != 2 or free_pages.dim() != 1:
        raise ValueError("block_table must be [B, max_pages], free_pages [num_pages]")
    B = block_table.shape[0]
    pool = hg_page_pool(B, page_size, free_pages.shape[0], block_table.shape[1], _array(block_table, "block_table", block_table.shape),
                        _array(lens, "lens", (B,)), _array(free_pages, "free_pages", free_pages.shape), _array(n_free, "n_free", (1,)))
    pool.tensors = (block_table, lens, free_pages, n_free)
    return pool


def alloc_page_pool(B: int, max_pages: int, num_pages: int, page_size: int, device="cuda") -> hg_page_pool:
    """A pool of empty rows, all pages free (page 0 on top); its tensors
    (block_table, lens, free_pages, n_free) are pool.tensors."""
    return make_page_pool(torch.full((B, max_pages), -1, dtype=torch.int32, device=device),
                          torch.zeros(B, dtype=torch.int32, device=device),
                          torch.arange(num_pages - 1, -1, -1, dtype=torch.int32, device=device),
                          torch.full((1,), num_pages, dtype=torch.int32, device=device), page_size)


def hg_resize_rows(pool: hg_page_pool, targets: torch.Tensor, result: torch.Tensor, cu_new: Optional[torch.Tensor] = None,
                   slots: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue the change of the rows' lengths to targets [B]: pages go on and
    come off the free ones, block table and lengths follow.  cu_new [B + 1]:
    offsets of the tokens that rows gain; slots int64 [N], positions int32 [N]:
    each one's place in the pages and in its row, -1 past the last; result
    int32 [4]: 0 or why nothing changed, pages missing, tokens gained, pages free."""
    _kind(pool, hg_page_pool)
    N = 0 if slots is None and positions is None else (positions if slots is None else slots).shape[0]
    B = pool.B
    args = _resize_args(N, _array(targets, "targets", (B,)), _array(cu_new, "cu_new", (B + 1,)),
                        _array(slots, "slots", (N,), torch.int64), _array(positions, "positions", (N,)),
                        _array(result, "result", (4,)))
    status = _resize_call(_address(pool), args, _stream(stream))
    if status:
        _check(status)
