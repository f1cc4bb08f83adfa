"""ctypes binding of libattncache.so: argument marshalling only.

Every function mirrors one C entry point of ``include/attncache.h`` under the
same name.  Tensors are torch CUDA tensors (PyTorch supplies device memory and
streams, nothing else); this layer checks device / dtype / shape / contiguity
so that no malformed pointer can reach a kernel, then passes ``data_ptr()`` and
the current stream.  There is no CPU fallback: without the built library, or
without a GPU tensor, the calls raise.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

import torch

from . import build as _build

AC_F32, AC_F16, AC_BF16 = 0, 1, 2
AC_IP, AC_L2 = 0, 1
AC_LAYOUT_DENSE, AC_LAYOUT_PACKED = 0, 1
AC_MAX_K = 64
AC_ROTARY_PLAIN, AC_ROTARY_LINEAR, AC_ROTARY_BASE, AC_ROTARY_RAMP = 0, 1, 2, 3

_DTYPE_CODE = {torch.float32: AC_F32, torch.float16: AC_F16, torch.bfloat16: AC_BF16}

SYMBOLS = ["attncache_workspace_bytes", "attncache_map_entry_bytes", "attncache_pack_maps",
           "attncache_build_db", "attncache_destroy_db",
           "attncache_search", "attncache_search_static", "attncache_apply", "attention_exact", "attncache_insert",
           "attncache_cache_stats", "attncache_cache_reset",
           "attncache_project_workspace_bytes", "attncache_project",
           "attncache_page_plan", "attncache_page_append", "attention_paged_workspace_bytes", "attention_paged",
           "attention_cross_workspace_bytes", "attention_cross",
           "attncache_rotate", "attncache_rotary_frequencies", "attncache_page_fork_workspace_bytes", "attncache_page_fork",
           "attention_paged_shared_workspace_bytes", "attention_paged_shared", "attention_window", "attention_paged_window",
           "attncache_status_string",
           "attncache_last_hip_error", "attncache_version", "attncache_set_pointer_checks"]


class AttnCacheError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().attncache_status_string(status).decode()
        hip = lib().attncache_last_hip_error() if status == -8 else 0
        super().__init__(f"{where}: status {status} ({msg})" + (f", hipError {hip}" if hip else ""))


class DbDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_emb", "emb_dim", "emb_dtype", "metric", "n_entries", "n_layers", "n_q_heads",
        "n_kv_heads", "head_dim", "seq_len", "map_dtype", "causal", "maps_on_host", "map_layout")]


_lib = None


def lib_path() -> str:
    return _build.LIB


def lib():
    """Load libattncache.so (it must have been built: see build.py / __graft_entry__.build)."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build the HIP library first "
                               "(python -m paper_2510_25979_amd.build)")
        L = ctypes.CDLL(path)
        i32, f32, vp, sz = ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
        L.attncache_workspace_bytes.restype = i32
        L.attncache_workspace_bytes.argtypes = [ctypes.POINTER(DbDesc), i32, i32, ctypes.POINTER(sz)]
        L.attncache_map_entry_bytes.restype = i32
        L.attncache_map_entry_bytes.argtypes = [ctypes.POINTER(DbDesc), ctypes.POINTER(sz)]
        L.attncache_pack_maps.restype = i32
        L.attncache_pack_maps.argtypes = [ctypes.POINTER(DbDesc), vp, i32, vp, vp]
        L.attncache_build_db.restype = i32
        L.attncache_build_db.argtypes = [ctypes.POINTER(DbDesc), vp, vp, vp, vp, sz, vp,
                                         ctypes.POINTER(vp)]
        L.attncache_destroy_db.restype = i32
        L.attncache_destroy_db.argtypes = [vp]
        L.attncache_search.restype = i32
        L.attncache_search.argtypes = [vp, vp, i32, i32, f32, vp, vp, vp, vp, sz, vp]
        L.attncache_search_static.restype = i32
        L.attncache_search_static.argtypes = [vp, vp, i32, i32, f32, vp, vp, vp, vp]
        L.attncache_apply.restype = i32
        L.attncache_apply.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp]
        L.attention_exact.restype = i32
        L.attention_exact.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, vp]
        L.attncache_insert.restype = i32
        L.attncache_insert.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, f32, vp]
        L.attncache_cache_stats.restype = i32
        L.attncache_cache_stats.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(ctypes.c_uint64)]
        L.attncache_cache_reset.restype = i32
        L.attncache_cache_reset.argtypes = [vp]
        L.attncache_project_workspace_bytes.restype = sz
        L.attncache_project_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.attncache_project.restype = i32
        L.attncache_project.argtypes = [vp] * 7 + [i32] * 8 + [vp, sz, vp]
        i64 = ctypes.c_int64
        L.attncache_page_plan.restype = i32
        L.attncache_page_plan.argtypes = [vp] * 9 + [i32] * 5 + [vp]
        L.attncache_page_append.restype = i32
        L.attncache_page_append.argtypes = [vp] * 5 + [i32] * 6 + [i64, i32, vp]
        L.attention_paged_workspace_bytes.restype = sz
        L.attention_paged_workspace_bytes.argtypes = [i32] * 4
        L.attention_paged.restype = i32
        L.attention_paged.argtypes = [vp] * 6 + [i32] * 7 + [i64, i32, f32, vp, sz, vp]
        L.attention_cross_workspace_bytes.restype = sz
        L.attention_cross_workspace_bytes.argtypes = [i32] * 7
        L.attention_cross.restype = i32
        L.attention_cross.argtypes = [vp] * 6 + [i32] * 7 + [f32, vp, sz, vp]
        f64 = ctypes.c_double
        L.attncache_rotate.restype = i32
        L.attncache_rotate.argtypes = [vp] * 11 + [i32] * 6 + [i64] * 2 + [i32] * 2 + [i64] + [i32] * 2 + [f32] * 2 + [vp]
        L.attncache_rotary_frequencies.restype = i32
        L.attncache_rotary_frequencies.argtypes = [vp, i32, f64, i32, f64, f64, f64, f64]
        L.attncache_page_fork_workspace_bytes.restype = sz
        L.attncache_page_fork_workspace_bytes.argtypes = [i32] * 3
        L.attncache_page_fork.restype = i32
        L.attncache_page_fork.argtypes = [vp] * 10 + [i32] * 6 + [i64] + [i32] * 3 + [vp, sz, vp]
        L.attention_paged_shared_workspace_bytes.restype = sz
        L.attention_paged_shared_workspace_bytes.argtypes = [i32] * 5
        L.attention_paged_shared.restype = i32
        L.attention_paged_shared.argtypes = [vp] * 8 + [i32] * 8 + [i64, i32, f32, vp, sz, vp]
        L.attention_window.restype = i32
        L.attention_window.argtypes = [vp] * 6 + [i32] * 8 + [f32, vp]
        L.attention_paged_window.restype = i32
        L.attention_paged_window.argtypes = [vp] * 6 + [i32] * 7 + [i64] + [i32] * 3 + [f32, vp, sz, vp]
        L.attncache_status_string.restype = ctypes.c_char_p
        L.attncache_status_string.argtypes = [i32]
        L.attncache_last_hip_error.restype = i32
        L.attncache_last_hip_error.argtypes = []
        L.attncache_set_pointer_checks.restype = i32
        L.attncache_set_pointer_checks.argtypes = [i32]
        L.attncache_version.restype = i32
        L.attncache_version.argtypes = []
        L.calls = {}
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != 0:
        raise AttnCacheError(status, where)


# The check below in one native call (csrc/tensor_arg.cpp): where the tensor starts, or None if it is not plainly what
# is wanted.  Without the built module the Python code decides alone, 0.4 us a tensor slower.
try:
    from ._tensor_arg import address as _address
except ImportError:
    def _address(t, dtype, shape):
        return None

try:
    from . import _tensor_arg as _native
except ImportError:
    _native = None


def _call(name: str):
    """An entry point of many arguments, by the native module where it is built: ctypes takes 1.6 to 2.4 us to convert them (0.6 so)."""
    calls = lib().calls
    f = calls.get(name)
    if f is None:
        f = getattr(lib(), name)
        if hasattr(_native, name):
            f = functools.partial(getattr(_native, name), ctypes.cast(f, ctypes.c_void_p).value)
        calls[name] = f
    return f


def _dev(t: torch.Tensor, name: str, dtype=None, shape=None) -> int:
    p = _address(t, dtype, shape)
    if p is not None:
        return p
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, has {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, has {tuple(t.shape)}")
    return t.data_ptr()


# Not part of torch's documented interface; a torch without them goes the long way (_stream).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    """The raw stream handle.  The current one is asked for directly: building a torch.cuda.Stream
    object to read it from took 2.7 of the 9.5 us a call spent on the host (6.9 us so)."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


class Database:
    """Owner of an ``attncache_db`` handle; keeps the borrowed tensors alive."""

    def __init__(self, handle, desc: DbDesc, keep):
        self.handle = handle
        self.desc = desc
        self._keep = keep

    def close(self):
        if self.handle:
            _check(lib().attncache_destroy_db(self.handle), "attncache_destroy_db")
            self.handle = None
            self._keep = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def attncache_set_pointer_checks(on: bool) -> bool:
    """Per-call memory-space checks on/off; returns the previous setting."""
    return bool(lib().attncache_set_pointer_checks(int(bool(on))))


def attncache_workspace_bytes(desc: DbDesc, max_batch: int, k: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().attncache_workspace_bytes(ctypes.byref(desc), max_batch, k, ctypes.byref(out)),
           "attncache_workspace_bytes")
    return int(out.value)


def attncache_map_entry_bytes(desc: DbDesc) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().attncache_map_entry_bytes(ctypes.byref(desc), ctypes.byref(out)),
           "attncache_map_entry_bytes")
    return int(out.value)


def packed_tile_elems(seq_len: int, causal: bool) -> int:
    """Elements of one packed [S][S] map (what attncache_map_entry_bytes reports per head)."""
    d = DbDesc(n_emb=1, emb_dim=8, emb_dtype=AC_F16, metric=AC_IP, n_entries=1, n_layers=1,
               n_q_heads=1, n_kv_heads=1, head_dim=64, seq_len=seq_len, map_dtype=AC_BF16,
               causal=int(causal), maps_on_host=0, map_layout=AC_LAYOUT_PACKED)
    return attncache_map_entry_bytes(d) // 2


def attncache_pack_maps(dense: torch.Tensor, packed: torch.Tensor, *, causal: bool = True,
                        stream: Optional[torch.cuda.Stream] = None) -> None:
    """dense [n,L,Hq,S,S] bf16 (cuda) -> packed [n,L,Hq,packed_tile_elems(S)] bf16 (cuda)."""
    if dense.dim() != 5 or dense.shape[3] != dense.shape[4]:
        raise ValueError("dense must be [n,L,Hq,S,S]")
    n, L, Hq, S, _ = dense.shape
    d = DbDesc(n_emb=1, emb_dim=8, emb_dtype=AC_F16, metric=AC_IP, n_entries=max(n, 1), n_layers=L,
               n_q_heads=Hq, n_kv_heads=Hq, head_dim=64, seq_len=S, map_dtype=AC_BF16,
               causal=int(causal), maps_on_host=0, map_layout=AC_LAYOUT_PACKED)
    dp = _dev(dense, "dense", torch.bfloat16)
    pp = _dev(packed, "packed", torch.bfloat16, (n, L, Hq, packed_tile_elems(S, causal)))
    _check(lib().attncache_pack_maps(ctypes.byref(d), dp, n, pp, _stream(stream)),
           "attncache_pack_maps")


def attncache_build_db(emb: torch.Tensor, maps: torch.Tensor, *, n_kv_heads: int, head_dim: int,
                       metric: int = AC_IP, causal: bool = True,
                       map_of: Optional[torch.Tensor] = None,
                       staging: Optional[torch.Tensor] = None,
                       side_stream: Optional[torch.cuda.Stream] = None,
                       seq_len: Optional[int] = None) -> Database:
    """emb [N,E] (cuda, f16/f32); maps (cuda, or pinned host) bf16/f32: dense [M,L,Hq,S,S], or
    packed [M,L,Hq,packed_tile_elems(S)] with ``seq_len`` given."""
    packed = maps.dim() == 4
    if packed:
        if seq_len is None or maps.shape[3] != packed_tile_elems(seq_len, causal):
            raise ValueError("packed maps must be [M,L,Hq,packed_tile_elems(seq_len)]")
    elif emb.dim() != 2 or maps.dim() != 5 or maps.shape[3] != maps.shape[4]:
        raise ValueError("emb must be [N,E] and maps [M,L,Hq,S,S]")
    else:
        if seq_len is not None and seq_len != maps.shape[3]:
            raise ValueError("seq_len disagrees with the dense maps")
        seq_len = maps.shape[3]
    on_host = not maps.is_cuda
    if on_host and not maps.is_pinned():
        raise ValueError("host-resident maps must be pinned memory")
    if not maps.is_contiguous():
        raise ValueError("maps must be contiguous")
    if emb.dtype not in (torch.float16, torch.float32) or maps.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("unsupported dtype")
    d = DbDesc(n_emb=emb.shape[0], emb_dim=emb.shape[1], emb_dtype=_DTYPE_CODE[emb.dtype],
               metric=metric, n_entries=maps.shape[0], n_layers=maps.shape[1],
               n_q_heads=maps.shape[2], n_kv_heads=n_kv_heads, head_dim=head_dim,
               seq_len=seq_len, map_dtype=_DTYPE_CODE[maps.dtype], causal=int(causal),
               maps_on_host=int(on_host),
               map_layout=AC_LAYOUT_PACKED if packed else AC_LAYOUT_DENSE)
    emb_p = _dev(emb, "emb")
    mo_p = None if map_of is None else _dev(map_of, "map_of", torch.int32, (emb.shape[0],))
    st_p, st_bytes, ss = None, 0, None
    if on_host:
        if staging is None or side_stream is None:
            raise ValueError("host-resident maps need a staging tensor and a side stream")
        st_p = _dev(staging, "staging")
        st_bytes = staging.numel() * staging.element_size()
        ss = side_stream.cuda_stream
    handle = ctypes.c_void_p()
    _check(lib().attncache_build_db(ctypes.byref(d), emb_p, mo_p, maps.data_ptr(), st_p, st_bytes,
                                    ss, ctypes.byref(handle)), "attncache_build_db")
    return Database(handle, d, (emb, maps, map_of, staging, side_stream))


def attncache_search(db: Database, q: torch.Tensor, k: int, threshold: float,
                     idx: torch.Tensor, score: torch.Tensor, hit: torch.Tensor,
                     ws: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    d = db.desc
    B = q.shape[0]
    emb_dt = torch.float16 if d.emb_dtype == AC_F16 else torch.float32
    qp = _dev(q, "q", emb_dt, (B, d.emb_dim))
    ip = _dev(idx, "idx", torch.int32, (B, k))
    sp = _dev(score, "score", torch.float32, (B, k))
    hp = _dev(hit, "hit", torch.int32, (B,))
    wp = _dev(ws, "ws")
    _check(lib().attncache_search(db.handle, qp, B, k, float(threshold), ip, sp, hp, wp,
                                  ws.numel() * ws.element_size(), _stream(stream)),
           "attncache_search")


AC_STATIC_SCRATCH_BYTES = 4 << 20


def attncache_search_static(db: Database, q: torch.Tensor, k: int, threshold: float,
                            idx: torch.Tensor, score: torch.Tensor, hit: torch.Tensor,
                            stream: Optional[torch.cuda.Stream] = None) -> None:
    """attncache_search on the library's built-in workspace (no allocation anywhere)."""
    d = db.desc
    B = q.shape[0]
    emb_dt = torch.float16 if d.emb_dtype == AC_F16 else torch.float32
    qp = _dev(q, "q", emb_dt, (B, d.emb_dim))
    ip = _dev(idx, "idx", torch.int32, (B, k))
    sp = _dev(score, "score", torch.float32, (B, k))
    hp = _dev(hit, "hit", torch.int32, (B,))
    _check(lib().attncache_search_static(db.handle, qp, B, k, float(threshold), ip, sp, hp,
                                         _stream(stream)), "attncache_search_static")


def attncache_apply(db: Database, hit: torch.Tensor, V: torch.Tensor, O: torch.Tensor,
                    layer_begin: int = 0, layer_count: Optional[int] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> None:
    d = db.desc
    Lc = d.n_layers - layer_begin if layer_count is None else layer_count
    B = V.shape[0]
    dt = torch.bfloat16 if d.map_dtype == AC_BF16 else torch.float32
    vp = _dev(V, "V", dt, (B, Lc, d.n_kv_heads, d.seq_len, d.head_dim))
    op = _dev(O, "O", dt, (B, Lc, d.n_q_heads, d.seq_len, d.head_dim))
    if d.maps_on_host:
        if hit.is_cuda or hit.dtype != torch.int32 or not hit.is_contiguous() or tuple(hit.shape) != (B,):
            raise ValueError("hit must be a contiguous host int32 tensor [B] for host-resident maps")
        hp = hit.data_ptr()
    else:
        hp = _dev(hit, "hit", torch.int32, (B,))
    _check(lib().attncache_apply(db.handle, hp, vp, op, B, layer_begin, Lc, _stream(stream)),
           "attncache_apply")


def attncache_cache_stats(db: Database):
    """(lookups, copies) of the entry cache of a host-resident database."""
    a, b = ctypes.c_uint64(), ctypes.c_uint64()
    _check(lib().attncache_cache_stats(db.handle, ctypes.byref(a), ctypes.byref(b)), "attncache_cache_stats")
    return a.value, b.value


def attncache_cache_reset(db: Database) -> None:
    _check(lib().attncache_cache_reset(db.handle), "attncache_cache_reset")


def attncache_insert(db: Database, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, O: torch.Tensor, *,
                     slot: Optional[torch.Tensor] = None, feat: Optional[torch.Tensor] = None,
                     row_sel: Optional[torch.Tensor] = None,
                     key_len: Optional[torch.Tensor] = None, layer_begin: int = 0,
                     scale: float = 0.0, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Q,O [B,Lc,Hq,S,D]; K,V [B,Lc,Hkv,S,D] bf16; slot, row_sel, key_len [B] int32; feat [B,E]."""
    d = db.desc
    if Q.dim() != 5:
        raise ValueError("Q must be [B,Lc,Hq,S,D]")
    B, Lc = Q.shape[0], Q.shape[1]
    dt = torch.bfloat16
    qp = _dev(Q, "Q", dt, (B, Lc, d.n_q_heads, d.seq_len, d.head_dim))
    kp = _dev(K, "K", dt, (B, Lc, d.n_kv_heads, d.seq_len, d.head_dim))
    vp = _dev(V, "V", dt, (B, Lc, d.n_kv_heads, d.seq_len, d.head_dim))
    op = _dev(O, "O", dt, (B, Lc, d.n_q_heads, d.seq_len, d.head_dim))
    sp = None if slot is None else _dev(slot, "slot", torch.int32, (B,))
    rp = None if row_sel is None else _dev(row_sel, "row_sel", torch.int32, (B,))
    lp = None if key_len is None else _dev(key_len, "key_len", torch.int32, (B,))
    fdt = torch.float16 if d.emb_dtype == AC_F16 else torch.float32
    fp = None if feat is None else _dev(feat, "feat", fdt, (B, d.emb_dim))
    _check(lib().attncache_insert(db.handle, fp, sp, rp, lp, qp, kp, vp, op, B, layer_begin, Lc,
                                  float(scale), _stream(stream)), "attncache_insert")


def attention_exact(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, O: torch.Tensor, *,
                    causal: bool = True, scale: float = 0.0,
                    row_sel: Optional[torch.Tensor] = None,
                    key_len: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> None:
    """Q,O [B,Hq,S,D]; K,V [B,Hkv,S,D]; bf16 or f32; row_sel, key_len [B] int32."""
    if Q.dim() != 4 or K.dim() != 4:
        raise ValueError("Q must be [B,Hq,S,D] and K,V [B,Hkv,S,D]")
    B, Hq, S, D = Q.shape
    Hkv = K.shape[1]
    if Q.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("unsupported dtype")
    qp = _dev(Q, "Q")
    kp = _dev(K, "K", Q.dtype, (B, Hkv, S, D))
    vp = _dev(V, "V", Q.dtype, (B, Hkv, S, D))
    op = _dev(O, "O", Q.dtype, (B, Hq, S, D))
    rp = None if row_sel is None else _dev(row_sel, "row_sel", torch.int32, (B,))
    lp = None if key_len is None else _dev(key_len, "key_len", torch.int32, (B,))
    _check(lib().attention_exact(qp, kp, vp, op, rp, lp, B, Hq, Hkv, S, D, _DTYPE_CODE[Q.dtype],
                                 int(causal), float(scale), _stream(stream)), "attention_exact")


def attncache_project_workspace_bytes(B: int, model_dim: int, hidden_dim: int, emb_dim: int) -> int:
    return int(lib().attncache_project_workspace_bytes(B, model_dim, hidden_dim, emb_dim))


def attncache_project(h: torch.Tensor, W1: torch.Tensor, b1: Optional[torch.Tensor],
                      W2: torch.Tensor, b2: Optional[torch.Tensor], feat: torch.Tensor,
                      workspace: torch.Tensor, *, seq_len: Optional[torch.Tensor] = None,
                      normalize: bool = True, stream: Optional[torch.cuda.Stream] = None) -> None:
    """h [B,S,dm] bf16|f32; W1 [hid,dm], b1 [hid], W2 [E,hid], b2 [E] f32; feat [B,E] f16|f32."""
    if h.dim() != 3 or W1.dim() != 2 or W2.dim() != 2:
        raise ValueError("h must be [B,S,dm], W1 [hid,dm], W2 [E,hid]")
    B, S, dm = h.shape
    hid, E = W1.shape[0], W2.shape[0]
    if h.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("h must be bf16 or f32")
    if feat.dtype not in (torch.float16, torch.float32):
        raise ValueError("feat must be f16 or f32")
    f32 = torch.float32
    hp = _dev(h, "h")
    w1 = _dev(W1, "W1", f32, (hid, dm))
    w2 = _dev(W2, "W2", f32, (E, hid))
    b1p = None if b1 is None else _dev(b1, "b1", f32, (hid,))
    b2p = None if b2 is None else _dev(b2, "b2", f32, (E,))
    fp = _dev(feat, "feat", None, (B, E))
    sp = None if seq_len is None else _dev(seq_len, "seq_len", torch.int32, (B,))
    wp = _dev(workspace, "workspace")
    _check(lib().attncache_project(hp, sp, w1, b1p, w2, b2p, fp, B, S, dm, hid, E,
                                   _DTYPE_CODE[h.dtype], _DTYPE_CODE[feat.dtype], int(normalize),
                                   wp, workspace.numel() * workspace.element_size(),
                                   _stream(stream)), "attncache_project")


def attncache_page_plan(seq_len: torch.Tensor, new_len: torch.Tensor, free_state: torch.Tensor,
                        free_pages: torch.Tensor, page_table: torch.Tensor, seq_len_out: torch.Tensor,
                        added: torch.Tensor, free_state_out: torch.Tensor, slot: torch.Tensor, *,
                        page_size: int, stream: Optional[torch.cuda.Stream] = None) -> None:
    """All int32: seq_len, new_len, seq_len_out, added [B]; free_state, free_state_out [2]; free_pages [n_pages];
    page_table [B,max_pages]; slot [B,S].  The outputs may be the inputs of the same meaning."""
    if page_table.dim() != 2 or slot.dim() != 2 or free_pages.dim() != 1:
        raise ValueError("page_table must be [B,max_pages], slot [B,S] and free_pages [n_pages]")
    i32, per_request, two = torch.int32, (page_table.shape[0],), (2,)
    (B, max_pages), S, n = page_table.shape, slot.shape[1], free_pages.shape[0]
    lp = _dev(seq_len, "seq_len", i32, per_request)
    np_ = _dev(new_len, "new_len", i32, per_request)
    fs = _dev(free_state, "free_state", i32, two)
    fp = _dev(free_pages, "free_pages", i32)
    tp = _dev(page_table, "page_table", i32)
    lo = _dev(seq_len_out, "seq_len_out", i32, per_request)
    ap = _dev(added, "added", i32, per_request)
    fo = _dev(free_state_out, "free_state_out", i32, two)
    sp = _dev(slot, "slot", i32, (B, S))
    _check(lib().attncache_page_plan(lp, np_, fs, fp, tp, lo, ap, fo, sp, B, S, max_pages, page_size, n,
                                     _stream(stream)), "attncache_page_plan")


def _pages(k_pages: torch.Tensor, v_pages: torch.Tensor, dtype, heads: int, D: int):
    """Addresses, page count, page size and page stride of [n,heads,page,D] arrays whose pages may lie further apart."""
    shape = tuple(k_pages.shape)
    if len(shape) != 4 or shape[1] != heads or shape[3] != D or shape != tuple(v_pages.shape):
        raise ValueError(f"k_pages and v_pages must be [n_pages,{heads},page_size,{D}], have "
                         f"{shape} and {tuple(v_pages.shape)}")
    n, _, page, _ = shape
    stride = dense = heads * page * D
    kp, vp = _address(k_pages, dtype, None), _address(v_pages, dtype, None)
    if kp is not None and vp is not None:   # dense, both
        return kp, vp, n, page, stride
    if n > 1:
        stride = k_pages.stride(0)
    # (the stride of a dimension of one element says nothing)
    inner = all(t.shape[d] == 1 or t.stride(d) == w for t in (k_pages, v_pages)
                for d, w in ((1, page * D), (2, D), (3, 1)))
    if not inner or stride < dense or (n > 1 and v_pages.stride(0) != stride):
        raise ValueError("k_pages and v_pages must be contiguous within a page and have one page stride")
    for t, name in ((k_pages, "k_pages"), (v_pages, "v_pages")):
        if not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
        if t.dtype != dtype:
            raise ValueError(f"{name} must have dtype {dtype}, has {t.dtype}")
    return k_pages.data_ptr(), v_pages.data_ptr(), n, page, stride


def attncache_page_append(K: torch.Tensor, V: torch.Tensor, slot: torch.Tensor, k_pages: torch.Tensor,
                          v_pages: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """K,V [B,H,S,D] bf16 or f32; slot [B,S] int32; k_pages,v_pages [n_pages,H,page_size,D], whose pages may lie further
    apart than their size."""
    shape, dtype = tuple(K.shape), K.dtype
    if len(shape) != 4:
        raise ValueError("K and V must be [B,H,S,D]")
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("unsupported dtype")
    B, H, S, D = shape
    kp = _dev(K, "K")
    vp = _dev(V, "V", dtype, shape)
    sp = _dev(slot, "slot", torch.int32, (B, S))
    kc, vc, n, page, stride = _pages(k_pages, v_pages, dtype, H, D)
    _check(lib().attncache_page_append(kp, vp, sp, kc, vc, B, H, S, D, n, page, stride, _DTYPE_CODE[dtype],
                                       _stream(stream)), "attncache_page_append")


def attention_paged_workspace_bytes(B: int, Hq: int, Hkv: int, D: int) -> int:
    return int(lib().attention_paged_workspace_bytes(B, Hq, Hkv, D))


def attention_paged(Q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor,
                    seq_len: torch.Tensor, O: torch.Tensor, workspace: torch.Tensor, *, scale: float = 0.0,
                    stream: Optional[torch.cuda.Stream] = None) -> None:
    """Q,O [B,Hq,D]; k_pages,v_pages [n_pages,Hkv,page_size,D], whose pages may lie further apart than their size; bf16 or
    f32; page_table [B,max_pages], seq_len [B] int32."""
    if Q.dim() != 3 or k_pages.dim() != 4 or page_table.dim() != 2:
        raise ValueError("Q must be [B,Hq,D], k_pages and v_pages [n_pages,Hkv,page_size,D], page_table [B,max_pages]")
    B, Hq, D = Q.shape
    Hkv, max_pages = k_pages.shape[1], page_table.shape[1]
    if Q.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("unsupported dtype")
    qp = _dev(Q, "Q")
    op = _dev(O, "O", Q.dtype, (B, Hq, D))
    tp = _dev(page_table, "page_table", torch.int32, (B, max_pages))
    lp = _dev(seq_len, "seq_len", torch.int32, (B,))
    kc, vc, n, page, stride = _pages(k_pages, v_pages, Q.dtype, Hkv, D)
    wp = _dev(workspace, "workspace")
    _check(lib().attention_paged(qp, kc, vc, tp, lp, op, B, Hq, Hkv, D, n, page, max_pages, stride,
                                 _DTYPE_CODE[Q.dtype], float(scale), wp,
                                 workspace.numel() * workspace.element_size(), _stream(stream)), "attention_paged")


def attention_cross_workspace_bytes(B: int, Hq: int, Hkv: int, Sq: int, Sk: int, D: int,
                                    dtype: Optional[torch.dtype] = None) -> int:
    """Without ``dtype``: enough for either type."""
    codes = (AC_BF16, AC_F32) if dtype is None else (_DTYPE_CODE[dtype],)
    return max(int(lib().attention_cross_workspace_bytes(B, Hq, Hkv, Sq, Sk, D, c)) for c in codes)


def attention_cross(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, O: torch.Tensor,
                    workspace: Optional[torch.Tensor] = None, *, scale: float = 0.0,
                    row_sel: Optional[torch.Tensor] = None, key_len: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> None:
    """Q,O [B,Hq,Sq,D]; K,V [B,Hkv,Sk,D]; bf16 or f32; row_sel, key_len [B] int32.  The workspace may be left out where
    attention_cross_workspace_bytes says 0."""
    if Q.dim() != 4 or K.dim() != 4:
        raise ValueError("Q must be [B,Hq,Sq,D] and K,V [B,Hkv,Sk,D]")
    B, Hq, Sq, D = Q.shape
    Hkv, Sk = K.shape[1], K.shape[2]
    if Q.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("unsupported dtype")
    qp = _dev(Q, "Q")
    kp = _dev(K, "K", Q.dtype, (B, Hkv, Sk, D))
    vp = _dev(V, "V", Q.dtype, (B, Hkv, Sk, D))
    op = _dev(O, "O", Q.dtype, (B, Hq, Sq, D))
    rp = None if row_sel is None else _dev(row_sel, "row_sel", torch.int32, (B,))
    lp = None if key_len is None else _dev(key_len, "key_len", torch.int32, (B,))
    wp, w_bytes = (None, 0) if workspace is None else (
        _dev(workspace, "workspace"), workspace.numel() * workspace.element_size())
    _check(lib().attention_cross(qp, kp, vp, op, rp, lp, B, Hq, Hkv, Sq, Sk, D, _DTYPE_CODE[Q.dtype], float(scale),
                                 wp, w_bytes, _stream(stream)), "attention_cross")


def attncache_rotary_frequencies(rot: int, *, base: float = 10000.0, scaling: int = AC_ROTARY_PLAIN, factor: float = 1.0,
                                 original_len: float = 0.0, low: float = 1.0, high: float = 4.0) -> torch.Tensor:
    """[rot/2] f64 on the host: what attncache_rotate takes, once it is on the device."""
    freq = torch.empty(max(rot, 0) // 2, dtype=torch.float64)
    _check(lib().attncache_rotary_frequencies(freq.data_ptr(), rot, base, scaling, factor, original_len, low, high),
           "attncache_rotary_frequencies")
    return freq


def attncache_rotate(X: torch.Tensor, pos: torch.Tensor, freq: Optional[torch.Tensor], Q: torch.Tensor,
                     K: Optional[torch.Tensor] = None, V: Optional[torch.Tensor] = None, *,
                     q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     amplitude: float = 1.0, interleaved: bool = False, slot: Optional[torch.Tensor] = None,
                     k_pages: Optional[torch.Tensor] = None, v_pages: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> None:
    """X [B,S,(Hq+2Hkv)*D] bf16 or f32, of any strides but the last; pos [B,S] int32; freq [rot/2] f64 or None; Q [B,Hq,S,D];
    K,V [B,Hkv,S,D]; q_weight, k_weight [D] f32; slot [B,S] int32 with k_pages,v_pages [n_pages,Hkv,page_size,D]."""
    if X.dim() != 3 or Q.dim() != 4:
        raise ValueError("X must be [B,S,(Hq+2Hkv)*D] and Q [B,Hq,S,D]")
    dtype = X.dtype
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("unsupported dtype")
    (B, S, width), (_, Hq, _, D) = X.shape, Q.shape
    Hkv = (width // D - Hq) // 2 if D > 0 else 0
    if Hkv < 1 or (Hq + 2 * Hkv) * D != width:
        raise ValueError(f"rows of X must hold {Hq} + 2 Hkv heads of {D}, have {width} elements")
    if K is None and V is not None or V is None and K is not None:
        raise ValueError("K and V must be given both, or none of them")
    if (slot is None) != (k_pages is None) or (slot is None) != (v_pages is None):
        raise ValueError("slot, k_pages and v_pages must be given all, or none of them")
    if K is None and slot is None:
        raise ValueError("K and V need a place: K and V, or slot, k_pages and v_pages")
    i32, f32 = torch.int32, torch.float32
    xp = _address(X, dtype, None)
    if xp is None:
        if not X.is_cuda:
            raise ValueError("X must be a CUDA tensor")
        if width > 1 and X.stride(2) != 1:
            raise ValueError("rows of X must be contiguous")
        xp = X.data_ptr()
    # (the stride of a dimension of one element says nothing)
    row_stride = X.stride(1) if S > 1 else width
    batch_stride = X.stride(0) if B > 1 else 0
    pp = _dev(pos, "pos", i32, (B, S))
    rot = 0 if freq is None else 2 * freq.numel()
    fp = None if rot == 0 else _dev(freq, "freq", torch.float64, (rot // 2,))
    qw = None if q_weight is None else _dev(q_weight, "q_weight", f32, (D,))
    kw = None if k_weight is None else _dev(k_weight, "k_weight", f32, (D,))
    qp = _dev(Q, "Q", dtype, (B, Hq, S, D))
    kp = None if K is None else _dev(K, "K", dtype, (B, Hkv, S, D))
    vp = None if V is None else _dev(V, "V", dtype, (B, Hkv, S, D))
    sp, kc, vc, n, page, stride = None, None, None, 0, 0, 0
    if slot is not None:
        sp = _dev(slot, "slot", i32, (B, S))
        kc, vc, n, page, stride = _pages(k_pages, v_pages, dtype, Hkv, D)
    _check(_call("attncache_rotate")(xp, qw, kw, pp, fp, sp, qp, kp, vp, kc, vc, B, S, Hq, Hkv, D, rot, batch_stride, row_stride,
                                     n, page, stride, _DTYPE_CODE[dtype], int(interleaved), float(eps), float(amplitude),
                                     _stream(stream)), "attncache_rotate")


def attncache_page_fork_workspace_bytes(B: int, max_pages: int, n_pages: int) -> int:
    return int(lib().attncache_page_fork_workspace_bytes(B, max_pages, n_pages))


def attncache_page_fork(from_row: torch.Tensor, seq_len: torch.Tensor, free_state: torch.Tensor, free_pages: torch.Tensor,
                        page_table: torch.Tensor, page_table_out: torch.Tensor, seq_len_out: torch.Tensor,
                        free_state_out: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, workspace: torch.Tensor, *,
                        sinks: int = 0, window: int = 0, stream: Optional[torch.cuda.Stream] = None) -> None:
    """All int32: from_row, seq_len, seq_len_out [B]; free_state, free_state_out [2]; free_pages [n_pages]; page_table,
    page_table_out [B,max_pages].  The outputs may be the inputs of the same meaning.  k_pages,v_pages
    [n_pages,H,page_size,D] bf16 or f32, whose pages may lie further apart than their size."""
    if page_table.dim() != 2 or k_pages.dim() != 4:
        raise ValueError("page_table must be [B,max_pages], k_pages and v_pages [n_pages,H,page_size,D]")
    if k_pages.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("unsupported dtype")
    i32, (B, max_pages), (_, H, _, D) = torch.int32, page_table.shape, k_pages.shape
    kc, vc, n, page, stride = _pages(k_pages, v_pages, k_pages.dtype, H, D)
    rp = _dev(from_row, "from_row", i32, (B,))
    lp = _dev(seq_len, "seq_len", i32, (B,))
    fs = _dev(free_state, "free_state", i32, (2,))
    fp = _dev(free_pages, "free_pages", i32, (n,))
    tp = _dev(page_table, "page_table", i32)
    to = _dev(page_table_out, "page_table_out", i32, (B, max_pages))
    lo = _dev(seq_len_out, "seq_len_out", i32, (B,))
    fo = _dev(free_state_out, "free_state_out", i32, (2,))
    wp = _dev(workspace, "workspace")
    _check(_call("attncache_page_fork")(rp, lp, fs, fp, tp, to, lo, fo, kc, vc, B, H, D, max_pages, n, page, stride, sinks, window,
                                        _DTYPE_CODE[k_pages.dtype], wp, workspace.numel() * workspace.element_size(),
                                        _stream(stream)), "attncache_page_fork")


def attention_paged_shared_workspace_bytes(B: int, Hq: int, Hkv: int, D: int, G: int) -> int:
    return int(lib().attention_paged_shared_workspace_bytes(B, Hq, Hkv, D, G))


def attention_paged_shared(Q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor,
                           seq_len: torch.Tensor, share_first: torch.Tensor, share_len: torch.Tensor, O: torch.Tensor,
                           workspace: torch.Tensor, *, scale: float = 0.0, stream: Optional[torch.cuda.Stream] = None) -> None:
    """As attention_paged; share_first [G+1] and share_len [G] int32: requests share_first[q] to share_first[q+1]-1 have their
    first share_len[q] tokens in common."""
    if Q.dim() != 3 or k_pages.dim() != 4 or page_table.dim() != 2 or share_len.dim() != 1:
        raise ValueError("Q must be [B,Hq,D], k_pages and v_pages [n_pages,Hkv,page_size,D], page_table [B,max_pages], share_len [G]")
    (B, Hq, D), G = Q.shape, share_len.shape[0]
    Hkv, max_pages = k_pages.shape[1], page_table.shape[1]
    if Q.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("unsupported dtype")
    qp = _dev(Q, "Q")
    op = _dev(O, "O", Q.dtype, (B, Hq, D))
    tp = _dev(page_table, "page_table", torch.int32, (B, max_pages))
    lp = _dev(seq_len, "seq_len", torch.int32, (B,))
    fp = _dev(share_first, "share_first", torch.int32, (G + 1,))
    sp = _dev(share_len, "share_len", torch.int32)
    kc, vc, n, page, stride = _pages(k_pages, v_pages, Q.dtype, Hkv, D)
    wp = _dev(workspace, "workspace")
    _check(_call("attention_paged_shared")(qp, kc, vc, tp, lp, fp, sp, op, B, Hq, Hkv, D, G, n, page, max_pages, stride,
                                           _DTYPE_CODE[Q.dtype], float(scale), wp,
                                           workspace.numel() * workspace.element_size(), _stream(stream)), "attention_paged_shared")


def attention_window(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, O: torch.Tensor, *, window: int, sinks: int = 0,
                     scale: float = 0.0, row_sel: Optional[torch.Tensor] = None, key_len: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> None:
    """Q,O [B,Hq,S,D]; K,V [B,Hkv,S,D]; bf16 or f32; row_sel, key_len [B] int32."""
    if Q.dim() != 4 or K.dim() != 4:
        raise ValueError("Q must be [B,Hq,S,D] and K,V [B,Hkv,S,D]")
    B, Hq, S, D = Q.shape
    Hkv = K.shape[1]
    if Q.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("unsupported dtype")
    qp = _dev(Q, "Q")
    kp = _dev(K, "K", Q.dtype, (B, Hkv, S, D))
    vp = _dev(V, "V", Q.dtype, (B, Hkv, S, D))
    op = _dev(O, "O", Q.dtype, (B, Hq, S, D))
    rp = None if row_sel is None else _dev(row_sel, "row_sel", torch.int32, (B,))
    lp = None if key_len is None else _dev(key_len, "key_len", torch.int32, (B,))
    _check(_call("attention_window")(qp, kp, vp, op, rp, lp, B, Hq, Hkv, S, D, _DTYPE_CODE[Q.dtype], window, sinks, float(scale),
                                     _stream(stream)), "attention_window")


def attention_paged_window(Q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor,
                           seq_len: torch.Tensor, O: torch.Tensor, workspace: torch.Tensor, *, window: int, sinks: int = 0,
                           scale: float = 0.0, stream: Optional[torch.cuda.Stream] = None) -> None:
    """As attention_paged, of whose keys the first ``sinks`` and the last ``window`` of each request are seen."""
    if Q.dim() != 3 or k_pages.dim() != 4 or page_table.dim() != 2:
        raise ValueError("Q must be [B,Hq,D], k_pages and v_pages [n_pages,Hkv,page_size,D], page_table [B,max_pages]")
    B, Hq, D = Q.shape
    Hkv, max_pages = k_pages.shape[1], page_table.shape[1]
    if Q.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("unsupported dtype")
    qp = _dev(Q, "Q")
    op = _dev(O, "O", Q.dtype, (B, Hq, D))
    tp = _dev(page_table, "page_table", torch.int32, (B, max_pages))
    lp = _dev(seq_len, "seq_len", torch.int32, (B,))
    kc, vc, n, page, stride = _pages(k_pages, v_pages, Q.dtype, Hkv, D)
    wp = _dev(workspace, "workspace")
    _check(_call("attention_paged_window")(qp, kc, vc, tp, lp, op, B, Hq, Hkv, D, n, page, max_pages, stride,
                                           _DTYPE_CODE[Q.dtype], window, sinks, float(scale), wp,
                                           workspace.numel() * workspace.element_size(), _stream(stream)), "attention_paged_window")
