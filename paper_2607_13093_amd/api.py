"""Thin torch-facing binding of libsph: argument marshalling only.

torch supplies device memory and the current stream; every step of the
computation runs in the library's HIP kernels.  Tensors must live on the GPU
and be contiguous along their last dimension (row strides are passed on).
"""

from __future__ import annotations

from typing import Optional

import torch

from . import _lib
from ._lib import SphError, check  # noqa: F401

GREEDY = _lib.SPH_GREEDY
SAMPLE = _lib.SPH_SAMPLE


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# the stream's handle alone, where torch gives it: a Stream object costs 2 us, and a
# decode call is 10
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle(device: torch.device) -> int:
    if device.index is None or _raw_stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    return _raw_stream(device.index)


def _require_gpu(name: str, t: torch.Tensor) -> None:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dim() >= 1 and t.stride(-1) != 1 and t.numel() > 0:
        raise ValueError(f"{name} must be contiguous along its last dimension")


def _as_bits16(t: torch.Tensor) -> torch.Tensor:
    if t.dtype in (torch.bfloat16, torch.int16, torch.uint16):
        return t
    raise TypeError(f"expected bf16 (or its 16-bit patterns), got {t.dtype}")


class Subset:
    """Device plan of a vocabulary subset V_l (strictly ascending ids)."""

    def __init__(self, ids=None, vocab: int = 0, full: bool = False, device=None):
        lib = _lib.load()
        self._lib = lib
        self.handle = ctypes_vp()
        dev = torch.device("cuda") if device is None else torch.device(device)
        with torch.cuda.device(dev):
            stream = _stream_handle(dev)
            if full:
                check(lib.sph_subset_create_full(int(vocab), stream, self.handle))
            else:
                import numpy as np
                host = np.ascontiguousarray(np.asarray(ids, dtype=np.int32))
                check(lib.sph_subset_create(host.ctypes.data, host.size, int(vocab), stream,
                                            self.handle))
        n = _lib.c_i64()
        v = _lib.c_i64()
        check(lib.sph_subset_size(self.handle, n, v))
        self.n, self.vocab = n.value, v.value
        self.device = dev

    def device_ids_ptr(self) -> int:
        p = _lib.c_vp()
        check(self._lib.sph_subset_device_ids(self.handle, p))
        return p.value

    def close(self) -> None:
        if self.handle is not None and self.handle.value:
            self._lib.sph_subset_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GcmKey:
    """Device AES-GCM key (16- or 32-byte key) for sealing payload rows (eq. 19)."""

    def __init__(self, key: bytes, device=None):
        import ctypes
        lib = _lib.load()
        self._lib = lib
        self.handle = ctypes_vp()
        key = bytes(key)
        buf = ctypes.create_string_buffer(key, len(key))
        dev = torch.device("cuda") if device is None else torch.device(device)
        with torch.cuda.device(dev):
            check(lib.sph_gcm_key_create(ctypes.addressof(buf), len(key), _stream_handle(dev),
                                         self.handle))
        ctypes.memset(buf, 0, len(key))
        self.device = dev

    def close(self) -> None:
        if self.handle is not None and self.handle.value:
            self._lib.sph_gcm_key_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def gcm_workspace(rows: int, row_bytes: int) -> int:
    return int(_lib.load().sph_gcm_workspace(int(rows), int(row_bytes)))


def _rows_u8(t: torch.Tensor, name: str):
    _require_gpu(name, t)
    shape, strides = t.shape, t.stride()
    if len(shape) != 2 or (shape[0] > 0 and shape[1] > 1 and strides[1] != 1):
        raise ValueError(f"{name}: expected a 2-D tensor whose rows are contiguous")
    rows, item = shape[0], t.element_size()
    row_bytes = shape[1] * item
    return rows, row_bytes, strides[0] * item if rows > 0 else row_bytes


def _check_bytes(t: torch.Tensor, name: str, shape) -> None:
    _require_gpu(name, t)
    if t.dtype != torch.uint8 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous uint8 {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")


def _check_msg_args(rows: int, iv: torch.Tensor, aad: Optional[torch.Tensor]) -> None:
    _check_bytes(iv, "iv", (rows, 12))
    if aad is not None:
        _require_gpu("aad", aad)
        if aad.dtype != torch.uint8 or aad.dim() != 2 or aad.shape[0] != rows or \
                (aad.shape[1] > 1 and aad.stride(1) != 1):
            raise ValueError("aad: expected uint8 [rows, a] with contiguous rows")


def gcm_seal(key: GcmKey, pt: torch.Tensor, iv: torch.Tensor, aad: Optional[torch.Tensor] = None,
             out=None, workspace: Optional[torch.Tensor] = None):
    """Seal each row of pt (a 2-D device tensor; rows are the messages) under
    iv uint8 [rows, 12] and aad uint8 [rows, a].  Returns (ct uint8 [rows,
    row_bytes], tag uint8 [rows, 16])."""
    lib = _lib.load()
    rows, row_bytes, ld = _rows_u8(pt, "pt")
    _check_msg_args(rows, iv, aad)
    dev = pt.device
    if out is None:
        ct = torch.empty((rows, row_bytes), dtype=torch.uint8, device=dev)
        tag = torch.empty((rows, 16), dtype=torch.uint8, device=dev)
    else:
        ct, tag = out
    na = 0 if aad is None else aad.shape[1]
    if workspace is None:
        workspace = torch.empty(max(gcm_workspace(rows, row_bytes), 1), dtype=torch.uint8, device=dev)
    check(lib.sph_gcm_seal(key.handle, pt.data_ptr(), ld, rows, row_bytes, iv.data_ptr(),
                           _ptr(aad), aad.stride(0) if aad is not None else 0, na,
                           ct.data_ptr(), ct.stride(0) * ct.element_size() if rows > 0 else row_bytes,
                           tag.data_ptr(), workspace.data_ptr(), workspace.numel(),
                           _stream_handle(dev)))
    return ct, tag


def gcm_open(key: GcmKey, ct: torch.Tensor, iv: torch.Tensor, tag: torch.Tensor,
             aad: Optional[torch.Tensor] = None, out=None, workspace: Optional[torch.Tensor] = None):
    """Open each row of ct; returns (pt uint8 [rows, row_bytes], ok int32
    [rows]): ok[m] = 1 when row m's tag verifies (use no row with ok 0)."""
    lib = _lib.load()
    rows, row_bytes, ld = _rows_u8(ct, "ct")
    _check_msg_args(rows, iv, aad)
    _check_bytes(tag, "tag", (rows, 16))
    dev = ct.device
    if out is None:
        pt = torch.empty((rows, row_bytes), dtype=torch.uint8, device=dev)
        ok = torch.empty((rows,), dtype=torch.int32, device=dev)
    else:
        pt, ok = out
    na = 0 if aad is None else aad.shape[1]
    if workspace is None:
        workspace = torch.empty(max(gcm_workspace(rows, row_bytes), 1), dtype=torch.uint8, device=dev)
    check(lib.sph_gcm_open(key.handle, ct.data_ptr(), ld, rows, row_bytes, iv.data_ptr(),
                           _ptr(aad), aad.stride(0) if aad is not None else 0, na, tag.data_ptr(),
                           pt.data_ptr(), pt.stride(0) * pt.element_size() if rows > 0 else row_bytes,
                           ok.data_ptr(), workspace.data_ptr(), workspace.numel(),
                           _stream_handle(dev)))
    return pt, ok


def _segment_array(ins, outs, rows: int, what: str):
    if not 1 <= len(ins) <= _lib.SPH_GCM_MAX_SEGMENTS or len(outs) != len(ins):
        raise ValueError(f"{what}: 1..{_lib.SPH_GCM_MAX_SEGMENTS} segments with one output each")
    arr = (_lib.GcmSegment * len(ins))()
    total = 0
    for k, (a, b) in enumerate(zip(ins, outs)):
        r, nb, ld = _rows_u8(a, f"{what} segment {k}")
        ro, nbo, ldo = _rows_u8(b, f"{what} output {k}")
        if r != rows or ro != rows or nbo != nb:
            raise ValueError(f"{what}: segment {k} is {r} x {nb} bytes, output {ro} x {nbo}, rows {rows}")
        arr[k] = _lib.GcmSegment(a.data_ptr(), ld, b.data_ptr(), ldo, nb)
        total += nb
    return arr, total


def gcm_seal_segments(key: GcmKey, segments, iv: torch.Tensor, aad: Optional[torch.Tensor] = None,
                      out=None, tag: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None):
    """Seal messages that are the concatenation of row m of each tensor in
    `segments` (2-D device tensors with the same number of rows, e.g. the
    payload codes and their scales).  Returns ([ct per segment, uint8, same
    rows x bytes], tag uint8 [rows, 16]); pass `out` (a list of uint8
    tensors, may be the inputs themselves) to write in place."""
    lib = _lib.load()
    segments = list(segments)
    rows = segments[0].shape[0] if segments else 0
    dev = segments[0].device if segments else torch.device("cuda")
    if out is None:
        out = [torch.empty((rows, _rows_u8(a, "segment")[1]), dtype=torch.uint8, device=dev)
               for a in segments]
    arr, total = _segment_array(segments, list(out), rows, "gcm_seal_segments")
    _check_msg_args(rows, iv, aad)
    if tag is None:
        tag = torch.empty((rows, 16), dtype=torch.uint8, device=dev)
    _check_bytes(tag, "tag", (rows, 16))
    na = 0 if aad is None else aad.shape[1]
    if workspace is None:
        workspace = torch.empty(max(gcm_workspace(rows, total), 1), dtype=torch.uint8, device=dev)
    check(lib.sph_gcm_seal_segments(key.handle, arr, len(segments), rows, iv.data_ptr(), _ptr(aad),
                                    aad.stride(0) if aad is not None else 0, na, tag.data_ptr(),
                                    workspace.data_ptr(), workspace.numel(), _stream_handle(dev)))
    return list(out), tag


def gcm_open_segments(key: GcmKey, segments, iv: torch.Tensor, tag: torch.Tensor,
                      aad: Optional[torch.Tensor] = None, out=None, ok: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None):
    """Open messages sealed by gcm_seal_segments; returns ([pt per segment],
    ok int32 [rows]) with ok[m] = 1 when message m's tag verifies."""
    lib = _lib.load()
    segments = list(segments)
    rows = segments[0].shape[0] if segments else 0
    dev = segments[0].device if segments else torch.device("cuda")
    if out is None:
        out = [torch.empty((rows, _rows_u8(a, "segment")[1]), dtype=torch.uint8, device=dev)
               for a in segments]
    arr, total = _segment_array(segments, list(out), rows, "gcm_open_segments")
    _check_msg_args(rows, iv, aad)
    _check_bytes(tag, "tag", (rows, 16))
    if ok is None:
        ok = torch.empty((rows,), dtype=torch.int32, device=dev)
    elif ok.dtype != torch.int32 or tuple(ok.shape) != (rows,) or not ok.is_cuda:
        raise ValueError(f"ok: expected int32 ({rows},) on the GPU")
    na = 0 if aad is None else aad.shape[1]
    if workspace is None:
        workspace = torch.empty(max(gcm_workspace(rows, total), 1), dtype=torch.uint8, device=dev)
    check(lib.sph_gcm_open_segments(key.handle, arr, len(segments), rows, iv.data_ptr(), _ptr(aad),
                                    aad.stride(0) if aad is not None else 0, na, tag.data_ptr(),
                                    ok.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                    _stream_handle(dev)))
    return list(out), ok


def ctypes_vp():
    return _lib.c_vp()


def cloud_partial_workspace(M: int, subset: Subset) -> int:
    return int(_lib.load().sph_cloud_partial_workspace(int(M), subset.handle))


def fuse_verify_workspace(M: int, subset: Subset, mode: int = GREEDY) -> int:
    return int(_lib.load().sph_fuse_verify_workspace(int(M), subset.handle, int(mode)))


def payload_code_bytes(n: int, bits: int = 8) -> int:
    """Bytes of one payload row's codes (include/sph.h)."""
    return int(_lib.load().sph_payload_code_bytes(int(n), int(bits)))


def payload_scale_count(n: int, block: int = 0) -> int:
    """Scales of one payload row (include/sph.h)."""
    return int(_lib.load().sph_payload_scale_count(int(n), int(block)))


def cloud_partial(h_cloud: torch.Tensor, w_cloud: torch.Tensor, subset: Subset, clip_c: float,
                  w_row_scale: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                  want_z: bool = False, workspace: Optional[torch.Tensor] = None, out=None,
                  bits: int = 8, block: int = 0):
    """Cloud half: returns (q, scale, z fp32 [M, n] or None).

    h_cloud: bf16 [M, d_cloud] view (rows may be strided, e.g. h[:, d_end:]).
    w_cloud: bf16 [V, d_cloud] or fp8 E4M3 (torch.float8_e4m3fn / uint8) with
    w_row_scale fp32 [V].
    Payload format (bits, block): q is int8 [M, n] for 8-bit codes, uint8
    [M, ceil(n/2)] (two codes per byte) for 4-bit codes; scale is fp32 [M]
    for one scale per row (block 0), else [M, ceil(n / block)].
    """
    lib = _lib.load()
    _require_gpu("h_cloud", h_cloud)
    _require_gpu("w_cloud", w_cloud)
    h_cloud = _as_bits16(h_cloud)
    if w_cloud.dtype in (torch.bfloat16, torch.int16, torch.uint16):
        wtype = _lib.SPH_W_BF16
    elif w_cloud.dtype in (torch.float8_e4m3fn, torch.uint8):
        wtype = _lib.SPH_W_FP8_E4M3
    else:
        raise TypeError(f"unsupported weight dtype {w_cloud.dtype}")
    M, d_cloud = h_cloud.shape
    dev = h_cloud.device
    if out is None:
        nb = payload_scale_count(subset.n, block)
        if bits == 8:
            q = torch.empty((M, subset.n), dtype=torch.int8, device=dev)
        else:
            q = torch.empty((M, max(payload_code_bytes(subset.n, bits), 0)), dtype=torch.uint8, device=dev)
        scale = torch.empty((M,) if block == 0 else (M, max(nb, 0)), dtype=torch.float32, device=dev)
        z = torch.empty((M, subset.n), dtype=torch.float32, device=dev) if want_z else None
    else:
        q, scale, z = out
    if workspace is None:
        need = cloud_partial_workspace(M, subset)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    check(lib.sph_cloud_partial_fmt(
        h_cloud.data_ptr(), h_cloud.stride(0) if M > 0 else d_cloud, M, d_cloud,
        w_cloud.data_ptr(), w_cloud.stride(0), wtype, _ptr(w_row_scale),
        _ptr(bias), subset.handle, float(clip_c), int(bits), int(block),
        q.data_ptr(), scale.data_ptr(), _ptr(z),
        workspace.data_ptr(), workspace.numel(), _stream_handle(dev)))
    return q, scale, z


NOALLOC_SCRATCH_BYTES = 16 << 20


def cloud_partial_noalloc(h_cloud: torch.Tensor, w_cloud: torch.Tensor, subset: Subset,
                          clip_c: float, out, w_row_scale: Optional[torch.Tensor] = None,
                          bias: Optional[torch.Tensor] = None, bits: int = 8, block: int = 0):
    """cloud_partial without a workspace: the library's static device scratch
    (NOALLOC_SCRATCH_BYTES per GPU) stands in for it.  `out` = (q, scale, z or
    None) must be given; nothing is allocated.  Calls that overlap on one GPU
    race (they share the scratch)."""
    lib = _lib.load()
    _require_gpu("h_cloud", h_cloud)
    _require_gpu("w_cloud", w_cloud)
    h_cloud = _as_bits16(h_cloud)
    if w_cloud.dtype in (torch.bfloat16, torch.int16, torch.uint16):
        wtype = _lib.SPH_W_BF16
    elif w_cloud.dtype in (torch.float8_e4m3fn, torch.uint8):
        wtype = _lib.SPH_W_FP8_E4M3
    else:
        raise TypeError(f"unsupported weight dtype {w_cloud.dtype}")
    M, d_cloud = h_cloud.shape
    q, scale, z = out
    check(lib.sph_cloud_partial_noalloc(
        h_cloud.data_ptr(), h_cloud.stride(0) if M > 0 else d_cloud, M, d_cloud,
        w_cloud.data_ptr(), w_cloud.stride(0), wtype, _ptr(w_row_scale),
        _ptr(bias), subset.handle, float(clip_c), int(bits), int(block),
        q.data_ptr(), scale.data_ptr(), _ptr(z), _stream_handle(h_cloud.device)))
    return q, scale, z


def fuse_verify(q: torch.Tensor, scale: torch.Tensor, h_end: Optional[torch.Tensor],
                w_end: Optional[torch.Tensor], subset: Subset, n_sessions: int,
                rows_per_session: int, drafts: Optional[torch.Tensor], mode: int = GREEDY,
                temperature: float = 1.0, top_p: float = 1.0, seed: int = 0,
                want_fused: bool = False, workspace: Optional[torch.Tensor] = None, out=None,
                bits: int = 8, block: int = 0):
    """Endpoint half: returns (tokens int32 [M], accept_len int32 [S], fused fp32 or None).
    (q, scale) is a payload of cloud_partial in format (bits, block)."""
    lib = _lib.load()
    dev = q.device
    M = int(n_sessions) * int(rows_per_session)
    if h_end is not None and h_end.shape[1] > 0:
        _require_gpu("h_end", h_end)
        _require_gpu("w_end", w_end)
        h_end = _as_bits16(h_end)
        w_end = _as_bits16(w_end)
        d_end = h_end.shape[1]
        hp, ldh, wp, ldw = h_end.data_ptr(), h_end.stride(0), w_end.data_ptr(), w_end.stride(0)
    else:
        d_end, hp, ldh, wp, ldw = 0, None, 0, None, 0
    if out is None:
        tokens = torch.empty((M,), dtype=torch.int32, device=dev)
        accept = torch.empty((int(n_sessions),), dtype=torch.int32, device=dev)
        fused = torch.empty((M, subset.n), dtype=torch.float32, device=dev) if want_fused else None
    else:
        tokens, accept, fused = out
    if workspace is None:
        need = fuse_verify_workspace(M, subset, mode)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    check(lib.sph_fuse_verify_fmt(
        q.data_ptr(), scale.data_ptr(), int(bits), int(block), hp, ldh, d_end, wp, ldw, subset.handle,
        int(n_sessions), int(rows_per_session), _ptr(drafts),
        int(mode), float(temperature), float(top_p), int(seed) & 0xFFFFFFFFFFFFFFFF,
        tokens.data_ptr(), accept.data_ptr(), _ptr(fused),
        workspace.data_ptr(), workspace.numel(), _stream_handle(dev)))
    return tokens, accept, fused


def hidden_quantize(h: torch.Tensor, out=None):
    """Per-row int8 codes of bf16 hidden rows h [M, d] (rows may be strided):
    returns (codes int8 [M, d], scales fp32 [M])."""
    lib = _lib.load()
    _require_gpu("h", h)
    h = _as_bits16(h)
    M, d = h.shape
    if out is None:
        hq = torch.empty((M, d), dtype=torch.int8, device=h.device)
        hs = torch.empty((M,), dtype=torch.float32, device=h.device)
    else:
        hq, hs = out
    check(lib.sph_hidden_quantize(h.data_ptr(), h.stride(0) if M > 0 else d, M, d, hq.data_ptr(),
                                  hq.stride(0) if M > 0 else d, hs.data_ptr(),
                                  _stream_handle(h.device)))
    return hq, hs


def fuse_verify_hq_workspace(M: int, d_end: int, subset: Subset, mode: int = GREEDY) -> int:
    return int(_lib.load().sph_fuse_verify_hq_workspace(int(M), int(d_end), subset.handle, int(mode)))


def fuse_verify_hq(q: torch.Tensor, scale: torch.Tensor, hq: torch.Tensor, h_scale: torch.Tensor,
                   d_end: int, w_end: Optional[torch.Tensor], subset: Subset, n_sessions: int,
                   rows_per_session: int, drafts: Optional[torch.Tensor], mode: int = GREEDY,
                   temperature: float = 1.0, top_p: float = 1.0, seed: int = 0,
                   want_fused: bool = False, workspace: Optional[torch.Tensor] = None, out=None,
                   bits: int = 8, block: int = 0):
    """Endpoint half on hidden-state codes: hq int8 [M, >= d_end] and h_scale
    fp32 [M] from hidden_quantize; the first d_end columns enter eq. 11.
    Returns (tokens int32 [M], accept_len int32 [S], fused fp32 or None)."""
    lib = _lib.load()
    dev = q.device
    M = int(n_sessions) * int(rows_per_session)
    d_end = int(d_end)
    if d_end > 0:
        _require_gpu("hq", hq)
        if hq.dtype != torch.int8 or hq.dim() != 2 or hq.shape[0] != M or hq.shape[1] < d_end or \
                hq.stride(1) != 1:
            raise ValueError(f"hq: expected int8 [{M}, >= {d_end}] with contiguous rows")
        if h_scale.dtype != torch.float32 or tuple(h_scale.shape) != (M,) or not h_scale.is_contiguous():
            raise ValueError(f"h_scale: expected contiguous float32 [{M}]")
        _require_gpu("w_end", w_end)
        w_end = _as_bits16(w_end)
        hp, ldh, sp = hq.data_ptr(), hq.stride(0), h_scale.data_ptr()
        wp, ldw = w_end.data_ptr(), w_end.stride(0)
    else:
        hp, ldh, sp, wp, ldw = None, 0, None, None, 0
    if out is None:
        tokens = torch.empty((M,), dtype=torch.int32, device=dev)
        accept = torch.empty((int(n_sessions),), dtype=torch.int32, device=dev)
        fused = torch.empty((M, subset.n), dtype=torch.float32, device=dev) if want_fused else None
    else:
        tokens, accept, fused = out
    if workspace is None:
        need = fuse_verify_hq_workspace(M, d_end, subset, mode)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    check(lib.sph_fuse_verify_hq(
        q.data_ptr(), scale.data_ptr(), int(bits), int(block), hp, ldh, sp, d_end, wp, ldw,
        subset.handle, int(n_sessions), int(rows_per_session), _ptr(drafts),
        int(mode), float(temperature), float(top_p), int(seed) & 0xFFFFFFFFFFFFFFFF,
        tokens.data_ptr(), accept.data_ptr(), _ptr(fused),
        workspace.data_ptr(), workspace.numel(), _stream_handle(dev)))
    return tokens, accept, fused


class KvCache:
    """A paged 4-bit key/value cache (include/sph.h) on tensors of the caller:

    pool  uint8 [layers, pages, >= kv_page_bytes], pages contiguous
    table int32 [slots, max_pages], -1 where there is no page
    lens  int32 [slots] tokens held, refs int32 [pages] slots that hold a page

    The tensors are kept alive, and changed in place by the calls below, which go by
    the addresses and sizes of when the cache was made: its attributes are fixed."""

    def __init__(self, pool: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, refs: torch.Tensor,
                 kv_heads: int, head_dim: int, page_tokens: int):
        import ctypes
        for name, t, dims, dtype in (("pool", pool, 3, torch.uint8), ("table", table, 2, torch.int32),
                                     ("lens", lens, 1, torch.int32), ("refs", refs, 1, torch.int32)):
            _require_gpu(name, t)
            if t.dtype != dtype or t.dim() != dims or t.device != pool.device:
                raise ValueError(f"{name}: expected {dtype} with {dims} dimensions on the pool's device, "
                                 f"got {t.dtype} {tuple(t.shape)} on {t.device}")
        need = kv_page_bytes(kv_heads, head_dim, page_tokens)
        if pool.shape[2] < need:
            raise ValueError(f"pool: pages of {pool.shape[2]} bytes, need {need}")
        if lens.shape[0] != table.shape[0] or refs.shape[0] != pool.shape[1]:
            raise ValueError(f"lens {tuple(lens.shape)} and refs {tuple(refs.shape)} do not fit table "
                             f"{tuple(table.shape)} and pool {tuple(pool.shape)}")
        self.pool, self.table, self.lens, self.refs = pool, table, lens, refs
        self.kv_heads, self.head_dim, self.page_tokens = int(kv_heads), int(head_dim), int(page_tokens)
        self.layers, self.n_pages, self.n_slots = pool.shape[0], pool.shape[1], table.shape[0]
        self.device = pool.device
        self._struct = _lib.KvCacheStruct(
            pool.data_ptr(), pool.shape[0], pool.stride(0), pool.shape[1], pool.stride(1),
            table.data_ptr(), table.stride(0), table.shape[1], lens.data_ptr(), refs.data_ptr(),
            table.shape[0], self.kv_heads, self.head_dim, self.page_tokens)
        self.ptr = ctypes.addressof(self._struct)
        lib = _lib.load()
        self._grow_bytes, self._compact_bytes = (lib.sph_pages_grow_workspace(self.ptr),
                                                 lib.sph_pages_compact_workspace(self.ptr))
        self._fixed = frozenset(self.__dict__)

    def __setattr__(self, name, value):
        if name in self.__dict__.get("_fixed", ()):
            raise AttributeError(f"KvCache.{name} is fixed: make another cache, or change the tensor in place")
        super().__setattr__(name, value)

    @classmethod
    def empty(cls, layers: int, n_pages: int, n_slots: int, max_pages: int, kv_heads: int,
              head_dim: int, page_tokens: int, device=None) -> "KvCache":
        """An empty cache with tensors of its own."""
        dev = torch.device("cuda") if device is None else torch.device(device)
        nb = kv_page_bytes(kv_heads, head_dim, page_tokens)
        return cls(torch.empty((layers, n_pages, nb), dtype=torch.uint8, device=dev),
                   torch.full((n_slots, max_pages), -1, dtype=torch.int32, device=dev),
                   torch.zeros((n_slots,), dtype=torch.int32, device=dev),
                   torch.zeros((n_pages,), dtype=torch.int32, device=dev), kv_heads, head_dim, page_tokens)


def kv_page_bytes(kv_heads: int, head_dim: int, page_tokens: int) -> int:
    """Bytes of one page of one layer (include/sph.h)."""
    n = int(_lib.load().sph_kv_page_bytes(int(kv_heads), int(head_dim), int(page_tokens)))
    if n < 0:
        raise SphError(_lib.SPH_E_UNSUPPORTED, f"no cache of kv_heads={kv_heads} head_dim={head_dim} "
                                               f"page_tokens={page_tokens}")
    return n


def _kv_rows(name: str, t: torch.Tensor, heads: Optional[int], d: int, device):
    """Row and head strides of a bf16 [M, heads, d] tensor."""
    shape = t.shape
    if t.dtype != torch.bfloat16 or len(shape) != 3 or shape[2] != d or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name}: expected bf16 [rows, {'heads' if heads is None else heads}, {d}], "
                         f"got {t.dtype} {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the cache on {device}")
    row, head, one = t.stride()
    if one != 1:
        raise ValueError(f"{name} must be contiguous along its last dimension")
    # strides of axes of length one or none mean nothing
    return row if shape[0] > 1 else max(row, d), head if shape[1] > 1 else max(head, d)


def _kv_ints(name: str, t: Optional[torch.Tensor], n: int, device) -> Optional[int]:
    if t is None:
        return None
    if t.dtype != torch.int32 or t.shape != (n,) or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous int32 ({n},) on {device}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _kv_workspace(t: torch.Tensor, device):
    """Address and bytes of a workspace of the caller's."""
    if t.device != device or not t.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous tensor on {device}, got one "
                         f"on {t.device} with strides {t.stride()}")
    return t.data_ptr(), t.numel() * t.element_size()


def _kv_sessions(M: int, R: int) -> int:
    if R < 1 or M % R != 0:
        raise ValueError(f"{M} rows are no whole number of sessions of {R}")
    return M // R


def kv_append(cache: KvCache, layer: int, k: torch.Tensor, v: torch.Tensor, rows_per_session: int,
              rows: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None) -> None:
    """Quantise the rows k, v bf16 [sessions * R, kv_heads, head_dim] (rows and
    heads may be strided) into their pages: row r of a session stands at position
    lens - rows + r of its slot, so pages_grow comes first.  rows int32
    [sessions]: rows of each (R if None); slots int32 [sessions]: where each is
    (0, 1, ... if None)."""
    R, dev = int(rows_per_session), cache.device
    ks = _kv_rows("k", k, cache.kv_heads, cache.head_dim, dev)
    vs = _kv_rows("v", v, cache.kv_heads, cache.head_dim, dev)
    if k.shape[0] != v.shape[0]:
        raise ValueError(f"k has {k.shape[0]} rows, v {v.shape[0]}")
    n = _kv_sessions(k.shape[0], R)
    check(_lib.load().sph_kv_append(cache.ptr, int(layer), k.data_ptr(), *ks, v.data_ptr(), *vs, n, R,
                                    _kv_ints("rows", rows, n, dev), _kv_ints("slots", slots, n, dev),
                                    _stream_handle(dev)))


def kv_read(cache: KvCache, layer: int, rows_per_session: int, rows: Optional[torch.Tensor] = None,
            slots: Optional[torch.Tensor] = None, n_sessions: Optional[int] = None, out=None):
    """The same rows as the values that the cache holds: (k, v) bf16 [sessions *
    R, kv_heads, head_dim], zeros past a session's rows.  n_sessions: all slots
    (or all of `rows` or `slots`) if None."""
    R, dev = int(rows_per_session), cache.device
    n = n_sessions
    if n is None:
        given = rows if rows is not None else slots
        n = cache.n_slots if given is None else given.shape[0]
    heads, d = cache.kv_heads, cache.head_dim
    if out is None:
        k = torch.empty((int(n) * R, heads, d), dtype=torch.bfloat16, device=dev)
        v = torch.empty_like(k)
        ks = vs = heads * d, d
    else:
        k, v = out
        ks, vs = _kv_rows("k", k, heads, d, dev), _kv_rows("v", v, heads, d, dev)
        if k.shape[0] != n * R or v.shape[0] != n * R:
            raise ValueError(f"out: expected {n * R} rows, got {k.shape[0]} and {v.shape[0]}")
    check(_lib.load().sph_kv_read(cache.ptr, int(layer), k.data_ptr(), *ks, v.data_ptr(), *vs, int(n), R,
                                  _kv_ints("rows", rows, n, dev), _kv_ints("slots", slots, n, dev),
                                  _stream_handle(dev)))
    return k, v


def kv_attend_workspace(cache: KvCache, q_heads: int, n_sessions: int, rows_per_session: int,
                        window: int = 0, max_len: int = 0) -> int:
    return int(_lib.load().sph_kv_attend_workspace(cache.ptr, int(q_heads), int(n_sessions),
                                                   int(rows_per_session), int(window), int(max_len)))


def kv_attend(cache: KvCache, layer: int, q: torch.Tensor, rows_per_session: int, scale: float,
              rows: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None, window: int = 0,
              max_len: int = 0, want_lse: bool = False, workspace: Optional[torch.Tensor] = None, out=None):
    """Attention of each session's last rows over its cache, the rows' own tokens
    among it (kv_append comes first).  q bf16 [sessions * R, q_heads, head_dim]
    (rows and heads may be strided), q_heads a multiple of kv_heads.  Returns
    (out bf16 [sessions * R, q_heads, head_dim], log-sum-exp fp32 [sessions * R,
    q_heads] or None).  max_len: the longest session, if the caller knows it (the
    work is shared out better); window: positions a row sees (0: all before it).
    out: (out, log-sum-exp or None) to write to; want_lse makes the second where it
    is None."""
    lib = _lib.load()
    R, dev = int(rows_per_session), cache.device
    qs = _kv_rows("q", q, None, cache.head_dim, dev)
    M, heads = q.shape[0], q.shape[1]
    n = _kv_sessions(M, R)
    d = cache.head_dim
    if out is None:
        o, lse = torch.empty_like(q) if q.is_contiguous() else q.new_empty((M, heads, d)), None
        os = heads * d, d
    else:
        o, lse = out
        os = _kv_rows("out", o, heads, d, dev)
        if o.shape[0] != M:
            raise ValueError(f"out: expected {M} rows, got {o.shape[0]}")
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != (M, heads) or not lse.is_contiguous()
                                or lse.device != dev):
            raise ValueError(f"lse: expected contiguous float32 ({M}, {heads}) on {dev}")
    if lse is None and want_lse:
        lse = torch.empty((M, heads), dtype=torch.float32, device=dev)
    if workspace is None:
        need = kv_attend_workspace(cache, heads, n, R, window, max_len)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
        ws = _ptr(workspace), need
    else:
        ws = _kv_workspace(workspace, dev)
    check(lib.sph_kv_attend(cache.ptr, int(layer), q.data_ptr(), *qs, heads, n, R,
                            _kv_ints("rows", rows, n, dev), _kv_ints("slots", slots, n, dev),
                            float(scale), int(window), int(max_len), o.data_ptr(), *os, _ptr(lse),
                            *ws, _stream_handle(dev)))
    return o, lse


def pages_grow(cache: KvCache, add: torch.Tensor, workspace: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """lens += add (int32 [slots]), with pages for the new tokens; a shared page
    that they begin in is copied first.  Returns the status, int32 [2]: pages
    lacking in the pool, slots whose row is too short; if either is not 0,
    nothing has changed."""
    lib = _lib.load()
    dev = cache.device
    status = torch.empty(2, dtype=torch.int32, device=dev) if out is None else out
    if workspace is None:
        workspace = torch.empty(cache._grow_bytes, dtype=torch.uint8, device=dev)
        ws = workspace.data_ptr(), cache._grow_bytes
    else:
        ws = _kv_workspace(workspace, dev)
    check(lib.sph_pages_grow(cache.ptr, _kv_ints("add", add, cache.n_slots, dev), _kv_ints("out", status, 2, dev),
                             *ws, _stream_handle(dev)))
    return status


def pages_trim(cache: KvCache, kept: torch.Tensor) -> None:
    """lens = min(lens, kept) (int32 [slots]); pages past that are given back."""
    dev = cache.device
    check(_lib.load().sph_pages_trim(cache.ptr, _kv_ints("kept", kept, cache.n_slots, dev), _stream_handle(dev)))


def pages_fork(cache: KvCache, parents: torch.Tensor, children: torch.Tensor) -> None:
    """Slots children[i] give back what they hold and share the pages of slots
    parents[i] (int32 [n]; children distinct, none of them a parent)."""
    n, dev = parents.shape[0], cache.device
    check(_lib.load().sph_pages_fork(cache.ptr, _kv_ints("parents", parents, n, dev),
                                     _kv_ints("children", children, n, dev), n, _stream_handle(dev)))


def pages_copy(cache: KvCache, src: torch.Tensor, dst: torch.Tensor) -> None:
    """Pages dst[i] become copies of pages src[i] in every layer (int32 [n])."""
    n, dev = src.shape[0], cache.device
    check(_lib.load().sph_pages_copy(cache.ptr, _kv_ints("src", src, n, dev), _kv_ints("dst", dst, n, dev), n,
                                     _stream_handle(dev)))


def pages_compact(cache: KvCache, out=None, workspace: Optional[torch.Tensor] = None):
    """Move the live pages to the front of the pool.  Returns (table, refs, live
    int32 [1]): the cache's own, changed in place, or `out` = (table, refs)."""
    lib = _lib.load()
    dev = cache.device
    table, refs = (cache.table, cache.refs) if out is None else out
    _require_gpu("table", table)
    if table.dtype != torch.int32 or table.shape != cache.table.shape or table.device != dev:
        raise ValueError(f"table: expected int32 {tuple(cache.table.shape)} on {dev}")
    live = torch.empty(1, dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = torch.empty(cache._compact_bytes, dtype=torch.uint8, device=dev)
        ws = workspace.data_ptr(), cache._compact_bytes
    else:
        ws = _kv_workspace(workspace, dev)
    check(lib.sph_pages_compact(cache.ptr, table.data_ptr(), table.stride(0), _kv_ints("refs", refs, cache.n_pages, dev),
                                live.data_ptr(), *ws, _stream_handle(dev)))
    return table, refs, live


def debug_sync(enable: Optional[bool] = None) -> bool:
    """Switch the library's debug synchronisation (a stream synchronisation
    and error check after every kernel launch region) on or off; None only
    queries.  Returns the previous state."""
    return bool(_lib.load().sph_debug_sync(-1 if enable is None else int(bool(enable))))


def trace_start(capacity: int) -> None:
    """Record HIP events around the next `capacity` kernel launches."""
    check(_lib.load().sph_trace_start(int(capacity)))


def trace_collect(capacity: int):
    """Stop tracing and return [(kernel name, milliseconds)] in launch order."""
    import ctypes
    lib = _lib.load()
    recs = (_lib.TraceRecord * int(capacity))()
    n = ctypes.c_int(0)
    check(lib.sph_trace_stop(recs, int(capacity), n))
    return [(recs[i].kernel.decode(), float(recs[i].ms)) for i in range(min(n.value, capacity))]


def probe_read(buf: torch.Tensor, sink: torch.Tensor) -> None:
    """Enqueue one streaming read of all of `buf` (measurement helper of
    include/sph_probe.h); time it with events on the current stream."""
    _require_gpu("buf", buf)
    _require_gpu("sink", sink)
    check(_lib.load().sph_probe_read(buf.data_ptr(), buf.numel() * buf.element_size(),
                                     sink.data_ptr(), _stream_handle(buf.device)))


def probe_mfma(iters: int, sink: torch.Tensor) -> float:
    """Enqueue one bf16 MFMA loop of `iters` iterations (measurement helper of
    include/sph_probe.h) and return its floating-point operation count."""
    import ctypes
    _require_gpu("sink", sink)
    flops = ctypes.c_double(0.0)
    check(_lib.load().sph_probe_mfma(int(iters), sink.data_ptr(), _stream_handle(sink.device),
                                     ctypes.byref(flops)))
    return flops.value
