"""Paged key/value cache and residual verification on torch CUDA tensors (argument marshalling only)."""
from __future__ import annotations

import ctypes as C
import struct
from dataclasses import dataclass
from typing import Optional

from .binding import DT_BF16, DT_F16, DT_F32, WisvError, _check, load_library


class _CacheConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_heads", "n_kv_heads", "head_dim", "page_size", "n_pages", "max_requests",
                                         "max_blocks", "dtype")] + [("workspace", C.c_void_p),
                                                                    ("workspace_bytes", C.c_int64)]


class _Pages(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("free_list", "n_free", "block_table", "n_blocks", "seq_len")]


class _Layout(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q_off", "kv_len", "slot_map", "positions", "status")]


class _Append(C.Structure):
    _fields_ = [("T", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64), ("v_token_stride", C.c_int64),
                ("v_head_stride", C.c_int64), ("k_pages", C.c_void_p), ("v_pages", C.c_void_p),
                ("kp_page_stride", C.c_int64), ("kp_token_stride", C.c_int64), ("kp_head_stride", C.c_int64),
                ("vp_page_stride", C.c_int64), ("vp_token_stride", C.c_int64), ("vp_head_stride", C.c_int64),
                ("slot_map", C.c_void_p)]


class _Attend(C.Structure):
    _fields_ = [("B", C.c_int32), ("T", C.c_int32), ("max_new", C.c_int32), ("q_off", C.c_void_p),
                ("kv_len", C.c_void_p), ("block_table", C.c_void_p), ("table_stride", C.c_int64),
                ("max_blocks", C.c_int32), ("q", C.c_void_p), ("q_token_stride", C.c_int64),
                ("q_head_stride", C.c_int64), ("k_pages", C.c_void_p), ("v_pages", C.c_void_p),
                ("kp_page_stride", C.c_int64), ("kp_token_stride", C.c_int64), ("kp_head_stride", C.c_int64),
                ("vp_page_stride", C.c_int64), ("vp_token_stride", C.c_int64), ("vp_head_stride", C.c_int64),
                ("out", C.c_void_p), ("o_token_stride", C.c_int64), ("o_head_stride", C.c_int64), ("lse", C.c_void_p),
                ("scale", C.c_float), ("clear_rest", C.c_int32)]


class _Residual(C.Structure):
    _fields_ = [("B", C.c_int32), ("K", C.c_int32), ("k_off", C.c_void_p), ("T_total", C.c_int32), ("V", C.c_int32),
                ("target_probs", C.c_void_p), ("target_stride", C.c_int64), ("target_dtype", C.c_int32),
                ("draft_tokens", C.c_void_p), ("draft_probs", C.c_void_p), ("draft_stride", C.c_int64),
                ("draft_dtype", C.c_int32), ("draft_ids", C.c_void_p), ("n_top", C.c_int32), ("uniforms", C.c_void_p),
                ("u_draw", C.c_void_p), ("accept_in", C.c_void_p), ("accept_len", C.c_void_p), ("token", C.c_void_p),
                ("mass", C.c_void_p), ("status", C.c_void_p)]


def _packer(cls):
    """struct.Struct of a ctypes structure's layout: filling 25 fields takes 0.5 us that way, 4 us through ctypes."""
    code = {C.c_int32: "i", C.c_int64: "q", C.c_void_p: "P", C.c_float: "f"}
    s = struct.Struct("@" + "".join(code[t] for _, t in cls._fields_) + "0q")
    assert s.size == C.sizeof(cls)
    return s.pack


_pack_layout, _pack_append, _pack_attend, _pack_residual = (_packer(c) for c in (_Layout, _Append, _Attend, _Residual))
_declared = False


def _lib():
    global _declared
    lib = load_library()
    if not _declared:
        P, I = C.c_void_p, C.c_int32                           # argument blocks go as packed bytes
        for name, args in (("wisv_cache_create", [C.POINTER(_CacheConfig), C.POINTER(P)]), ("wisv_cache_destroy", [P]),
                           ("wisv_cache_workspace", [C.POINTER(_CacheConfig), C.POINTER(C.c_int64)]),
                           ("wisv_cache_error", [P, P, C.POINTER(I)]),
                           ("wisv_cache_extend", [P, P, I, I, P, I, P, P]), ("wisv_cache_commit", [P, P, I, P, P, P]),
                           ("wisv_cache_append", [P, P, P]), ("wisv_cache_attend", [P, P, P]),
                           ("wisv_debug_cache_waits", [P, C.c_uint64, I]),
                           ("wisv_verify_residual", [P, P])):
            f = getattr(lib, name)
            f.restype, f.argtypes = C.c_int, args
        lib.wisv_cache_launch_count.restype = C.c_int64
        lib.wisv_cache_launch_count.argtypes = [P]
        _declared = True
    return lib


def _array(what, t, dtype, n, index):
    """Address of a contiguous tensor of the documented type, at least the documented size and on device `index`."""
    if t.dtype is dtype and t.get_device() == index and t.numel() >= n and t.is_contiguous():
        return t.data_ptr()
    raise ValueError("%s must be a contiguous %s tensor with %d entries on cuda:%d" % (what, dtype, n, index))


def _row_stride(t) -> int:
    """Elements from one row of a 2-D tensor to the next (a single row has none of its own)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _empty(torch, stream, shape, dtype, device):
    """torch.empty for a result that `stream` (None: the current one) writes."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _full(torch, stream, shape, value, dtype, device):
    """torch.full on `stream` (None: the current one)."""
    with torch.cuda.stream(stream):
        return torch.full(shape, value, dtype=dtype, device=device)


@dataclass
class WindowLayout:
    """What PagedCache.extend lays out for a round (see wisv_layout)."""
    q_off: "object"
    kv_len: "object"
    slot_map: "object"
    positions: "object"
    status: "object"


def _owned_array(i):
    """A cache's i-th bookkeeping array as an attribute that can be written in place (``+=`` included) but not replaced."""
    def get(self):
        return self._owned[i]

    def put(self, value):
        if value is not self._owned[i]:
            raise AttributeError("the library holds this array's address: write into it (copy_) instead of replacing it")
    return property(get, put)


class PagedCache:
    """wisv_cache_* on torch CUDA tensors: the paged key/value cache of a target model.

    The bookkeeping tensors (``free_list``, ``n_free``, ``block_table``, ``n_blocks``, ``seq_len``) are ordinary int32
    tensors of this object, with every page free at the start, to be written in place, not replaced.  The page pools of each
    layer are the caller's: ``k_pages`` / ``v_pages`` of shape [n_pages, page_size, n_kv_heads, head_dim] with any strides
    that keep a head's elements contiguous (a [n_pages, n_kv_heads, page_size, head_dim] pool is passed as
    ``.transpose(1, 2)``).
    Request b of a call is row b of ``block_table``.  Calls are asynchronous on the current (or given) torch
    stream and must be ordered on it; they share the object's workspace.
    """

    def __init__(self, *, n_heads: int, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, max_requests: int,
                 max_blocks: int, dtype: int = DT_BF16, device="cuda:0"):
        import torch
        self._torch = torch
        self.lib = _lib()
        device = torch.device(device)
        if device.type != "cuda":
            raise ValueError("the paged cache lives on a CUDA device")
        self.device = torch.device("cuda", torch.cuda.current_device() if device.index is None else device.index)
        cfg = _CacheConfig(n_heads, n_kv_heads, head_dim, page_size, n_pages, max_requests, max_blocks, dtype)
        h, need = C.c_void_p(), C.c_int64()
        with torch.cuda.device(self.device):
            _check(self.lib.wisv_cache_workspace(C.byref(cfg), C.byref(need)), "wisv_cache_create")
            self._workspace = torch.empty(need.value, dtype=torch.uint8, device=self.device)
            cfg.workspace, cfg.workspace_bytes = self._workspace.data_ptr(), need.value
            # (the allocator orders the memory on the current stream, the library clears it on the default one)
            torch.cuda.current_stream(self.device).synchronize()
            _check(self.lib.wisv_cache_create(C.byref(cfg), C.byref(h)), "wisv_cache_create")
        self._h = h
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim
        self.page_size, self.n_pages, self.max_requests, self.max_blocks = page_size, n_pages, max_requests, max_blocks
        self.dtype = torch.bfloat16 if dtype == DT_BF16 else torch.float16
        i32 = dict(dtype=torch.int32, device=self.device)
        # every call works on these arrays: the block holds their addresses, and the attributes cannot be set
        self._owned = (torch.arange(n_pages - 1, -1, -1, **i32), torch.full((1,), n_pages, **i32),
                       torch.full((max_requests, max_blocks), -1, **i32), torch.zeros(max_requests, **i32),
                       torch.zeros(max_requests, **i32))
        self._pages = _Pages(*(t.data_ptr() for t in self._owned))
        self._pages_at = C.addressof(self._pages)
        self._index = self.device.index
        self._row = (n_kv_heads, head_dim)
        self._pool = (n_pages, page_size, n_kv_heads, head_dim)
        self._raw_stream, self._current = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice

    free_list, n_free, block_table, n_blocks, seq_len = (_owned_array(i) for i in range(5))

    def close(self):
        if getattr(self, "_h", None):
            self._torch.cuda.synchronize(self.device)
            self.lib.wisv_cache_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------------ helpers
    def _call(self, name, stream, *args):
        """One library call with this cache's device current; the stream goes last."""
        index = self._index
        st = self._raw_stream(index) if stream is None else stream.cuda_stream
        if self._current() != index:
            with self._torch.cuda.device(self.device):
                rc = getattr(self.lib, name)(self._h, *args, st)
        else:
            rc = getattr(self.lib, name)(self._h, *args, st)
        if rc:
            raise WisvError(rc, name)

    def _rows(self, what, t, heads, rows=None):
        """(address, token stride, head stride, rows) of [rows, heads, head_dim] rows."""
        shape = t.shape
        if len(shape) == 3 and t.dtype is self.dtype and t.get_device() == self._index:
            n, h, d = shape
            a, b, c = t.stride()
            if h == heads and d == self.head_dim and c == 1 and (rows is None or n == rows):
                return t.data_ptr(), a, b, n
        raise ValueError("%s must be [%s, %d, %d] %s on %s with a head's elements contiguous" %
                         (what, "T" if rows is None else rows, heads, self.head_dim, self.dtype, self.device))

    def _pages_of(self, what, t):
        """(address, page stride, token stride, head stride) of a page pool."""
        if t.shape == self._pool and t.dtype is self.dtype and t.get_device() == self._index:
            a, b, c, d = t.stride()
            if d == 1:
                return t.data_ptr(), a, b, c
        raise ValueError("%s must be [%d, %d, %d, %d] %s on %s with a head's elements contiguous" %
                         ((what,) + self._pool + (self.dtype, self.device)))

    # ------------------------------------------------------------------ calls
    def extend(self, *, B: int, n_new, T: Optional[int] = None, out: Optional[WindowLayout] = None,
               stream=None) -> WindowLayout:
        """wisv_cache_extend: pages, slots and positions for n_new tokens per request (an int, or int32 [B] on the
        device with their sum T given)."""
        torch, dev = self._torch, self._index
        i32, i64 = torch.int32, torch.int64
        uniform = isinstance(n_new, int)
        if T is None:
            if not uniform:
                raise ValueError("T, the sum of n_new, must be given where n_new lives on the device")
            T = B * n_new
        ptr = None if uniform else _array("n_new", n_new, i32, B, dev)
        if out is None:
            # one allocation, the 64-bit slots first
            buf = _empty(torch, stream, 3 * (T + B) + 1, i32, self.device)
            slots, q_off, kv_len, status, positions = buf.split_with_sizes((2 * T, B + 1, B, B, T))
            out = WindowLayout(q_off, kv_len, slots.view(i64), positions, status)
            at = buf.data_ptr()
            lay = _pack_layout(at + 8 * T, at + 8 * T + 4 * (B + 1), at, at + 8 * T + 4 * (3 * B + 1), at + 8 * T + 4 * (2 * B + 1))
        else:
            lay = _pack_layout(_array("out.q_off", out.q_off, i32, B + 1, dev), _array("out.kv_len", out.kv_len, i32, B, dev),
                               _array("out.slot_map", out.slot_map, i64, T, dev),
                               _array("out.positions", out.positions, i32, T, dev),
                               0 if out.status is None else _array("out.status", out.status, i32, B, dev))
        self._call("wisv_cache_extend", stream, self._pages_at, B, T, ptr, n_new if uniform else 0, lay)
        return out

    def commit(self, new_len, *, B: int, status=None, stream=None):
        """wisv_cache_commit: the kept length of each request (int32 [B]); pages behind it go back.  Returns status.
        A request that extend flagged (status WISV_ST_NO_PAGES, kv_len 0) keeps its old length, seq_len: nothing of its window
        is cached."""
        i32 = self._torch.int32
        if status is None:
            status = _empty(self._torch, stream, B, i32, self.device)
            at = status.data_ptr()
        else:
            at = _array("status", status, i32, B, self._index)
        self._call("wisv_cache_commit", stream, self._pages_at, B, _array("new_len", new_len, i32, B, self._index), at)
        return status

    def append(self, k, v, k_pages, v_pages, slot_map, *, stream=None):
        """wisv_cache_append: one layer's new keys and values [T, n_kv_heads, head_dim] into their slots."""
        kp, kt, kh, T = self._rows("k", k, self.n_kv_heads)
        vp, vt, vh, _ = self._rows("v", v, self.n_kv_heads, T)
        kpool, k0, k1, k2 = self._pages_of("k_pages", k_pages)
        vpool, v0, v1, v2 = self._pages_of("v_pages", v_pages)
        self._call("wisv_cache_append", stream,
                   _pack_append(T, kp, vp, kt, kh, vt, vh, kpool, vpool, k0, k1, k2, v0, v1, v2,
                                _array("slot_map", slot_map, self._torch.int64, T, self._index)))

    def attend(self, q, k_pages, v_pages, kv_len, *, B: int, max_new: int, q_off=None, out=None, lse=None,
               scale: Optional[float] = None, block_table=None, clear_rest: Optional[bool] = None, stream=None):
        """wisv_cache_attend: attention of the new rows q [T, n_heads, head_dim] over the cache, causal among
        themselves.  kv_len: int32 [B], new tokens included; q_off: int32 [B+1], or None for max_new rows each.
        Rows of q before q_off[0] or from q_off[B] on give zeros (-inf in lse) with clear_rest, which is the default where
        the output is made here, and are left alone in an output that is given."""
        torch, dev = self._torch, self._index
        i32 = torch.int32
        H, D = self.n_heads, self.head_dim
        qp, qt, qh, T = self._rows("q", q, H)
        kpool, k0, k1, k2 = self._pages_of("k_pages", k_pages)
        vpool, v0, v1, v2 = self._pages_of("v_pages", v_pages)
        made = out is None
        if made:
            out = _empty(torch, stream, (T, H, D), self.dtype, self.device)
            op, ot, oh = out.data_ptr(), H * D, D
        else:
            op, ot, oh, _ = self._rows("out", out, H, T)
        if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (T, H) or
                                not lse.is_contiguous() or lse.get_device() != dev):
            raise ValueError("lse must be a contiguous float32 [T, n_heads] tensor")
        if scale is not None and not scale > 0:
            raise ValueError("scale must be positive")
        table, blocks, step = self._owned[2], self.max_blocks, self.max_blocks
        if block_table is not None:
            table = block_table
            if table.dtype is not i32 or table.dim() != 2 or table.shape[0] < B or table.stride(1) != 1 or table.get_device() != dev:
                raise ValueError("block_table must be int32 [B, blocks] on %s" % self.device)
            blocks, step = table.shape[1], _row_stride(table)
        self._call("wisv_cache_attend", stream,
                   _pack_attend(B, T, max_new, 0 if q_off is None else _array("q_off", q_off, i32, B + 1, dev),
                                _array("kv_len", kv_len, i32, B, dev), table.data_ptr(), step, blocks, qp, qt, qh,
                                kpool, vpool, k0, k1, k2, v0, v1, v2, op, ot, oh, 0 if lse is None else lse.data_ptr(),
                                0.0 if scale is None else scale, made if clear_rest is None else bool(clear_rest)))
        return out

    def device_error(self) -> int:
        v = C.c_int32(0)
        with self._torch.cuda.device(self.device):
            _check(self.lib.wisv_cache_error(self._h, self._raw_stream(self._index), C.byref(v)), "wisv_cache_error")
        return v.value

    def debug_waits(self, limit_cycles: int = 0, block: int = -1):
        """wisv_debug_cache_waits: a shorter limit for the waits of attend, and a block that never copies values."""
        _check(self.lib.wisv_debug_cache_waits(self._h, limit_cycles, block), "wisv_debug_cache_waits")

    def launch_count(self) -> int:
        return int(self.lib.wisv_cache_launch_count(self._h))


_residual_call = None


def _torch_and_call():
    global _residual_call
    if _residual_call is None:
        import torch
        _residual_call = torch, _lib().wisv_verify_residual
    return _residual_call


@dataclass
class ResidualOutput:
    accept_len: "object"
    token: "object"
    mass: "object" = None
    status: "object" = None


def _probs(torch, t, index):
    """(address, rows, columns, row stride, WISV_DT_*) of a matrix of probabilities on device `index`."""
    dt, stride = t.dtype, t.stride()
    code = DT_F32 if dt is torch.float32 else DT_BF16 if dt is torch.bfloat16 else DT_F16 if dt is torch.float16 else None
    if code is None or len(stride) != 2 or stride[1] != 1 or t.get_device() != index:
        raise ValueError("probabilities must be 2-D float32, bfloat16 or float16 tensors with contiguous rows, on one device")
    rows, columns = t.shape
    return t.data_ptr(), rows, columns, stride[0] if rows > 1 else columns, code


def verify_residual(target_probs, draft_tokens, uniforms, u_draw, *, B: int, K: int = 0, k_off=None,
                    T: Optional[int] = None, draft_probs=None, draft_ids=None, accept_len=None,
                    out: Optional[ResidualOutput] = None, stream=None) -> ResidualOutput:
    """wisv_verify_residual: verify drafts against the target's probabilities [T + B, V] and draw the next token.

    draft_probs: the drafter's distributions, [T, V] dense, or float32 [T, n_top] with draft_ids int32 [T, n_top] (n_top = 0
    names no token: Q is 0 everywhere), or None for a deterministic drafter.  uniforms [T] decide acceptance, u_draw [B]
    the token.  With accept_len (int32 [B], a verdict of Verifier.verify) the windows are taken as decided and only the
    token is drawn.
    Asynchronous on the current (or given) torch stream; nothing is kept between calls.
    """
    torch, call = _torch_and_call()
    dev, i32, f32 = target_probs.get_device(), torch.int32, torch.float32
    if dev < 0:
        raise ValueError("target_probs must be a CUDA tensor")
    if T is None:
        T = B * K if k_off is None else draft_tokens.shape[0]
    tp, rows, V, ts, tdt = _probs(torch, target_probs, dev)
    if rows < T + B:
        raise ValueError("target_probs must have T + B rows")
    qp, qs, qdt, n_top, ids = 0, 0, DT_F32, 0, 0
    if draft_probs is not None:
        qp, n, width, qs, qdt = _probs(torch, draft_probs, dev)
        if n < T:
            raise ValueError("draft_probs must have T rows")
        if draft_ids is not None:
            if qdt != DT_F32 or draft_ids.shape != draft_probs.shape:
                raise ValueError("listed draft_probs are float32 and of draft_ids' shape")
            if width == 0:
                # lists without entries name no token; torch gives them the address 0, which stands for a deterministic drafter
                draft_ids = _full(torch, stream, (T, 1), -1, i32, target_probs.device)
                draft_probs = _full(torch, stream, (T, 1), 0.0, f32, target_probs.device)
                qp, qs, width = draft_probs.data_ptr(), 1, 1
            n_top = width
            ids = _array("draft_ids", draft_ids, i32, T * n_top, dev)
        elif width != V:
            raise ValueError("dense draft_probs must have the target's vocabulary")
    elif draft_ids is not None:
        raise ValueError("draft_ids without draft_probs")
    if out is None:
        buf = _empty(torch, stream, 4 * B, i32, target_probs.device)
        a, t, m, st = buf.split_with_sizes((B, B, B, B))
        out = ResidualOutput(a, t, m.view(f32), st)
        at = buf.data_ptr()
        outs = (at, at + 4 * B, at + 8 * B, at + 12 * B)
    else:
        outs = (_array("out.accept_len", out.accept_len, i32, B, dev), _array("out.token", out.token, i32, B, dev),
                0 if out.mass is None else _array("out.mass", out.mass, f32, B, dev),
                0 if out.status is None else _array("out.status", out.status, i32, B, dev))
    r = _pack_residual(B, 0 if k_off is not None else K, 0 if k_off is None else _array("k_off", k_off, i32, B + 1, dev), T, V,
                       tp, ts, tdt,
                       _array("draft_tokens", draft_tokens, i32, T, dev), qp, qs, qdt, ids, n_top,
                       0 if uniforms is None else _array("uniforms", uniforms, f32, T, dev),
                       _array("u_draw", u_draw, f32, B, dev),
                       0 if accept_len is None else _array("accept_len", accept_len, i32, B, dev), *outs)
    s = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
    if torch._C._cuda_getDevice() != dev:
        with torch.cuda.device(dev):
            rc = call(r, s)
    else:
        rc = call(r, s)
    if rc:
        raise WisvError(rc, "wisv_verify_residual")
    return out
