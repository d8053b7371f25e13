"""Paged key/value cache and residual verification on torch CUDA tensors (argument marshalling only)."""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import Optional

from .binding import DT_BF16, DT_F16, DT_F32, WisvError, _check, _ptr, load_library


class _CacheConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_heads", "n_kv_heads", "head_dim", "page_size", "n_pages", "max_requests",
                                         "max_blocks", "dtype")]


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
                ("scale", C.c_float)]


class _Residual(C.Structure):
    _fields_ = [("B", C.c_int32), ("K", C.c_int32), ("k_off", C.c_void_p), ("T_total", C.c_int32), ("V", C.c_int32),
                ("target_probs", C.c_void_p), ("target_stride", C.c_int64), ("target_dtype", C.c_int32),
                ("draft_tokens", C.c_void_p), ("draft_probs", C.c_void_p), ("draft_stride", C.c_int64),
                ("draft_dtype", C.c_int32), ("draft_ids", C.c_void_p), ("n_top", C.c_int32), ("uniforms", C.c_void_p),
                ("u_draw", C.c_void_p), ("accept_in", C.c_void_p), ("accept_len", C.c_void_p), ("token", C.c_void_p),
                ("mass", C.c_void_p), ("status", C.c_void_p)]


_declared = False


def _lib():
    global _declared
    lib = load_library()
    if not _declared:
        P = C.c_void_p
        for name, args in (("wisv_cache_create", [C.POINTER(_CacheConfig), C.POINTER(P)]),
                           ("wisv_cache_destroy", [P]),
                           ("wisv_cache_error", [P, P, C.POINTER(C.c_int32)]),
                           ("wisv_cache_extend", [P, P, C.c_int32, C.c_int32, P, C.c_int32, C.POINTER(_Layout), P]),
                           ("wisv_cache_commit", [P, P, C.c_int32, P, P, P]),
                           ("wisv_cache_append", [P, C.POINTER(_Append), P]),
                           ("wisv_cache_attend", [P, C.POINTER(_Attend), P]),
                           ("wisv_verify_residual", [C.POINTER(_Residual), P])):
            f = getattr(lib, name)
            f.restype, f.argtypes = C.c_int, args
        lib.wisv_cache_launch_count.restype = C.c_int64
        lib.wisv_cache_launch_count.argtypes = [P]
        _declared = True
    return lib


def _ints(torch, device, what, t, dtype, *shape):
    """A contiguous tensor of the documented type and at least the documented size, or ValueError."""
    if t.dtype is not dtype or t.device != device or not t.is_contiguous() or t.numel() < shape[0]:
        raise ValueError("%s must be a contiguous %s tensor with %d entries on %s" % (what, dtype, shape[0], device))
    return t.data_ptr()


def _row_stride(t) -> int:
    """Elements from one row of a 2-D tensor to the next (a single row has none of its own)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _empty(torch, stream, *args, **kw):
    """torch.empty for a result that `stream` (None: the current one) writes."""
    if stream is None:
        return torch.empty(*args, **kw)
    with torch.cuda.stream(stream):
        return torch.empty(*args, **kw)


@dataclass
class WindowLayout:
    """What PagedCache.extend lays out for a round (see wisv_layout)."""
    q_off: "object"
    kv_len: "object"
    slot_map: "object"
    positions: "object"
    status: "object"


class PagedCache:
    """wisv_cache_* on torch CUDA tensors: the paged key/value cache of a target model.

    The bookkeeping tensors (``free_list``, ``n_free``, ``block_table``, ``n_blocks``, ``seq_len``) are ordinary int32
    tensors of this object, with every page free at the start; the page pools of each layer are the caller's:
    ``k_pages`` / ``v_pages`` of shape [n_pages, page_size, n_kv_heads, head_dim] with any strides that keep a
    head's elements contiguous (a [n_pages, n_kv_heads, page_size, head_dim] pool is passed as ``.transpose(1, 2)``).
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
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(self.lib.wisv_cache_create(C.byref(cfg), C.byref(h)), "wisv_cache_create")
        self._h = h
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim
        self.page_size, self.n_pages, self.max_requests, self.max_blocks = page_size, n_pages, max_requests, max_blocks
        self.dtype = torch.bfloat16 if dtype == DT_BF16 else torch.float16
        i32 = dict(dtype=torch.int32, device=self.device)
        self.free_list = torch.arange(n_pages - 1, -1, -1, **i32)
        self.n_free = torch.full((1,), n_pages, **i32)
        self.block_table = torch.full((max_requests, max_blocks), -1, **i32)
        self.n_blocks = torch.zeros(max_requests, **i32)
        self.seq_len = torch.zeros(max_requests, **i32)
        self._pages = _Pages(*(t.data_ptr() for t in (self.free_list, self.n_free, self.block_table, self.n_blocks,
                                                      self.seq_len)))
        # the arrays whose addresses the block above holds
        self._owned = (self.free_list, self.n_free, self.block_table, self.n_blocks, self.seq_len)
        self._pages_ref = C.byref(self._pages)

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
    def _stream(self, stream):
        return (stream if stream is not None else self._torch.cuda.current_stream(self.device)).cuda_stream

    def _call(self, name, *args):
        """One library call with this cache's device current."""
        f = getattr(self.lib, name)
        torch = self._torch
        if torch.cuda.current_device() != self.device.index:
            with torch.cuda.device(self.device):
                rc = f(self._h, *args)
        else:
            rc = f(self._h, *args)
        if rc:
            raise WisvError(rc, name)

    def _check_rows(self, what, t, heads, rows=None):
        s = t.shape
        if t.dtype is not self.dtype or len(s) != 3 or s[1] != heads or s[2] != self.head_dim or t.stride(2) != 1 or \
                t.device != self.device or (rows is not None and s[0] != rows):
            raise ValueError("%s must be [%s, %d, %d] %s on %s with a head's elements contiguous" %
                             (what, "T" if rows is None else rows, heads, self.head_dim, self.dtype, self.device))
        return t.data_ptr(), t.stride(0), t.stride(1)

    def _check_pool(self, what, t):
        if t.dtype is not self.dtype or t.stride(3) != 1 or t.device != self.device or \
                t.shape != (self.n_pages, self.page_size, self.n_kv_heads, self.head_dim):
            raise ValueError("%s must be [%d, %d, %d, %d] %s on %s with a head's elements contiguous" %
                             (what, self.n_pages, self.page_size, self.n_kv_heads, self.head_dim, self.dtype, self.device))
        st = t.stride()
        return t.data_ptr(), st[0], st[1], st[2]

    # ------------------------------------------------------------------ calls
    def extend(self, *, B: int, n_new, T: Optional[int] = None, out: Optional[WindowLayout] = None,
               stream=None) -> WindowLayout:
        """wisv_cache_extend: pages, slots and positions for n_new tokens per request (an int, or int32 [B] on the
        device with their sum T given)."""
        torch = self._torch
        uniform = isinstance(n_new, int)
        if T is None:
            if not uniform:
                raise ValueError("T, the sum of n_new, must be given where n_new lives on the device")
            T = B * n_new
        ptr = None if uniform else _ints(torch, self.device, "n_new", n_new, torch.int32, B)
        if out is None:
            # one allocation for the int32 arrays
            buf = _empty(torch, stream, 3 * B + 1 + T, dtype=torch.int32, device=self.device)
            out = WindowLayout(buf[:B + 1], buf[B + 1:2 * B + 1],
                               _empty(torch, stream, T, dtype=torch.int64, device=self.device), buf[3 * B + 1:], buf[2 * B + 1:3 * B + 1])
        else:
            i32 = torch.int32
            _ints(torch, self.device, "out.q_off", out.q_off, i32, B + 1)
            _ints(torch, self.device, "out.kv_len", out.kv_len, i32, B)
            _ints(torch, self.device, "out.positions", out.positions, i32, T)
            _ints(torch, self.device, "out.slot_map", out.slot_map, torch.int64, T)
            if out.status is not None:
                _ints(torch, self.device, "out.status", out.status, i32, B)
        lay = _Layout(out.q_off.data_ptr(), out.kv_len.data_ptr(), out.slot_map.data_ptr(), out.positions.data_ptr(),
                      _ptr(out.status))
        self._call("wisv_cache_extend", self._pages_ref, B, T, ptr, n_new if uniform else 0, C.byref(lay),
                   self._stream(stream))
        return out

    def commit(self, new_len, *, B: int, status=None, stream=None):
        """wisv_cache_commit: the kept length of each request (int32 [B]); pages behind it go back.  Returns status."""
        torch = self._torch
        ptr = _ints(torch, self.device, "new_len", new_len, torch.int32, B)
        if status is None:
            status = _empty(torch, stream, B, dtype=torch.int32, device=self.device)
        else:
            _ints(torch, self.device, "status", status, torch.int32, B)
        self._call("wisv_cache_commit", self._pages_ref, B, ptr, status.data_ptr(), self._stream(stream))
        return status

    def append(self, k, v, k_pages, v_pages, slot_map, *, stream=None):
        """wisv_cache_append: one layer's new keys and values [T, n_kv_heads, head_dim] into their slots."""
        T = k.shape[0]
        kp, kt, kh = self._check_rows("k", k, self.n_kv_heads)
        vp, vt, vh = self._check_rows("v", v, self.n_kv_heads, T)
        kpool, k0, k1, k2 = self._check_pool("k_pages", k_pages)
        vpool, v0, v1, v2 = self._check_pool("v_pages", v_pages)
        a = _Append(T, kp, vp, kt, kh, vt, vh, kpool, vpool, k0, k1, k2, v0, v1, v2,
                    _ints(self._torch, self.device, "slot_map", slot_map, self._torch.int64, T))
        self._call("wisv_cache_append", C.byref(a), self._stream(stream))

    def attend(self, q, k_pages, v_pages, kv_len, *, B: int, max_new: int, q_off=None, out=None, lse=None,
               scale: Optional[float] = None, block_table=None, stream=None):
        """wisv_cache_attend: attention of the new rows q [T, n_heads, head_dim] over the cache, causal among
        themselves.  kv_len: int32 [B], new tokens included; q_off: int32 [B+1], or None for max_new rows each."""
        torch = self._torch
        i32 = torch.int32
        qp, qt, qh = self._check_rows("q", q, self.n_heads)
        T = q.shape[0]
        kpool, k0, k1, k2 = self._check_pool("k_pages", k_pages)
        vpool, v0, v1, v2 = self._check_pool("v_pages", v_pages)
        if out is None:
            out = _empty(torch, stream, (T, self.n_heads, self.head_dim), dtype=self.dtype, device=self.device)
        op, ot, oh = self._check_rows("out", out, self.n_heads, T)
        if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (T, self.n_heads) or
                                not lse.is_contiguous() or lse.device != self.device):
            raise ValueError("lse must be a contiguous float32 [T, n_heads] tensor")
        if scale is not None and not scale > 0:
            raise ValueError("scale must be positive")
        table = self.block_table if block_table is None else block_table
        if table is not self.block_table and (table.dtype is not i32 or table.dim() != 2 or table.shape[0] < B or
                                              table.stride(1) != 1 or table.device != self.device):
            raise ValueError("block_table must be int32 [B, blocks] on %s" % self.device)
        a = _Attend(B, T, max_new,
                    None if q_off is None else _ints(torch, self.device, "q_off", q_off, i32, B + 1),
                    _ints(torch, self.device, "kv_len", kv_len, i32, B), table.data_ptr(),
                    _row_stride(table), table.shape[1], qp, qt, qh, kpool, vpool, k0, k1, k2, v0, v1, v2,
                    op, ot, oh, _ptr(lse), 0.0 if scale is None else scale)
        self._call("wisv_cache_attend", C.byref(a), self._stream(stream))
        return out

    def device_error(self) -> int:
        v = C.c_int32(0)
        self._call("wisv_cache_error", self._stream(None), C.byref(v))
        return v.value

    def launch_count(self) -> int:
        return int(self.lib.wisv_cache_launch_count(self._h))


@dataclass
class ResidualOutput:
    accept_len: "object"
    token: "object"
    mass: "object" = None
    status: "object" = None


def _probs_dtype(torch, t) -> int:
    code = {torch.float32: DT_F32, torch.bfloat16: DT_BF16, torch.float16: DT_F16}.get(t.dtype)
    if code is None or t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("probabilities must be 2-D float32, bfloat16 or float16 tensors with contiguous rows")
    return code


def verify_residual(target_probs, draft_tokens, uniforms, u_draw, *, B: int, K: int = 0, k_off=None,
                    T: Optional[int] = None, draft_probs=None, draft_ids=None, accept_len=None,
                    out: Optional[ResidualOutput] = None, stream=None) -> ResidualOutput:
    """wisv_verify_residual: verify drafts against the target's probabilities [T + B, V] and draw the next token.

    draft_probs: the drafter's distributions, [T, V] dense, or float32 [T, n_top] with draft_ids int32 [T, n_top], or
    None for a deterministic drafter.  uniforms [T] decide acceptance, u_draw [B] the token.  With accept_len (int32
    [B], a verdict of Verifier.verify) the windows are taken as decided and only the token is drawn.
    Asynchronous on the current (or given) torch stream; nothing is kept between calls.
    """
    import torch
    lib = _lib()
    device = target_probs.device
    if T is None:
        T = B * K if k_off is None else draft_tokens.shape[0]
    tdt = _probs_dtype(torch, target_probs)
    if target_probs.shape[0] < T + B:
        raise ValueError("target_probs must have T + B rows")
    V = target_probs.shape[1]
    qp, qs, qdt, n_top, ids = None, 0, DT_F32, 0, None
    if draft_probs is not None:
        qdt = _probs_dtype(torch, draft_probs)
        if draft_probs.shape[0] < T or draft_probs.device != device:
            raise ValueError("draft_probs must have T rows on the target's device")
        qp, qs = draft_probs.data_ptr(), _row_stride(draft_probs)
        if draft_ids is not None:
            if qdt != DT_F32 or draft_ids.shape != draft_probs.shape:
                raise ValueError("listed draft_probs are float32 and of draft_ids' shape")
            n_top = draft_ids.shape[1]
            ids = _ints(torch, device, "draft_ids", draft_ids, torch.int32, T * n_top)
        elif draft_probs.shape[1] != V:
            raise ValueError("dense draft_probs must have the target's vocabulary")
    elif draft_ids is not None:
        raise ValueError("draft_ids without draft_probs")
    if out is None:
        buf = _empty(torch, stream, 3 * B, dtype=torch.int32, device=device)
        out = ResidualOutput(buf[:B], buf[B:2 * B], _empty(torch, stream, B, dtype=torch.float32, device=device), buf[2 * B:])
    else:
        for name, t, dt in (("accept_len", out.accept_len, torch.int32), ("token", out.token, torch.int32),
                            ("mass", out.mass, torch.float32), ("status", out.status, torch.int32)):
            if t is not None:
                _ints(torch, device, "out." + name, t, dt, B)
    r = _Residual(B, 0 if k_off is not None else K,
                  None if k_off is None else _ints(torch, device, "k_off", k_off, torch.int32, B + 1), T, V,
                  target_probs.data_ptr(), _row_stride(target_probs), tdt,
                  _ints(torch, device, "draft_tokens", draft_tokens, torch.int32, T), qp, qs, qdt,
                  ids, n_top, None if uniforms is None else _ints(torch, device, "uniforms", uniforms, torch.float32, T),
                  _ints(torch, device, "u_draw", u_draw, torch.float32, B),
                  None if accept_len is None else _ints(torch, device, "accept_len", accept_len, torch.int32, B),
                  out.accept_len.data_ptr(), out.token.data_ptr(), _ptr(out.mass), _ptr(out.status))
    st = (stream if stream is not None else torch.cuda.current_stream(device)).cuda_stream
    if torch.cuda.current_device() != device.index:
        with torch.cuda.device(device):
            _check(lib.wisv_verify_residual(C.byref(r), st), "wisv_verify_residual")
    else:
        _check(lib.wisv_verify_residual(C.byref(r), st), "wisv_verify_residual")
    return out
