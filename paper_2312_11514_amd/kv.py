"""Paged key-value cache and its attention: ctypes binding of the lif_kv calls of include/lif.h, argument marshalling only.

    kv = KVCache(layers=32, heads=32, kv_heads=8, head_dim=128, page_tokens=16, pages=4096, max_seqs=64, max_pages=512)
    kv.reserve(counts)                            # pages for this step's tokens, once for all layers
    for l in range(32):
        kv.append(l, q, k, v, q_out)              # norms, rotation, keys and values into their pages
        kv.attend(l, q_out, out)
"""
from __future__ import annotations

import ctypes as C
import struct

from . import binding as _b
from .binding import LIF_INVALID_ARG, LifError

# lif_kv_rows and lif_kv_query, filled in one go: setting the fields of a ctypes structure one by one is a third of the cost of a call
_ROWS, _QUERY = struct.Struct("@4P4q6P2i"), struct.Struct("@3P2q3P3i4x")
assert _ROWS.size == C.sizeof(_b.LifKvRows) and _QUERY.size == C.sizeof(_b.LifKvQuery)

_DTYPES = {"f32": _b.LIF_F32, "f16": _b.LIF_F16, "bf16": _b.LIF_BF16}


def rope_frequencies(rotary_dim, base=10000.0, scaling=_b.ROPE_PLAIN, factor=1.0, trained=0.0, slow=1.0, fast=32.0):
    """lif_rope_frequencies: angle per position of every rotated pair, a float64 tensor on the CPU."""
    import torch
    out = torch.zeros(max(1, int(rotary_dim) // 2), dtype=torch.float64)
    _b._check(_b.load_library().lif_rope_frequencies(int(rotary_dim), float(base), int(scaling), float(factor), float(trained), float(slow),
                                                     float(fast), C.cast(out.data_ptr(), C.POINTER(C.c_double))))
    return out


def _refuse(message):
    raise LifError(LIF_INVALID_ARG, message)


class KVCache:
    """The cache of a stack of attention layers behind the C ABI.  Owns (through torch) every array the library uses; `table`, `lengths`,
    `fresh` and `refs` may be read at any time, and written before adopt().  All calls but state() enqueue on torch's current stream and
    return immediately.

    frequencies: float64 tensor [rotary_dim / 2] (rope_frequencies), needed if rotary_dim > 0.  scale: of the scores, 1 / sqrt(head_dim) if None.
    """

    def __init__(self, *, layers, heads, kv_heads, head_dim, page_tokens, pages, max_seqs, max_pages, max_tokens=1, dtype="f16",
                 norm=_b.NORM_NONE, norm_eps=1e-5, rotary=_b.ROTARY_HALF, rotary_dim=0, rotary_scale=1.0, frequencies=None, scale=None,
                 device="cuda"):
        import torch
        self.lib = _b.load_library()
        self.torch = torch
        if dtype not in _DTYPES:
            _refuse("dtype must be f32, f16 or bf16")
        self.cfg = _b.LifKvConfig(layers, heads, kv_heads, head_dim, page_tokens, pages, max_seqs, max_pages, max_tokens, _DTYPES[dtype],
                                  norm, rotary, rotary_dim, norm_eps, rotary_scale, max(head_dim, 1) ** -0.5 if scale is None else scale)
        ws_bytes = self.lib.lif_kv_workspace_bytes(C.byref(self.cfg))
        if ws_bytes == 0:
            _refuse("configuration rejected by lif_kv_workspace_bytes")
        self.tdtype = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        if rotary_dim and (frequencies is None or frequencies.dtype != torch.float64 or frequencies.numel() != rotary_dim // 2):
            _refuse("frequencies must be a float64 tensor of rotary_dim / 2 elements")
        n = 4 if dtype == "f32" else 8
        new = lambda shape, dt: torch.empty(shape, dtype=dt, device=device)
        self.k = new((layers, pages, kv_heads, page_tokens, head_dim), self.tdtype)
        self.v = new((layers, pages, kv_heads, page_tokens // n, head_dim, n), self.tdtype)
        self.table = new((max_seqs, max_pages), torch.int32)
        self.lengths, self.fresh = new((max_seqs,), torch.int32), new((max_seqs,), torch.int32)
        self.refs = new((pages,), torch.int32)
        self.frequencies = frequencies.to(device).contiguous() if rotary_dim else None
        self.workspace = new((ws_bytes,), torch.uint8)
        self.buf = _b.LifKvBuffers(*[_b._ptr(t) for t in (self.k, self.v, self.table, self.lengths, self.fresh, self.refs, self.frequencies,
                                                          self.workspace)], ws_bytes)
        h = C.c_void_p()
        _b._check(self.lib.lif_kv_create(C.byref(self.cfg), C.byref(self.buf), C.byref(h)))
        self.handle = h
        self._bind()
        self.reset()

    def _bind(self):
        """What the calls of a decode step need again and again, as plain Python values; the argument structures are filled anew per call."""
        c, torch = self.cfg, self.torch
        self._heads, self._kv_heads, self._dim, self._seqs, self._gpu = c.heads, c.kv_heads, c.head_dim, c.max_seqs, self.table.get_device()
        self._int32, self._float32, self._int64 = torch.int32, torch.float32, torch.int64
        self._append_call, self._attend_call = self.lib.lif_kv_append, self.lib.lif_kv_attend
        self._rows_arg, self._query_arg = _b.LifKvRows(), _b.LifKvQuery()
        self._rows_ref, self._query_ref = C.byref(self._rows_arg), C.byref(self._query_arg)

    def close(self):
        if getattr(self, "handle", None):
            self.lib.lif_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- argument checks (on the path of every layer of a step) --------------------------------------------------------------
    def _ints(self, t, count, what):
        if t.dtype is not self._int32 or t.numel() != count or t.get_device() != self._gpu or not t.is_contiguous():
            _refuse(f"{what} must be a contiguous int32 tensor of {count} elements beside the cache")
        return t.data_ptr()

    def _slots(self, slots, batch):
        if slots is not None:
            return self._ints(slots, batch, "slots")
        if batch > self._seqs:
            _refuse("more rows than slots")
        return 0

    def _rows(self, t, shape, what):
        """The stride between tokens of [batch, tokens, heads, head_dim], heads contiguous."""
        if t.dtype is self.tdtype and t.get_device() == self._gpu and t.shape == shape:
            batch, tokens, heads, d = shape
            if t.is_contiguous():
                return heads * d
            sb, sn, sh, sd = t.stride()
            if batch == 1:
                sb = tokens * sn
            if tokens == 1:
                sn = sb if batch > 1 else heads * d
                sb = sn
            if sd == 1 and (sh == d or heads == 1) and sb == tokens * sn:
                return sn
        _refuse(f"{what} must be {list(shape)} of the cache's type beside the cache, heads contiguous, tokens at one stride")

    def _norm(self, t, what):
        if t is None:
            return 0
        if t.dtype is not self._float32 or t.numel() != self._dim or t.get_device() != self._gpu or not t.is_contiguous():
            _refuse(f"{what} must be a contiguous float32 tensor of head_dim elements beside the cache")
        return t.data_ptr()

    # ---- the C-ABI calls, same names -------------------------------------------------------------------------------------
    def reset(self):
        _b._check(self.lib.lif_kv_reset(self.handle, _b._stream()))

    def adopt(self):
        _b._check(self.lib.lif_kv_adopt(self.handle, _b._stream()))

    def reserve(self, counts):
        _b._check(self.lib.lif_kv_reserve(self.handle, self._ints(counts, self.cfg.max_seqs, "counts"), _b._stream()))

    def truncate(self, lengths):
        _b._check(self.lib.lif_kv_truncate(self.handle, self._ints(lengths, self.cfg.max_seqs, "lengths"), _b._stream()))

    def fork(self, src, dst):
        n = src.numel()
        _b._check(self.lib.lif_kv_fork(self.handle, self._ints(src, n, "src"), self._ints(dst, n, "dst"), n, _b._stream()))

    def compact(self):
        _b._check(self.lib.lif_kv_compact(self.handle, _b._stream()))

    def append(self, layer, q, k, v, q_out, norm=None, positions=None, slots=None):
        """q, q_out [batch, tokens, heads, head_dim], k, v [batch, tokens, kv_heads, head_dim].  norm: (q weight, q bias, k weight, k bias),
        each float32 [head_dim] or None."""
        if q.dim() != 4:
            _refuse("q must be [batch, tokens, heads, head_dim]")
        batch, tokens, _, _ = q.shape
        of_q, of_k = (batch, tokens, self._heads, self._dim), (batch, tokens, self._kv_heads, self._dim)
        q_stride, k_stride, v_stride = self._rows(q, of_q, "q"), self._rows(k, of_k, "k"), self._rows(v, of_k, "v")
        out_stride = self._rows(q_out, of_q, "q_out")
        qw = qb = kw = kb = 0
        if norm is not None:
            qw, qb, kw, kb = norm
            qw, qb = self._norm(qw, "q weight"), self._norm(qb, "q bias")
            kw, kb = self._norm(kw, "k weight"), self._norm(kb, "k bias")
        _ROWS.pack_into(self._rows_arg, 0, q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr(), q_stride, k_stride, v_stride, out_stride,
                        qw, qb, kw, kb, self._ints(positions, batch * tokens, "positions") if positions is not None else 0,
                        self._slots(slots, batch), batch, tokens)
        rc = self._append_call(self.handle, layer, self._rows_ref, _b._stream())
        if rc:
            _b._check(rc)

    def attend(self, layer, q, out, lse=None, window=0, starts=None, tree=None, slots=None):
        """q, out [batch, tokens, heads, head_dim], out may be q; lse float32 [batch, tokens, heads]; starts int32 [batch]; tree int64 [batch, tokens], a
        bit per new token that is seen; slots int32 [batch]."""
        if q.dim() != 4:
            _refuse("q must be [batch, tokens, heads, head_dim]")
        shape = batch, tokens, _, _ = q.shape
        if shape[2] != self._heads or shape[3] != self._dim:
            _refuse(f"q must be [batch, tokens, {self._heads}, {self._dim}]")
        q_stride, out_stride = self._rows(q, shape, "q"), self._rows(out, shape, "out")
        if lse is not None and (lse.dtype is not self._float32 or lse.numel() != batch * tokens * self._heads or
                                lse.get_device() != self._gpu or not lse.is_contiguous()):
            _refuse("lse must be a contiguous float32 tensor [batch, tokens, heads] beside the cache")
        if tree is not None and (tree.dtype is not self._int64 or tree.numel() != batch * tokens or tree.get_device() != self._gpu or
                                 not tree.is_contiguous()):
            _refuse("tree must be a contiguous int64 tensor [batch, tokens] beside the cache")
        _QUERY.pack_into(self._query_arg, 0, q.data_ptr(), out.data_ptr(), lse.data_ptr() if lse is not None else 0, q_stride, out_stride,
                         self._slots(slots, batch), self._ints(starts, batch, "starts") if starts is not None else 0,
                         tree.data_ptr() if tree is not None else 0, batch, tokens, window)
        rc = self._attend_call(self.handle, layer, self._query_ref, _b._stream())
        if rc:
            _b._check(rc)

    def set_expected_tokens(self, tokens: int):
        """Cached tokens of a sequence as a rule (0: as many as a table row holds): for attend(), where tables are much wider than sequences."""
        _b._check(self.lib.lif_kv_set_expected_tokens(self.handle, int(tokens)))

    # ---- introspection ---------------------------------------------------------------------------------------------------
    def state(self) -> dict:
        s = _b.LifKvState()
        _b._check(self.lib.lif_kv_get_state(self.handle, C.byref(s), _b._stream()))
        return {n: getattr(s, n) for n, _ in _b.LifKvState._fields_}
