"""Tensor wrappers of the attention path: the 8-bit key and value cache, and the norms and rotation of query and key heads.

Like Linear and quant_rows they check their arguments and call the library; every operand lives on one GPU, which is the current
one, `stream` (default: the current one) is where a call runs and where what it allocates belongs, and nothing is recorded by autograd.
"""
from __future__ import annotations

import ctypes as C
import math

from . import binding as B


_int32 = _bfloat16 = _uint8 = None  # torch's, from the first object on: an import in a call takes 0.2 us


def _types():
    global _int32, _bfloat16, _uint8
    import torch
    _int32, _bfloat16, _uint8 = torch.int32, torch.bfloat16, torch.uint8


def _ints(t, what, n, device):
    """The address of n contiguous int32 on GPU `device`."""
    if t.dtype is not _int32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} must be {n} contiguous int32")
    if t.get_device() != device:
        raise B._elsewhere(t, what, device)
    return t.data_ptr()


def _check_device(t, what):
    device = t.get_device()
    if device < 0 or device != B._current_device():
        raise B._not_current(t, what)
    return device


def _table(table, requests, device):
    rows, width, ld = B._matrix(table, "table", device)
    if table.dtype is not _int32 or rows != requests:
        raise ValueError(f"table must be int32 with {requests} rows")
    return width, ld


class KVCache:
    """Owns one ``dr_kv_cache`` over codes k and v [blocks, kv heads, block tokens, head dim] (float8_e4m3fn or uint8, contiguous) and
    their scales [blocks, kv heads] (fp32): a value is its code times the scale of its block and head.  Keeps references to the tensors."""

    def __init__(self, k, v, k_scale, v_scale):
        import torch
        _types()
        self.device = _check_device(k, "k")
        for t, what in ((k, "k"), (v, "v")):
            if t.get_device() != self.device:
                raise B._elsewhere(t, what, self.device)
            if t.dim() != 4 or not B._holds_codes(t) or not t.is_contiguous() or tuple(t.shape) != tuple(k.shape):
                raise ValueError(f"{what} must be contiguous e4m3 codes [blocks, kv heads, block tokens, head dim], k and v alike")
        for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t.get_device() != self.device:
                raise B._elsewhere(t, what, self.device)
            if t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != tuple(k.shape[:2]):
                raise ValueError(f"{what} must be contiguous fp32 [blocks, kv heads]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_blocks, self.kv_heads, self.block_tokens, self.head_dim = k.shape
        desc = B.dr_kv_cache_desc(struct_size=C.sizeof(B.dr_kv_cache_desc), n_blocks=self.n_blocks, kv_heads=self.kv_heads,
                                  block_tokens=self.block_tokens, head_dim=self.head_dim, k_dev=k.data_ptr(), v_dev=v.data_ptr(),
                                  k_scale_dev=k_scale.data_ptr(), v_scale_dev=v_scale.data_ptr())
        rc, self.handle = B.dr_kv_cache_create(desc)
        if rc:
            self.handle = None
            raise B.DrError(rc, "dr_kv_cache_create")
        self._word, self._work = self.handle.value or 0, {}

    @classmethod
    def empty(cls, n_blocks, kv_heads, block_tokens, head_dim, device=None):
        """A cache of its own memory (blocks need no initial values)."""
        import torch
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
        k, v = (torch.empty(n_blocks, kv_heads, block_tokens, head_dim, dtype=torch.float8_e4m3fn, device=device) for _ in range(2))
        ks, vs = (torch.empty(n_blocks, kv_heads, dtype=torch.float32, device=device) for _ in range(2))
        return cls(k, v, ks, vs)

    def close(self):
        if getattr(self, "handle", None):
            B.dr_kv_cache_destroy(self.handle)
            self.handle, self._word = None, 0

    def __del__(self):
        if B is not None and B.lib is not None:  # at the interpreter's end the module may be gone before its objects
            self.close()

    def runs_for(self, requests, rows):
        """Entries that `runs` needs for a step of so many rows."""
        return min(rows, rows // self.block_tokens + 2 * requests)

    def extend(self, added, lengths, table, free, state, rows, *, lengths_out=None, state_out=None, offsets=None, positions=None,
               runs=None, stream=None):
        """dr_kv_extend: one step's block table, positions and runs of slots from the requests' lengths, all on the GPU.  added, lengths
        [requests], table [requests, width], free [blocks], state [2] (free blocks, requests refused) are int32; lengths and state are
        updated in place unless lengths_out and state_out are given; rows: the step's rows.  Rows of refused requests have position -1, and
        what attend makes of them has no meaning.  A length lowered by hand loses blocks, unless they are put on the free list.  Returns (offsets [requests + 1],
        positions [rows], runs [runs_for(requests, rows), 4])."""
        device = self.device
        if device != B._current_device():
            raise B._not_current(self.k, "the cache")
        n = lengths.numel()
        p_added, p_lengths = _ints(added, "added", n, device), _ints(lengths, "lengths", n, device)
        p_out = p_lengths if lengths_out is None else _ints(lengths_out, "lengths_out", n, device)
        p_free, p_state = _ints(free, "free", self.n_blocks, device), _ints(state, "state", 2, device)
        p_state_out = p_state if state_out is None else _ints(state_out, "state_out", 2, device)
        width, ld = _table(table, n, device)
        if rows < 0:
            raise ValueError("rows must not be negative")
        if offsets is None:
            offsets = B._empty(1, n + 1, _int32, lengths.device, stream).view(-1)
        if positions is None:
            positions = B._empty(1, rows, _int32, lengths.device, stream).view(-1)
        if runs is None:
            runs = B._empty(self.runs_for(n, rows), 4, _int32, lengths.device, stream)
        p_runs, n_runs = self._runs(runs)
        rc = B._fn("dr_kv_extend")(self._word, p_added, p_lengths, p_out, n, table.data_ptr(), ld, width, p_free, p_state, p_state_out,
                                   rows, _ints(offsets, "offsets", n + 1, device), _ints(positions, "positions", rows, device), p_runs, n_runs,
                                   B._stream_of(device, stream))
        if rc:
            raise B.DrError(rc, "dr_kv_extend")
        return offsets, positions, runs

    def _runs(self, runs):
        n, four = runs.shape
        if runs.dtype is not _int32 or four != 4 or not runs.is_contiguous():
            raise ValueError("runs must be contiguous int32 of four columns")
        if runs.get_device() != self.device:
            raise B._elsewhere(runs, "runs", self.device)
        return runs.data_ptr(), n

    def attend(self, q, lengths, table, offsets=None, *, window=0, sinks=0, scale=None, out=None, stream=None):
        """dr_attend: q [rows, query heads * head dim] (bf16; any number of rows apart, so the query columns of a qkv product will do),
        lengths [requests] with the step's tokens among them, table [requests, width], offsets [requests + 1] (None: one row a
        request) -> out [rows, query heads * head dim] bf16.  A token sees those before it and itself; window > 0: the last `window` of
        them and the first `sinks`.  scale: head_dim ** -0.5 by default.  Rows of an allocated output that no request owns are not
        initialised."""
        device = q.get_device()
        if device != self.device or device != B._current_device():
            raise B._elsewhere(q, "q", self.device) if device != self.device else B._not_current(q, "q")
        if q.requires_grad:
            _refuse("q")
        rows, cols, ldq = B._matrix(q, "q", device)
        if q.dtype is not _bfloat16:
            raise TypeError(f"q must be bfloat16, not {q.dtype}")
        n_q = cols // self.head_dim
        if cols % self.head_dim or n_q < 1 or n_q % self.kv_heads:
            raise ValueError(f"q must hold heads of {self.head_dim}, a multiple of the cache's {self.kv_heads}")
        if window < 0 or sinks < 0:
            raise ValueError("window and sinks must not be negative")
        n = lengths.numel()
        p_lengths = _ints(lengths, "lengths", n, device)
        p_offsets = 0 if offsets is None else _ints(offsets, "offsets", n + 1, device)
        if offsets is None and rows != n:
            raise ValueError("without offsets q has one row for each request")
        width, ld = _table(table, n, device)
        if out is None:
            out, ldo = B._empty(rows, cols, _bfloat16, q.device, stream), cols
        else:
            got_rows, got_cols, ldo = B._matrix(out, "out", device)
            if got_rows != rows or got_cols != cols or out.dtype is not _bfloat16:
                raise ValueError(f"out must be bfloat16, {rows} x {cols}")
        # (the library checks the sizes, and that this is enough: none for tables of 512 tokens at most)
        need, p_work = 0, 0
        if width * self.block_tokens > 512:
            need = self._work.get(n_q)
        if need is None:
            rc, need = B.dr_attend_work(self.handle, n_q, n, rows)
            if rc:
                raise B.DrError(rc, "dr_attend_work")
            self._work[n_q] = need
        if need:
            work = B._empty(1, need, _uint8, q.device, stream)
            p_work = work.data_ptr()
        rc = B._fn("dr_attend")(self._word, q.data_ptr(), ldq, n_q, rows, p_offsets, p_lengths, n, table.data_ptr(), ld, width,
                                1.0 / math.sqrt(self.head_dim) if scale is None else scale, window, sinks, out.data_ptr(), ldo,
                                p_work, need, B._stream_of(device, stream))
        if rc:
            raise B.DrError(rc, "dr_attend")
        return out


def _refuse(what):
    import torch
    if torch.is_grad_enabled():
        raise RuntimeError(f"{what} requires a gradient, which this call does not record: make it under torch.no_grad() or on detached "
                           "tensors, and take the gradients of norms and rotation with QKHeads.grad")


class QKHeads:
    """Owns one ``dr_qk``: the norms of n_q_heads query and n_kv_heads key heads of head_dim (q_norm, k_norm [head_dim], bf16 or fp32; both
    None: no norm) and the rotation by position, base^(-2 i / head_dim) for pair (i, i + head_dim / 2).  Keeps references to the norms."""

    def __init__(self, n_q_heads, n_kv_heads, head_dim, q_norm=None, k_norm=None, *, base=1e6, eps=1e-6):
        _types()
        self.n_q_heads, self.n_kv_heads, self.head_dim, self.q_norm, self.k_norm = n_q_heads, n_kv_heads, head_dim, q_norm, k_norm
        self.device = None
        if q_norm is not None or k_norm is not None:
            if q_norm is None or k_norm is None:
                raise ValueError("q_norm and k_norm come together")
            self.device = _check_device(q_norm, "q_norm")
            for t, what in ((q_norm, "q_norm"), (k_norm, "k_norm")):
                if t.get_device() != self.device:
                    raise B._elsewhere(t, what, self.device)
                if t.dim() != 1 or t.shape[0] != head_dim or not t.is_contiguous() or t.dtype != q_norm.dtype:
                    raise ValueError(f"{what} must be a contiguous vector of {head_dim}, both of one type")
        desc = B.dr_qk_desc(struct_size=C.sizeof(B.dr_qk_desc), n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim,
                            norm_dtype=0 if q_norm is None else B._code_of(q_norm, "q_norm"), eps=eps, base=base,
                            q_norm_dev=None if q_norm is None else q_norm.data_ptr(),
                            k_norm_dev=None if k_norm is None else k_norm.data_ptr())
        if self.device is None:
            self.device = B._current_device()
        rc, self.handle = B.dr_qk_create(desc)
        if rc:
            self.handle = None
            raise B.DrError(rc, "dr_qk_create")
        self._word, self._work = self.handle.value or 0, None
        self._norms = () if q_norm is None else (q_norm, k_norm)

    def close(self):
        if getattr(self, "handle", None):
            B.dr_qk_destroy(self.handle)
            self.handle, self._word = None, 0

    def __del__(self):
        if B is not None and B.lib is not None:
            self.close()

    def _rows(self, x, heads, what, record=True):
        device = x.get_device()
        if device != self.device or device != B._current_device():
            raise B._elsewhere(x, what, self.device) if device != self.device else B._not_current(x, what)
        norms = self._norms
        if record and (x.requires_grad or (norms and (norms[0].requires_grad or norms[1].requires_grad))):
            _refuse(f"{what} or a norm")
        rows, cols, ld = B._matrix(x, what, device)
        if cols < heads * self.head_dim:
            raise ValueError(f"{what} must have {heads} heads of {self.head_dim}")
        return rows, ld if rows > 1 else cols, B._code_of(x, what)

    def _out(self, out, rows, heads, like, what, stream):
        cols = heads * self.head_dim
        if out is None:
            return B._empty(rows, cols, like.dtype, like.device, stream), cols
        got_rows, got_cols, ld = B._matrix(out, what, self.device)
        if got_rows != rows or got_cols != cols or out.dtype != like.dtype:
            raise ValueError(f"{what} must be {rows} x {cols} of {like.dtype}")
        return out, ld

    def forward(self, x, positions, out=None, stream=None):
        """dr_qk_forward: x [rows, at least (query + key heads) * head_dim], bf16 or fp32 (a qkv product's output), positions [rows] int32 ->
        the query and key heads, normed and rotated, in x's type.  `out` may be x's own columns.  Rows of negative position are left as
        they are (of an allocated output: not initialised)."""
        rows, ldx, code = self._rows(x, self.n_q_heads + self.n_kv_heads, "x")
        y, ldy = self._out(out, rows, self.n_q_heads + self.n_kv_heads, x, "out", stream)
        rc = B._fn("dr_qk_forward")(self._word, x.data_ptr(), code, ldx, _ints(positions, "positions", rows, self.device), rows,
                                    y.data_ptr(), ldy, B._stream_of(self.device, stream))
        if rc:
            raise B.DrError(rc, "dr_qk_forward")
        return y

    __call__ = forward

    def append(self, x, positions, runs, cache, out=None, stream=None):
        """dr_qk_append: x [rows, (query + 2 key-value heads) * head_dim] -> the query heads, normed and rotated ([rows, query heads *
        head_dim], `out` may be x's own columns); keys, normed and rotated, and values go into `cache` at `runs` (KVCache.extend).  Rows of
        negative position are left as they are (of an allocated output: not initialised)."""
        rows, ldx, code = self._rows(x, self.n_q_heads + 2 * self.n_kv_heads, "x")
        y, ldy = self._out(out, rows, self.n_q_heads, x, "out", stream)
        if cache.device != self.device:
            raise B._elsewhere(cache.k, "cache", self.device)
        p_runs, n_runs = cache._runs(runs)
        rc = B._fn("dr_qk_append")(self._word, x.data_ptr(), code, ldx, _ints(positions, "positions", rows, self.device), rows, p_runs,
                                   n_runs, cache._word, y.data_ptr(), ldy, B._stream_of(self.device, stream))
        if rc:
            raise B.DrError(rc, "dr_qk_append")
        return y

    def grad(self, x, positions, dy, dx=None, dq_norm=None, dk_norm=None, accumulate=False, stream=None):
        """dr_qk_grad: gradients of forward at x for dy [rows, (query + key heads) * head_dim] of x's type: (dx, dq_norm, dk_norm), the norms'
        in fp32 (None without norms; accumulate adds them to the ones given).  `dx` may be dy.  Rows of negative position add nothing to the
        norms' gradients and are left as they are in dx (allocated: not initialised)."""
        import torch
        heads = self.n_q_heads + self.n_kv_heads
        rows, ldx, code = self._rows(x, heads, "x", record=False)
        dy_rows, lddy, dy_code = self._rows(dy, heads, "dy", record=False)
        if dy_rows != rows or dy_code != code or dy.shape[1] != heads * self.head_dim:
            raise ValueError(f"dy must be {rows} x {heads * self.head_dim} of x's type")
        dx, lddx = self._out(dx, rows, heads, x, "dx", stream)
        need, p_work, p_dq, p_dk = 0, 0, 0, 0
        if self.q_norm is not None:
            if accumulate and (dq_norm is None or dk_norm is None):
                raise ValueError("accumulate adds to dq_norm and dk_norm: give both")
            grads = []
            for t, what in ((dq_norm, "dq_norm"), (dk_norm, "dk_norm")):
                if t is None:
                    t = B._empty(1, self.head_dim, torch.float32, x.device, stream).view(-1)
                if t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != self.head_dim or not t.is_contiguous():
                    raise ValueError(f"{what} must be {self.head_dim} contiguous fp32")
                if t.get_device() != self.device:
                    raise B._elsewhere(t, what, self.device)
                grads.append(t)
            dq_norm, dk_norm = grads
            p_dq, p_dk = dq_norm.data_ptr(), dk_norm.data_ptr()
            if self._work is None:
                rc, self._work = B.dr_qk_grad_work(self.handle)
                if rc:
                    raise B.DrError(rc, "dr_qk_grad_work")
            need = self._work
            work = B._empty(1, need, torch.uint8, x.device, stream)
            p_work = work.data_ptr()
        elif dq_norm is not None or dk_norm is not None:
            raise ValueError("without norms there are no gradients of them")
        rc = B._fn("dr_qk_grad")(self._word, x.data_ptr(), code, ldx, _ints(positions, "positions", rows, self.device), dy.data_ptr(), lddy,
                                 rows, dx.data_ptr(), lddx, p_dq, p_dk, int(accumulate), p_work, need, B._stream_of(self.device, stream))
        if rc:
            raise B.DrError(rc, "dr_qk_grad")
        return dx, dq_norm, dk_norm
