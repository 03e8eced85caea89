"""The clear side of split inference on torch tensors (argument marshalling only; include/she_clear.h has the definitions).

`Calls` is the part of a Context that runs between a decryption and the next encryption: adapters beside a shared projection,
norms and rotation of queries and keys, attention over a paged cache.  Tensors are on the context's GPU, in bfloat16 or float16 where
nothing else is said, with a contiguous last axis; their other strides are free.  Work is enqueued on the context's stream: when
torch's current stream is another one, that work waits for it and it waits for the work.
"""
from __future__ import annotations

import ctypes as C

import torch

EINVAL = -1


class SheError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"she error {code}: {text}")
        self.code = code


_i32, _u32, _i64, _f32, _p = C.c_int32, C.c_uint32, C.c_int64, C.c_float, C.c_void_p


def _struct(name, fields):
    """A C struct of include/she_clear.h: `fields` is lines of a ctypes type and the names that have it, in the header's order."""
    return type(name, (C.Structure,), {"_fields_": [(n, ty) for ty, names in fields for n in names.split()]})


_Adapters = _struct("she_adapters_args", [
    (_i32, "type base_type"), (_u32, "tokens inputs outputs adapters rank segments"), (_p, "x"), (_i64, "x_stride"), (_p, "down"),
    (_i64, "down_adapter down_rank"), (_p, "up"), (_i64, "up_adapter up_rank"), (_p, "starts which ranks scale base"),
    (_i64, "base_stride"), (_p, "step out"), (_i64, "out_stride")])
_AdaptersGrad = _struct("she_adapters_grad_args", [
    (_i32, "type base_type"), (_u32, "tokens inputs outputs adapters rank segments"), (_p, "dy"), (_i64, "dy_stride"), (_p, "x"),
    (_i64, "x_stride"), (_p, "down"), (_i64, "down_adapter down_rank"), (_p, "up"), (_i64, "up_adapter up_rank"),
    (_p, "starts which ranks scale base"), (_i64, "base_stride"), (_p, "dx"), (_i64, "dx_stride"), (_p, "ddown dup")])
_QkRotate = _struct("she_qk_rotate_args", [
    (_i32, "type interleaved"), (_u32, "tokens q_heads kv_heads head rot places"), (_f32, "eps"), (_p, "q k v"),
    (_i64, "q_token q_head k_token k_head v_token v_head"), (_p, "wq wk cosines sines positions q_out k_out"),
    (_i64, "q_out_token q_out_head k_out_token k_out_head"), (_p, "k_pages v_pages"), (_i64, "page_stride slot_stride page_head"),
    (_u32, "pages page_size"), (_p, "slots")])
_QkRotateGrad = _struct("she_qk_rotate_grad_args", [
    (_i32, "type interleaved"), (_u32, "tokens q_heads kv_heads head rot places"), (_f32, "eps"), (_p, "dq_out dk_out"),
    (_i64, "dq_out_token dq_out_head dk_out_token dk_out_head"), (_p, "q k"), (_i64, "q_token q_head k_token k_head"),
    (_p, "wq wk cosines sines positions dq dk"), (_i64, "dq_token dq_head dk_token dk_head"), (_p, "dwq dwk")])
_AttendPages = _struct("she_attend_pages_args", [
    (_i32, "type"), (_u32, "tokens requests q_heads kv_heads head window"), (_f32, "scale"), (_p, "q"), (_i64, "q_token q_head"),
    (_p, "k_pages v_pages"), (_i64, "page_stride slot_stride page_head"), (_u32, "pages page_size"), (_p, "table"),
    (_i64, "table_stride"), (_u32, "table_width"), (_p, "starts lengths out"), (_i64, "out_token out_head")])

SIGNATURES = {
    "she_adapters": (C.c_int, [_p, C.POINTER(_Adapters)]),
    "she_adapters_grad": (C.c_int, [_p, C.POINTER(_AdaptersGrad)]),
    "she_qk_rotate": (C.c_int, [_p, C.POINTER(_QkRotate)]),
    "she_qk_rotate_grad": (C.c_int, [_p, C.POINTER(_QkRotateGrad)]),
    "she_attend_pages": (C.c_int, [_p, C.POINTER(_AttendPages)]),
    "she_clear_bad_ids": (C.c_int, [_p, C.POINTER(C.c_uint64), C.c_int]),
}

_NO_BASE, _F32, _I32 = -1, 2, 3


def _refuse(text):
    raise SheError(EINVAL, text)


def _half(t, name):
    if t.dtype is torch.bfloat16:
        return 0
    if t.dtype is torch.float16:
        return 1
    _refuse(f"{name} must be bfloat16 or float16, not {t.dtype}")


def _see(t, name, dtype, shape):
    """A tensor's address; refuses one of another type, shape or place, or without a contiguous last axis."""
    if t.dtype is not dtype or t.shape != shape or not t.is_cuda or (t.stride(-1) != 1 and shape[-1] > 1):
        _refuse_tensor(t, name, dtype, shape)
    return t.data_ptr()


def _refuse_tensor(t, name, dtype, shape):
    if t.dtype is not dtype:
        _refuse(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        _refuse(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    if not t.is_cuda:
        _refuse(f"{name} must be on the GPU")
    _refuse(f"{name} must be contiguous along its last axis")


def _line(t, name, dtype, size):
    """A vector that a kernel reads densely; None: a null pointer."""
    return None if t is None else _see(t, name, dtype, (size,))


class Calls:
    """Mixed into Context."""

    def _call(self, fn, args):
        """Runs a call on the context's stream, ordered with torch's current stream where that is another one."""
        if torch._C._cuda_getCurrentRawStream(self._device) == self._stream:
            rc = fn(self._h, C.byref(args))
            if rc:
                self._check(rc)
            return
        if not self._stream and torch.cuda.is_current_stream_capturing():
            _refuse("the default stream cannot be captured: give the context the capturing stream first (set_stream)")
        current = torch.cuda.current_stream(self._device)
        mine = torch.cuda.ExternalStream(self._stream, self._device) if self._stream else torch.cuda.default_stream(self._device)
        mine.wait_stream(current)
        try:
            self._check(fn(self._h, C.byref(args)))
        finally:
            current.wait_stream(mine)

    def adapters(self, x, down, up, starts, which, scale, ranks=None, base=None, step=None, out=None):
        """base + scale[a] * up[a]^T (down[a] x) for the tokens of every segment, a = which[segment] (-1: none).

        x [tokens, inputs]; down [adapters, rank, inputs], up [adapters, rank, outputs]; starts [segments + 1], which [segments],
        ranks [adapters] or None: int32; scale [adapters] float32; base [tokens, outputs] of x's type, float32, or int32 sums times
        step [outputs] float32, or None.  Returns out [tokens, outputs]; base itself may be given for it."""
        ty, dtype = _half(x, "x"), x.dtype
        (T, K), (A, r, N) = x.shape, up.shape
        S = which.shape[0]
        pointers = (_see(x, "x", dtype, (T, K)), _see(down, "down", dtype, (A, r, K)), _see(up, "up", dtype, (A, r, N)),
                    _see(starts, "starts", torch.int32, (S + 1,)), _see(which, "which", torch.int32, (S,)))
        kind, base_at, base_stride = self._base(base, dtype, ty, (T, N))
        if step is not None and kind != _I32:
            _refuse("step belongs to int32 sums")
        if out is None:
            out = torch.empty(T, N, dtype=dtype, device=x.device)
        self._call(self._L.she_adapters, _Adapters(
            ty, kind, T, K, N, A, r, S, pointers[0], x.stride(0), pointers[1], down.stride(0), down.stride(1), pointers[2], up.stride(0),
            up.stride(1), pointers[3], pointers[4], _line(ranks, "ranks", torch.int32, A), _line(scale, "scale", torch.float32, A),
            base_at, base_stride, _line(step, "step", torch.float32, N), _see(out, "out", dtype, (T, N)), out.stride(0)))
        return out

    @staticmethod
    def _base(base, dtype, ty, shape):
        if base is None:
            return _NO_BASE, None, 0
        kind = {dtype: ty, torch.float32: _F32, torch.int32: _I32}.get(base.dtype)
        if kind is None:
            _refuse(f"base must be {dtype}, float32 or int32, not {base.dtype}")
        return kind, _see(base, "base", base.dtype, shape), base.stride(0)

    def adapters_grad(self, dy, x, down, up, starts, which, scale, ranks=None, base=None):
        """Gradients of `adapters` for dy [tokens, outputs]: (dx, ddown, dup), dx with `base` (the gradient that reaches x through the
        projection itself, of x's type or float32) added to it."""
        ty, dtype = _half(x, "x"), x.dtype
        (T, K), (A, r, N) = x.shape, up.shape
        S = which.shape[0]
        pointers = (_see(dy, "dy", dtype, (T, N)), _see(x, "x", dtype, (T, K)), _see(down, "down", dtype, (A, r, K)),
                    _see(up, "up", dtype, (A, r, N)), _see(starts, "starts", torch.int32, (S + 1,)),
                    _see(which, "which", torch.int32, (S,)))
        kind, base_at, base_stride = self._base(base, dtype, ty, (T, K))
        dx = torch.empty(T, K, dtype=dtype, device=x.device)
        ddown = torch.empty(A, r, K, dtype=dtype, device=x.device)
        dup = torch.empty(A, r, N, dtype=dtype, device=x.device)
        self._call(self._L.she_adapters_grad, _AdaptersGrad(
            ty, kind, T, K, N, A, r, S, pointers[0], dy.stride(0), pointers[1], x.stride(0), pointers[2], down.stride(0), down.stride(1),
            pointers[3], up.stride(0), up.stride(1), pointers[4], pointers[5], _line(ranks, "ranks", torch.int32, A),
            _line(scale, "scale", torch.float32, A), base_at, base_stride, dx.data_ptr(), dx.stride(0), ddown.data_ptr(), dup.data_ptr()))
        return dx, ddown, dup

    @staticmethod
    def _rotation(q, k, wq, wk, cos, sin, positions):
        """What the three calls on queries and keys have in common, checked: the first fields of their structs, and pointers."""
        ty, dtype = _half(q, "q"), q.dtype
        (T, Hq, D), Hkv = q.shape, k.shape[1]
        P, half = cos.shape
        _see(q, "q", dtype, (T, Hq, D)), _see(k, "k", dtype, (T, Hkv, D))
        tables = (_line(wq, "wq", torch.float32, D), _line(wk, "wk", torch.float32, D), _see(cos, "cos", torch.float32, (P, half)),
                  _see(sin, "sin", torch.float32, (P, half)), _see(positions, "positions", torch.int32, (T,)))
        if not (cos.is_contiguous() and sin.is_contiguous()):
            _refuse("cos and sin must be contiguous")
        return ty, dtype, (T, Hq, Hkv, D, 2 * half, P), tables

    def qk_rotate(self, q, k, wq, wk, cos, sin, positions, eps=1e-6, interleaved=False, out=None):
        """Norm of every head of q [tokens, q_heads, head] and k [tokens, kv_heads, head] with the weights wq, wk [head] float32 (or
        None), and the rotation by cos, sin [places, rot / 2] float32 at positions [tokens] int32.  Returns (q', k'); out: a pair
        for them, which may be (q, k)."""
        ty, dtype, (T, Hq, Hkv, D, rot, P), tables = self._rotation(q, k, wq, wk, cos, sin, positions)
        if out is None:
            out = torch.empty(T, Hq, D, dtype=dtype, device=q.device), torch.empty(T, Hkv, D, dtype=dtype, device=q.device)
        qo, ko = out
        self._call(self._L.she_qk_rotate, _QkRotate(
            ty, bool(interleaved), T, Hq, Hkv, D, rot, P, eps, q.data_ptr(), k.data_ptr(), None, q.stride(0), q.stride(1), k.stride(0),
            k.stride(1), 0, 0, *tables, _see(qo, "out", dtype, (T, Hq, D)), _see(ko, "out", dtype, (T, Hkv, D)), qo.stride(0),
            qo.stride(1), ko.stride(0), ko.stride(1)))
        return qo, ko

    def qk_rotate_append(self, q, k, v, wq, wk, cos, sin, positions, k_pages, v_pages, slots, eps=1e-6, interleaved=False, out=None):
        """qk_rotate whose keys, with the values v [tokens, kv_heads, head], go to the places slots [tokens] int64 (-1: nowhere) of
        k_pages, v_pages [pages, page_size, kv_heads, head].  Returns q'."""
        ty, dtype, (T, Hq, Hkv, D, rot, P), tables = self._rotation(q, k, wq, wk, cos, sin, positions)
        pages, size = k_pages.shape[:2]
        v_at, pages_at = _see(v, "v", dtype, (T, Hkv, D)), self._pages(k_pages, v_pages, dtype, Hkv, D)
        qo = torch.empty(T, Hq, D, dtype=dtype, device=q.device) if out is None else out
        self._call(self._L.she_qk_rotate, _QkRotate(
            ty, bool(interleaved), T, Hq, Hkv, D, rot, P, eps, q.data_ptr(), k.data_ptr(), v_at, q.stride(0), q.stride(1), k.stride(0),
            k.stride(1), v.stride(0), v.stride(1), *tables, _see(qo, "out", dtype, (T, Hq, D)), None, qo.stride(0), qo.stride(1), 0, 0,
            *pages_at, pages, size, _see(slots, "slots", torch.int64, (T,))))
        return qo

    @staticmethod
    def _pages(k_pages, v_pages, dtype, Hkv, D):
        shape = (*k_pages.shape[:2], Hkv, D)
        at = _see(k_pages, "k_pages", dtype, shape), _see(v_pages, "v_pages", dtype, shape)
        if k_pages.stride() != v_pages.stride():
            _refuse("k_pages and v_pages must have the same strides")
        return *at, *k_pages.stride()[:3]

    def qk_rotate_grad(self, dq_out, dk_out, q, k, wq, wk, cos, sin, positions, eps=1e-6, interleaved=False):
        """Gradients of qk_rotate: (dq, dk, dwq, dwk), the weights' in float32."""
        ty, dtype, (T, Hq, Hkv, D, rot, P), tables = self._rotation(q, k, wq, wk, cos, sin, positions)
        dq, dk = (torch.empty(T, h, D, dtype=dtype, device=q.device) for h in (Hq, Hkv))
        dw = torch.empty(2, D, dtype=torch.float32, device=q.device)
        at = dw.data_ptr()
        self._call(self._L.she_qk_rotate_grad, _QkRotateGrad(
            ty, bool(interleaved), T, Hq, Hkv, D, rot, P, eps, _see(dq_out, "dq_out", dtype, (T, Hq, D)),
            _see(dk_out, "dk_out", dtype, (T, Hkv, D)), dq_out.stride(0), dq_out.stride(1), dk_out.stride(0), dk_out.stride(1),
            q.data_ptr(), k.data_ptr(), q.stride(0), q.stride(1), k.stride(0), k.stride(1), *tables, dq.data_ptr(), dk.data_ptr(),
            dq.stride(0), dq.stride(1), dk.stride(0), dk.stride(1), at, at + 4 * D))
        return dq, dk, dw[0], dw[1]

    def attend_pages(self, q, k_pages, v_pages, table, starts, lengths, scale=None, window=0, out=None):
        """Attention of the new tokens q [tokens, q_heads, head] of every request, starts [requests + 1] int32, over its lengths
        [requests] int32 places in k_pages, v_pages [pages, page_size, kv_heads, head], found through table [requests, width] int32;
        causal, and over the last `window` places alone if that is not 0.  scale: head ** -0.5 if None.  Returns out like q."""
        ty, dtype = _half(q, "q"), q.dtype
        T, Hq, D = q.shape
        pages, size, Hkv = k_pages.shape[:3]
        R, width = table.shape
        q_at, pages_at = _see(q, "q", dtype, (T, Hq, D)), self._pages(k_pages, v_pages, dtype, Hkv, D)
        if not 0 <= window < 1 << 32:
            _refuse("window must be a number of places")
        if out is None:
            out = torch.empty(T, Hq, D, dtype=dtype, device=q.device)
        self._call(self._L.she_attend_pages, _AttendPages(
            ty, T, R, Hq, Hkv, D, window, D ** -0.5 if scale is None else scale, q_at, q.stride(0), q.stride(1), *pages_at, pages, size,
            _see(table, "table", torch.int32, (R, width)), table.stride(0), width, _see(starts, "starts", torch.int32, (R + 1,)),
            _see(lengths, "lengths", torch.int32, (R,)), _see(out, "out", dtype, (T, Hq, D)), out.stride(0), out.stride(1)))
        return out

    def clear_bad_ids(self, reset: bool = True) -> int:
        """Ids out of range in device arrays that these calls have left out since the last reset; waits for the stream."""
        n = C.c_uint64(0)
        self._check(self._L.she_clear_bad_ids(self._h, C.byref(n), int(reset)))
        return n.value
