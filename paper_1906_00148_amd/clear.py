"""The clear side of split inference on torch tensors (argument marshalling only; include/she_clear.h has the definitions).

`Calls` is the part of a Context that runs between a decryption and the next encryption: adapters beside a shared projection,
norms and rotation of queries and keys, attention over a paged cache.  Tensors are on the context's GPU (refused elsewhere), in
bfloat16 or float16 where nothing else is said, with a contiguous last axis; their other strides are free.  Gradients have calls of
their own: backward through a result raises, and what a call writes into (out, pages) counts as changed in place.  Work is enqueued
on the context's stream: when torch's current stream is another one, that work waits for it and it waits for the work.
"""
from __future__ import annotations

import ctypes as C
import struct

EINVAL = -1


class _Later:
    """Stands for torch until something of it is used: what a Context does on ciphertexts alone needs none."""

    def __getattr__(self, name):
        global torch
        import torch
        return getattr(torch, name)


torch = _Later()


class SheError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"she error {code}: {text}")
        self.code = code


class _Layout:
    """A struct of include/she_clear.h, packed into bytes of the native layout (a fifth of the time that a ctypes structure takes)."""

    def __init__(self, name, fields):
        """`fields`: a struct format character and the names that have it, in the header's order."""
        self.name, self.fields = name, [(n, ty) for ty, names in fields for n in names.split()]
        packer = struct.Struct("@" + "".join(ty for _, ty in self.fields))
        self.pack, self.size = packer.pack, packer.size

    def offsets(self):
        at = {}
        for k, (name, ty) in enumerate(self.fields):
            before = "@" + "".join(t for _, t in self.fields[:k])
            at[name] = struct.calcsize(before + ty) - struct.calcsize(ty)
        return at


_ADAPTERS = _Layout("she_adapters_args", [
    ("i", "type base_type"), ("I", "tokens inputs outputs adapters rank segments"), ("P", "x"), ("q", "x_stride"), ("P", "down"),
    ("q", "down_adapter down_rank"), ("P", "up"), ("q", "up_adapter up_rank"), ("P", "starts which ranks scale base"),
    ("q", "base_stride"), ("P", "step out"), ("q", "out_stride")])
_ADAPTERS_GRAD = _Layout("she_adapters_grad_args", [
    ("i", "type base_type"), ("I", "tokens inputs outputs adapters rank segments"), ("P", "dy"), ("q", "dy_stride"), ("P", "x"),
    ("q", "x_stride"), ("P", "down"), ("q", "down_adapter down_rank"), ("P", "up"), ("q", "up_adapter up_rank"),
    ("P", "starts which ranks scale base"), ("q", "base_stride"), ("P", "dx"), ("q", "dx_stride"), ("P", "ddown dup")])
_QK_ROTATE = _Layout("she_qk_rotate_args", [
    ("i", "type interleaved"), ("I", "tokens q_heads kv_heads head rot places"), ("f", "eps"), ("P", "q k v"),
    ("q", "q_token q_head k_token k_head v_token v_head"), ("P", "wq wk cosines sines positions q_out k_out"),
    ("q", "q_out_token q_out_head k_out_token k_out_head"), ("P", "k_pages v_pages"), ("q", "page_stride slot_stride page_head"),
    ("I", "pages page_size"), ("P", "slots")])
_QK_ROTATE_GRAD = _Layout("she_qk_rotate_grad_args", [
    ("i", "type interleaved"), ("I", "tokens q_heads kv_heads head rot places"), ("f", "eps"), ("P", "dq_out dk_out"),
    ("q", "dq_out_token dq_out_head dk_out_token dk_out_head"), ("P", "q k"), ("q", "q_token q_head k_token k_head"),
    ("P", "wq wk cosines sines positions dq dk"), ("q", "dq_token dq_head dk_token dk_head"), ("P", "dwq dwk")])
_ATTEND_PAGES = _Layout("she_attend_pages_args", [
    ("i", "type"), ("I", "tokens requests q_heads kv_heads head window"), ("f", "scale"), ("P", "q"), ("q", "q_token q_head"),
    ("P", "k_pages v_pages"), ("q", "page_stride slot_stride page_head"), ("I", "pages page_size"), ("P", "table"),
    ("q", "table_stride"), ("I", "table_width"), ("P", "starts lengths out"), ("q", "out_token out_head")])
LAYOUTS = [_ADAPTERS, _ADAPTERS_GRAD, _QK_ROTATE, _QK_ROTATE_GRAD, _ATTEND_PAGES]

SIGNATURES = {**{layout.name[:-len("_args")]: (C.c_int, [C.c_void_p, C.c_char_p]) for layout in LAYOUTS},
              "she_clear_bad_ids": (C.c_int, [C.c_void_p, C.POINTER(C.c_uint64), C.c_int]),
              "she_clear_device": (C.c_int, [C.c_void_p])}

_NO_BASE, _F32, _I32 = -1, 2, 3


def _refuse(text):
    raise SheError(EINVAL, text)


def _first(t, name, device):
    """Of the tensor that decides a call's type: that type, torch's name of it, its shape, address and strides."""
    dtype, shape, strides = t.dtype, t.shape, t.stride()
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        _refuse(f"{name} must be bfloat16 or float16, not {dtype}")
    if t.get_device() != device or (strides[-1] != 1 and shape[-1] > 1):
        _refuse_tensor(t, name, dtype, shape, device)
    return int(dtype is torch.float16), dtype, shape, t.data_ptr(), strides


def _see(t, name, dtype, shape, device):
    """A tensor's address and strides; refuses one of another type, shape or place, or without a contiguous last axis."""
    strides = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or (strides[-1] != 1 and shape[-1] > 1):
        _refuse_tensor(t, name, dtype, shape, device)
    return t.data_ptr(), strides


def _refuse_tensor(t, name, dtype, shape, device):
    if t.dtype is not dtype:
        _refuse(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        _refuse(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.get_device() != device:
        _refuse(f"{name} must be on the context's GPU, cuda:{device}, not {t.device}")
    _refuse(f"{name} must be contiguous{' along its last axis' if len(shape) > 1 else ''}")


def _line(t, name, dtype, size, device):
    """The address of a vector that a kernel reads densely; None: a null pointer."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != (size,) or t.get_device() != device or not t.is_contiguous():
        _refuse_tensor(t, name, dtype, (size,), device)
    return t.data_ptr()


_unrecorded = None


def _barred(result, instead, *inputs):
    """`result`, through which backward raises: a gradient of the inputs would get lost there."""
    global _unrecorded
    if _unrecorded is None:
        class Unrecorded(torch.autograd.Function):
            @staticmethod
            def forward(ctx, result, instead, *inputs):
                ctx.instead = instead
                return result.detach()

            @staticmethod
            def backward(ctx, *_):
                _refuse(f"this call's gradient is not recorded: {ctx.instead}")
        _unrecorded = Unrecorded
    return _unrecorded.apply(result, instead, *inputs)


class Calls:
    """Mixed into Context."""

    def _call(self, fn, args):
        """Runs a call on the context's GPU and stream, ordered with torch's current stream there where that is another one."""
        if torch._C._cuda_getCurrentRawStream(self._device) == self._stream:
            rc = fn(self._h, args)
            if rc and torch._C._cuda_getDevice() != self._device:  # refused for that reason, if not for another
                with torch.cuda.device(self._device):
                    rc = fn(self._h, args)
            if rc:
                self._check(rc)
            return
        if not self._stream and torch.cuda.is_current_stream_capturing():
            _refuse("the default stream cannot be captured: give the context the capturing stream first (set_stream)")
        current = torch.cuda.current_stream(self._device)
        mine = torch.cuda.ExternalStream(self._stream, self._device) if self._stream else torch.cuda.default_stream(self._device)
        mine.wait_stream(current)
        try:
            with torch.cuda.device(self._device):
                self._check(fn(self._h, args))
        finally:
            current.wait_stream(mine)

    def adapters(self, x, down, up, starts, which, scale, ranks=None, base=None, step=None, out=None):
        """base + scale[a] * up[a]^T (down[a] x) for the tokens of every segment, a = which[segment] (-1: none).

        x [tokens, inputs]; down [adapters, rank, inputs], up [adapters, rank, outputs]; starts [segments + 1], which [segments],
        ranks [adapters] or None: int32; scale [adapters] float32; base [tokens, outputs] of x's type, float32, or int32 sums times
        step [outputs] float32, or None.  Returns out [tokens, outputs]; base itself may be given for it."""
        dev = self._device
        ty, dtype, (T, K), x_at, xs = _first(x, "x", dev)
        A, r, N = up.shape
        S = which.shape[0]
        down_at, ds = _see(down, "down", dtype, (A, r, K), dev)
        up_at, us = _see(up, "up", dtype, (A, r, N), dev)
        kind, base_at, base_stride = self._base(base, dtype, ty, (T, N), dev)
        if step is not None and kind != _I32:
            _refuse("step belongs to int32 sums")
        given = out is not None
        if not given:
            out = torch.empty(T, N, dtype=dtype, device=x.device)
            out_at, out_stride = out.data_ptr(), N
        else:
            out_at, (out_stride, _) = _see(out, "out", dtype, (T, N), dev)
        self._call(self._L.she_adapters, _ADAPTERS.pack(
            ty, kind, T, K, N, A, r, S, x_at, xs[0], down_at, ds[0], ds[1], up_at, us[0], us[1], _line(starts, "starts", torch.int32, S + 1, dev),
            _line(which, "which", torch.int32, S, dev), _line(ranks, "ranks", torch.int32, A, dev), _line(scale, "scale", torch.float32, A, dev),
            base_at, base_stride, _line(step, "step", torch.float32, N, dev), out_at, out_stride))
        if given:
            torch.autograd.graph.increment_version(out)
        if torch.is_grad_enabled() and (x.requires_grad or down.requires_grad or up.requires_grad or scale.requires_grad or
                                        base is not None and base.requires_grad or step is not None and step.requires_grad):
            return _barred(out, "use adapters_grad", x, down, up, scale, base, step)
        return out

    @staticmethod
    def _base(base, dtype, ty, shape, dev):
        if base is None:
            return _NO_BASE, 0, 0
        its = base.dtype
        kind = ty if its is dtype else _F32 if its is torch.float32 else _I32 if its is torch.int32 else None
        if kind is None:
            _refuse(f"base must be {dtype}, float32 or int32, not {its}")
        at, strides = _see(base, "base", its, shape, dev)
        return kind, at, strides[0]

    def adapters_grad(self, dy, x, down, up, starts, which, scale, ranks=None, base=None):
        """Gradients of `adapters` for dy [tokens, outputs]: (dx, ddown, dup), dx with `base` (the gradient that reaches x through the
        projection itself, of x's type or float32) added to it."""
        dev = self._device
        ty, dtype, (T, K), x_at, xs = _first(x, "x", dev)
        A, r, N = up.shape
        S = which.shape[0]
        dy_at, dys = _see(dy, "dy", dtype, (T, N), dev)
        down_at, ds = _see(down, "down", dtype, (A, r, K), dev)
        up_at, us = _see(up, "up", dtype, (A, r, N), dev)
        kind, base_at, base_stride = self._base(base, dtype, ty, (T, K), dev)
        lines = (_line(starts, "starts", torch.int32, S + 1, dev), _line(which, "which", torch.int32, S, dev),
                 _line(ranks, "ranks", torch.int32, A, dev), _line(scale, "scale", torch.float32, A, dev))
        at = x.device
        dx, ddown = torch.empty(T, K, dtype=dtype, device=at), torch.empty(A, r, K, dtype=dtype, device=at)
        dup = torch.empty(A, r, N, dtype=dtype, device=at)
        self._call(self._L.she_adapters_grad, _ADAPTERS_GRAD.pack(
            ty, kind, T, K, N, A, r, S, dy_at, dys[0], x_at, xs[0], down_at, ds[0], ds[1], up_at, us[0], us[1], *lines,
            base_at, base_stride, dx.data_ptr(), K, ddown.data_ptr(), dup.data_ptr()))
        if torch.is_grad_enabled() and (dy.requires_grad or x.requires_grad or down.requires_grad or up.requires_grad or
                                        scale.requires_grad or base is not None and base.requires_grad):
            return tuple(_barred(t, "there is no second one", dy, x, down, up, scale, base) for t in (dx, ddown, dup))
        return dx, ddown, dup

    @staticmethod
    def _rotation(q, k, wq, wk, cos, sin, positions, dev):
        """What the three calls on queries and keys have in common, checked: type, sizes, addresses and strides."""
        ty, dtype, (T, Hq, D), q_at, qs = _first(q, "q", dev)
        Hkv = k.shape[1]
        P, half = cos.shape
        k_at, ks = _see(k, "k", dtype, (T, Hkv, D), dev)
        f32, table = torch.float32, (P, half)
        (c_at, cs), (s_at, ss) = _see(cos, "cos", f32, table, dev), _see(sin, "sin", f32, table, dev)
        if not (cs[0] == ss[0] == half or cos.is_contiguous() and sin.is_contiguous()):
            _refuse("cos and sin must be contiguous")
        tables = _line(wq, "wq", f32, D, dev), _line(wk, "wk", f32, D, dev), c_at, s_at, _line(positions, "positions", torch.int32, T, dev)
        return ty, dtype, (T, Hq, Hkv, D, 2 * half, P), (q_at, k_at), (qs[0], qs[1], ks[0], ks[1]), tables

    @staticmethod
    def _rotation_wanted(q, k, wq, wk, cos, sin):
        return (q.requires_grad or k.requires_grad or wq is not None and wq.requires_grad or wk is not None and wk.requires_grad or
                cos.requires_grad or sin.requires_grad)

    def qk_rotate(self, q, k, wq, wk, cos, sin, positions, eps=1e-6, interleaved=False, out=None):
        """Norm of every head of q [tokens, q_heads, head] and k [tokens, kv_heads, head] with the weights wq, wk [head] float32 (or
        None), and the rotation by cos, sin [places, rot / 2] float32 at positions [tokens] int32.  Returns (q', k'); out: a pair
        for them, which may be (q, k)."""
        dev = self._device
        ty, dtype, (T, Hq, Hkv, D, rot, P), at, strides, tables = self._rotation(q, k, wq, wk, cos, sin, positions, dev)
        given = out is not None
        if not given:
            out = torch.empty(T, Hq, D, dtype=dtype, device=q.device), torch.empty(T, Hkv, D, dtype=dtype, device=q.device)
        q_out, qs = _see(out[0], "out", dtype, (T, Hq, D), dev)
        k_out, ks = _see(out[1], "out", dtype, (T, Hkv, D), dev)
        self._call(self._L.she_qk_rotate, _QK_ROTATE.pack(
            ty, bool(interleaved), T, Hq, Hkv, D, rot, P, eps, *at, 0, *strides, 0, 0, *tables, q_out, k_out, qs[0], qs[1], ks[0], ks[1],
            0, 0, 0, 0, 0, 0, 0, 0))
        if given:
            torch.autograd.graph.increment_version((out[0], out[1]))
        if torch.is_grad_enabled() and self._rotation_wanted(q, k, wq, wk, cos, sin):
            return tuple(_barred(t, "use qk_rotate_grad", q, k, wq, wk, cos, sin) for t in (out[0], out[1]))
        return out[0], out[1]

    def qk_rotate_append(self, q, k, v, wq, wk, cos, sin, positions, k_pages, v_pages, slots, eps=1e-6, interleaved=False, out=None):
        """qk_rotate whose keys, with the values v [tokens, kv_heads, head], go to the places slots [tokens] int64 (-1: nowhere) of
        k_pages, v_pages [pages, page_size, kv_heads, head].  Returns q'."""
        dev = self._device
        ty, dtype, (T, Hq, Hkv, D, rot, P), at, strides, tables = self._rotation(q, k, wq, wk, cos, sin, positions, dev)
        v_at, vs = _see(v, "v", dtype, (T, Hkv, D), dev)
        pages_at, pages, size = self._pages(k_pages, v_pages, dtype, Hkv, D, dev)
        written = (k_pages, v_pages) if out is None else (k_pages, v_pages, out)
        if out is None:
            out = torch.empty(T, Hq, D, dtype=dtype, device=q.device)
        q_out, qs = _see(out, "out", dtype, (T, Hq, D), dev)
        self._call(self._L.she_qk_rotate, _QK_ROTATE.pack(
            ty, bool(interleaved), T, Hq, Hkv, D, rot, P, eps, *at, v_at, *strides, vs[0], vs[1], *tables, q_out, 0, qs[0], qs[1], 0, 0,
            *pages_at, pages, size, _line(slots, "slots", torch.int64, T, dev)))
        torch.autograd.graph.increment_version(written)
        if torch.is_grad_enabled() and (v.requires_grad or self._rotation_wanted(q, k, wq, wk, cos, sin)):
            return _barred(out, "a cache is for inference", q, k, v, wq, wk, cos, sin)
        return out

    @staticmethod
    def _pages(k_pages, v_pages, dtype, Hkv, D, dev):
        """(addresses and strides, pages, page size)"""
        pages, size = k_pages.shape[:2]
        k_at, strides = _see(k_pages, "k_pages", dtype, (pages, size, Hkv, D), dev)
        v_at, other = _see(v_pages, "v_pages", dtype, (pages, size, Hkv, D), dev)
        if strides != other:
            _refuse("k_pages and v_pages must have the same strides")
        return (k_at, v_at, strides[0], strides[1], strides[2]), pages, size

    def qk_rotate_grad(self, dq_out, dk_out, q, k, wq, wk, cos, sin, positions, eps=1e-6, interleaved=False):
        """Gradients of qk_rotate: (dq, dk, dwq, dwk), the weights' in float32."""
        dev = self._device
        ty, dtype, (T, Hq, Hkv, D, rot, P), at, strides, tables = self._rotation(q, k, wq, wk, cos, sin, positions, dev)
        dq_at, dqs = _see(dq_out, "dq_out", dtype, (T, Hq, D), dev)
        dk_at, dks = _see(dk_out, "dk_out", dtype, (T, Hkv, D), dev)
        dq, dk = (torch.empty(T, h, D, dtype=dtype, device=q.device) for h in (Hq, Hkv))
        dw = torch.empty(2, D, dtype=torch.float32, device=q.device)
        dw_at = dw.data_ptr()
        self._call(self._L.she_qk_rotate_grad, _QK_ROTATE_GRAD.pack(
            ty, bool(interleaved), T, Hq, Hkv, D, rot, P, eps, dq_at, dk_at, dqs[0], dqs[1], dks[0], dks[1], *at, *strides, *tables,
            dq.data_ptr(), dk.data_ptr(), Hq * D, D, Hkv * D, D, dw_at, dw_at + 4 * D))
        if torch.is_grad_enabled() and (dq_out.requires_grad or dk_out.requires_grad or self._rotation_wanted(q, k, wq, wk, cos, sin)):
            return tuple(_barred(t, "there is no second one", dq_out, dk_out, q, k, wq, wk, cos, sin) for t in (dq, dk, dw[0], dw[1]))
        return dq, dk, dw[0], dw[1]

    def attend_pages(self, q, k_pages, v_pages, table, starts, lengths, scale=None, window=0, out=None):
        """Attention of the new tokens q [tokens, q_heads, head] of every request, starts [requests + 1] int32, over its lengths
        [requests] int32 places in k_pages, v_pages [pages, page_size, kv_heads, head], found through table [requests, width] int32;
        causal, and over the last `window` places alone if that is not 0.  scale: head ** -0.5 if None.  Returns out like q."""
        dev = self._device
        ty, dtype, (T, Hq, D), q_at, qs = _first(q, "q", dev)
        Hkv = k_pages.shape[2]
        R, width = table.shape
        pages_at, pages, size = self._pages(k_pages, v_pages, dtype, Hkv, D, dev)
        table_at, ts = _see(table, "table", torch.int32, (R, width), dev)
        if not 0 <= window < 1 << 32:
            _refuse("window must be a number of places")
        given = out is not None
        if not given:
            out = torch.empty(T, Hq, D, dtype=dtype, device=q.device)
            out_at, out_token, out_head = out.data_ptr(), Hq * D, D
        else:
            out_at, (out_token, out_head, _) = _see(out, "out", dtype, (T, Hq, D), dev)
        self._call(self._L.she_attend_pages, _ATTEND_PAGES.pack(
            ty, T, R, Hq, Hkv, D, window, D ** -0.5 if scale is None else scale, q_at, qs[0], qs[1], *pages_at, pages, size, table_at, ts[0],
            width, _line(starts, "starts", torch.int32, R + 1, dev), _line(lengths, "lengths", torch.int32, R, dev), out_at, out_token, out_head))
        if given:
            torch.autograd.graph.increment_version(out)
        if torch.is_grad_enabled() and (q.requires_grad or k_pages.requires_grad or v_pages.requires_grad):
            return _barred(out, "a cache is for inference", q, k_pages, v_pages)
        return out

    def clear_bad_ids(self, reset: bool = True) -> int:
        """Ids out of range in device arrays that these calls have left out since the last reset; waits for the stream."""
        n = C.c_uint64(0)
        with torch.cuda.device(self._device):
            self._check(self._L.she_clear_bad_ids(self._h, C.byref(n), int(reset)))
        return n.value
