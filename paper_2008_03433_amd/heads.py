"""The operators of a multi-class softmax head, as include/tron.h declares them, on torch CUDA tensors: argument marshalling only.

Matrices are 2-D tensors whose last dimension is contiguous (or 1-D ones: a single row); the rows' stride is free, and a tensor that is only
read may be expanded over its rows.  Outputs are tensors of the caller's, as elsewhere in this package.  `stream` is a torch stream
or a stream's address, None: the current one of the tensors' device.  Work spaces are taken from torch's allocator on that stream, or
passed as `work` (a uint8 tensor of tron_..._work bytes)."""
from __future__ import annotations

from typing import Optional

from .binding import EINVAL, TronError, _check, load_library

ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
_ACT_NARROW = 256

_torch = None
_types = {}


def _load():
    """The library, and torch (which the package does not import by itself)."""
    global _torch
    lib = load_library()
    if _torch is None:
        import torch
        _types.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.float8_e4m3fn: 3})
        _torch = torch
    return lib


def _refuse(text: str):
    raise TronError(EINVAL, text)


def _current_stream(index: int) -> int:
    """Address of a device's current stream (without the Stream object: 2 of the 11 microseconds of a small call)."""
    raw = getattr(_torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw else _torch.cuda.current_stream(index).cuda_stream


class _Call:
    """One call's tensors: their device, stream and work space."""

    __slots__ = ("name", "device", "index", "stream", "address")

    def __init__(self, name: str, first, stream):
        self.name = name
        if not getattr(first, "is_cuda", False):
            _refuse(f"{name}: CUDA tensors are needed; there is no CPU fallback")
        self.device = first.device
        self.index = first.get_device()
        self.stream = stream
        if stream is None:
            self.address = _current_stream(self.index)
        else:
            self.address = stream if isinstance(stream, int) else stream.cuda_stream

    def matrix(self, t, what, rows=None, cols=None, dtype=None):
        """(address, rows, columns, row stride) of a tensor; (None, .., 0) for None."""
        if t is None:
            return None, rows, cols, 0
        if t.get_device() != self.index:
            _refuse(f"{self.name}: {what} is on {t.device}, other arguments on {self.device}")
        shape = t.shape
        if len(shape) == 2:
            r, c = shape
            ld, unit = t.stride()
        elif len(shape) == 1:
            r, c, ld, unit = 1, shape[0], shape[0], t.stride(0)
        else:
            _refuse(f"{self.name}: {what} has {len(shape)} dimensions, 1 or 2 are taken")
        if c > 1 and unit != 1:
            _refuse(f"{self.name}: the last dimension of {what} is not contiguous")
        if rows is not None and (r != rows or c != cols):
            _refuse(f"{self.name}: {what} is {r} x {c}, expected {rows} x {cols}")
        if dtype is not None and t.dtype != dtype:
            _refuse(f"{self.name}: {what} is of {t.dtype}, expected {dtype}")
        return t.data_ptr(), r, c, ld

    def vector(self, t, what, n):
        """Address of n contiguous floats, or None."""
        if t is None:
            return None
        if t.get_device() != self.index:
            _refuse(f"{self.name}: {what} is on {t.device}, other arguments on {self.device}")
        if t.dtype is not _torch.float32 or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
            _refuse(f"{self.name}: {what} has to be {n} contiguous float32 values")
        return t.data_ptr()

    def type(self, t, what):
        code = _types.get(t.dtype)
        if code is None:
            _refuse(f"{self.name}: {what} is of {t.dtype}; float32, bfloat16, float16 and float8_e4m3fn are known")
        return code

    def work(self, given, needed):
        """(tensor, address, bytes) of a work space, which belongs to the call's stream."""
        if given is not None:
            if given.device != self.device or not given.is_contiguous():
                _refuse(f"{self.name}: the work space has to be contiguous and on {self.device}")
            return given, given.data_ptr(), given.numel() * given.element_size()
        if needed == 0:
            return None, None, 0
        if self.stream is None:
            t = _torch.empty(needed, dtype=_torch.uint8, device=self.device)
        else:
            s = _torch.cuda.ExternalStream(self.stream, device=self.device) if isinstance(self.stream, int) else self.stream
            with _torch.cuda.stream(s):
                t = _torch.empty(needed, dtype=_torch.uint8, device=self.device)
        return t, t.data_ptr(), needed

    def run(self, function, *args):
        if _torch.cuda.current_device() == self.index:
            _check(function(*args))
        else:
            with _torch.cuda.device(self.device):
                _check(function(*args))


def tron_rms_norm(x, y, gain=None, eps=1e-6, residual=None, total=None, scale=None, rstd=None, stream=None) -> None:
    """y = s rstd gain with s = x + residual, written to `total` when given; rows of x.  y of x's type, or float8_e4m3fn with `scale`."""
    lib = _load()
    call = _Call("tron_rms_norm", x, stream)
    xp, m, d, ldx = call.matrix(x, "x")
    rp, _, _, ldr = call.matrix(residual, "residual", m, d, x.dtype)
    tp, _, _, ldt = call.matrix(total, "total", m, d, x.dtype)
    yp, _, _, ldy = call.matrix(y, "y", m, d)
    call.run(lib.tron_rms_norm, m, d, call.type(x, "x"), xp, ldx, rp, ldr, call.vector(gain, "gain", d), eps, tp, ldt, call.type(y, "y"), yp, ldy,
             call.vector(scale, "scale", m), call.vector(rstd, "rstd", m), call.address)


def tron_rms_norm_grad_work(m, d) -> int:
    return load_library().tron_rms_norm_grad_work(m, d)


def tron_rms_norm_grad(total, rstd, dy, dx, gain=None, dtotal=None, dgain=None, work=None, stream=None) -> None:
    """dx, the gradient of x and of the residual, and dgain when given, from the forward call's total (x itself without a residual) and rstd."""
    lib = _load()
    call = _Call("tron_rms_norm_grad", total, stream)
    sp, m, d, lds = call.matrix(total, "total")
    dyp, _, _, lddy = call.matrix(dy, "dy", m, d, total.dtype)
    dtp, _, _, lddt = call.matrix(dtotal, "dtotal", m, d, total.dtype)
    dxp, _, _, lddx = call.matrix(dx, "dx", m, d, total.dtype)
    if rstd is None:
        _refuse("tron_rms_norm_grad: rstd is needed")
    space, wp, wb = call.work(work, lib.tron_rms_norm_grad_work(m, d) if dgain is not None else 0)
    call.run(lib.tron_rms_norm_grad, m, d, call.type(total, "total"), sp, lds, call.vector(rstd, "rstd", m), call.vector(gain, "gain", d), dyp, lddy, dtp, lddt,
             dxp, lddx, call.vector(dgain, "dgain", d), wp, wb, call.address)


def tron_linear_work(m, n, k, dtype) -> int:
    lib = _load()
    return lib.tron_linear_work(m, n, k, _types.get(dtype, -1))


def tron_linear(x, w, y, bias=None, act=ACT_NONE, residual=None, pre=None, x_scale=None, w_scale=None, work=None, stream=None) -> None:
    """y = act(x w' + bias) + residual; the values before the activation go to `pre` when given.  x (m x k) and w (n x k) of one type:
    bfloat16, float16, or float8_e4m3fn with x_scale (m) and w_scale (n)."""
    lib = _load()
    call = _Call("tron_linear", x, stream)
    xp, m, k, ldx = call.matrix(x, "x")
    if w.dim() != 2:
        _refuse("tron_linear: w has to have 2 dimensions")
    n = w.shape[0]
    wp, _, _, ldw = call.matrix(w, "w", n, k, x.dtype)
    yp, _, _, ldy = call.matrix(y, "y", m, n)
    rp, _, _, ldr = call.matrix(residual, "residual", m, n, y.dtype)
    pp, _, _, ldp = call.matrix(pre, "pre", m, n, y.dtype)
    kind = call.type(x, "x")
    space, sp, sb = call.work(work, lib.tron_linear_work(m, n, k, kind))
    call.run(lib.tron_linear, m, n, k, kind, xp, ldx, call.vector(x_scale, "x_scale", m), wp, ldw, call.vector(w_scale, "w_scale", n),
             call.vector(bias, "bias", n), act, rp, ldr, call.type(y, "y"), yp, ldy, pp, ldp, sp, sb, call.address)


def tron_linear_grad_work(m, n, k, act=ACT_NONE, want_dx=True, want_dw=True, want_dbias=True, narrow=False) -> int:
    return load_library().tron_linear_grad_work(m, n, k, act | _ACT_NARROW if narrow else act, int(want_dx), int(want_dw), int(want_dbias))


def tron_linear_grad(x, w, dy, dx=None, dw=None, dbias=None, act=ACT_NONE, pre=None, work=None, stream=None, narrow=False) -> None:
    """The gradients that are given: dx (m x k), dw (n x k, of any float type), dbias (n).  x may be None without dw, w without dx.
    narrow: the products take the gradient before the activation rounded to 16 bits, for about half the time."""
    lib = _load()
    if narrow:
        act |= _ACT_NARROW
    call = _Call("tron_linear_grad", dy, stream)
    dyp, m, n, lddy = call.matrix(dy, "dy")
    if (dw is not None and x is None) or (dx is not None and w is None):
        _refuse("tron_linear_grad: x is needed for dw, and w for dx")
    k = next((t.shape[-1] for t in (x, w) if t is not None), 1)
    xp, _, _, ldx = call.matrix(x, "x", m, k, dy.dtype)
    wp, _, _, ldw = call.matrix(w, "w", n, k, dy.dtype)
    pp, _, _, ldp = call.matrix(pre, "pre", m, n, dy.dtype)
    dxp, _, _, lddx = call.matrix(dx, "dx", m, k, dy.dtype)
    dwp, _, _, lddw = call.matrix(dw, "dw", n, k)
    space, sp, sb = call.work(work, lib.tron_linear_grad_work(m, n, k, act, int(dx is not None), int(dw is not None), int(dbias is not None)))
    call.run(lib.tron_linear_grad, m, n, k, call.type(dy, "dy"), xp, ldx, wp, ldw, dyp, lddy, act, pp, ldp, dxp, lddx,
             0 if dw is None else call.type(dw, "dw"), dwp, lddw, call.vector(dbias, "dbias", n), sp, sb, call.address)


def _lists(call, ids, t, m):
    """(K, ids' address, bytes, row stride, t's address, row stride)."""
    ip, _, K, ldi = call.matrix(ids, "ids", m, ids.shape[-1])
    if ids.dtype not in (_torch.int32, _torch.int64):
        _refuse(f"{call.name}: ids are of {ids.dtype}, expected int32 or int64")
    tp, _, _, ldt = call.matrix(t, "t", m, K, _torch.float32)
    return K, ip, 4 if ids.dtype == _torch.int32 else 8, ldi, tp, ldt


def tron_distill_work(m, V) -> int:
    return load_library().tron_distill_work(m, V)


def tron_distill(z, ids, t, loss, lse=None, temperature=1.0, weight=None, dz=None, work=None, stream=None) -> None:
    """loss (m floats) of the logits z (m x V) against the teacher's listed entries ids, t (m x K); lse and the gradient dz when given."""
    lib = _load()
    call = _Call("tron_distill", z, stream)
    zp, m, V, ldz = call.matrix(z, "z")
    K, ip, ib, ldi, tp, ldt = _lists(call, ids, t, m)
    dp, _, _, lddz = call.matrix(dz, "dz", m, V, z.dtype)
    space, sp, sb = call.work(work, lib.tron_distill_work(m, V))
    call.run(lib.tron_distill, m, V, call.type(z, "z"), zp, ldz, K, ip, ib, ldi, tp, ldt, temperature, call.vector(weight, "weight", m),
             call.vector(loss, "loss", m), call.vector(lse, "lse", m), dp, lddz, sp, sb, call.address)


def tron_distill_grad(z, lse, ids, t, dz, temperature=1.0, weight=None, stream=None) -> None:
    """dz of tron_distill, from its lse."""
    lib = _load()
    call = _Call("tron_distill_grad", z, stream)
    zp, m, V, ldz = call.matrix(z, "z")
    K, ip, ib, ldi, tp, ldt = _lists(call, ids, t, m)
    dp, _, _, lddz = call.matrix(dz, "dz", m, V, z.dtype)
    call.run(lib.tron_distill_grad, m, V, call.type(z, "z"), zp, ldz, call.vector(lse, "lse", m), K, ip, ib, ldi, tp, ldt, temperature,
             call.vector(weight, "weight", m), dp, lddz, call.address)


def tron_distill_hv(z, lse, u, hu, ids=None, t=None, temperature=1.0, weight=None, work=None, stream=None) -> None:
    """hu = the Hessian of sum(loss) with respect to z, times u.  ids and t as in the forward call, or both None."""
    lib = _load()
    call = _Call("tron_distill_hv", z, stream)
    zp, m, V, ldz = call.matrix(z, "z")
    if (ids is None) != (t is None):
        _refuse("tron_distill_hv: ids and t go together")
    K, ip, ib, ldi, tp, ldt = (-1, None, 8, 0, None, 0) if ids is None else _lists(call, ids, t, m)
    up, _, _, ldu = call.matrix(u, "u", m, V, z.dtype)
    hp, _, _, ldh = call.matrix(hu, "hu", m, V, z.dtype)
    space, sp, sb = call.work(work, lib.tron_distill_work(m, V))
    call.run(lib.tron_distill_hv, m, V, call.type(z, "z"), zp, ldz, call.vector(lse, "lse", m), up, ldu, K, ip, ib, ldi, tp, ldt, temperature,
             call.vector(weight, "weight", m), hp, ldh, sp, sb, call.address)


# --------------------------------------------------------------------------- convenience wrapper
class SoftmaxHead:
    """The problem that a softmax head is trained on, with the calls of Dataset:

        f(W) = 1/2 W.W + C sum_i loss_i(z_i),   z = X W',   X = rms_norm(hidden + residual) gain

    for hidden states (m x d, bfloat16 or float16) and a teacher's ids and t (m x K).  W is n x d float32; the products take it rounded to
    the states' type.  fun_grad keeps the logits of its W for hv, as Dataset keeps D.

    hv is linear in its direction, whose size is the caller's (a gradient's, in the first product of a solve).  In float16 the products take it
    times a power of two, and the result by its reciprocal, so that neither the direction nor X V' leaves the type's range."""

    _LARGEST = 12   # log2 of a bound on |X V'|: four bits below float16's largest value, for weights and roundings

    def __init__(self, hidden, ids, t, gain=None, residual=None, eps=1e-6, temperature=1.0, weight=None):
        _load()
        self.m, self.d = hidden.shape
        self.ids, self.t, self.temperature, self.weight = ids, t, temperature, weight
        self.X = _torch.empty_like(hidden, memory_format=_torch.contiguous_format)
        tron_rms_norm(hidden, self.X, gain=gain, eps=eps, residual=residual)
        self.loss = _torch.empty(self.m, dtype=_torch.float32, device=hidden.device)
        self.lse = _torch.empty_like(self.loss)
        self.z = None
        self._reach = self._exponent(self.X.abs().sum(1, dtype=_torch.float32)) if self.X.dtype == _torch.float16 and self.m else None

    @staticmethod
    def _exponent(a):
        """e with |a| <= 2^e in every element, on the device."""
        return _torch.frexp(_torch.linalg.vector_norm(a, ord=float("inf"))).exponent

    def _scale(self, V):
        """The power of two by which |V| and |X V'| are at most 2^_LARGEST (|X V'| <= the largest sum of a row's |x| times the largest |v|)."""
        return _torch.exp2((self._LARGEST - self._reach.clamp(min=0) - self._exponent(V)).float().clamp(-120.0, 120.0))

    def _logits(self, W):
        """X W' of weights in the states' type."""
        z = _torch.empty((self.m, W.shape[0]), dtype=self.X.dtype, device=W.device)
        tron_linear(self.X, W, z)
        return z

    def _to_weights(self, dz, C, V, out):
        tron_linear_grad(self.X, None, dz, dw=out)
        out.mul_(C).add_(V)

    def fun_grad(self, C, W, G: Optional[object] = None) -> float:
        """f(W); the gradient goes to G (n x d float32) when given."""
        self.z = self._logits(W.to(self.X.dtype))
        dz = None if G is None else _torch.empty_like(self.z)
        tron_distill(self.z, self.ids, self.t, self.loss, self.lse, temperature=self.temperature, weight=self.weight, dz=dz)
        if G is not None:
            self._to_weights(dz, C, W, G)
        return 0.5 * float((W.double() ** 2).sum()) + C * float(self.loss.double().sum())

    def hv(self, C, V, HV) -> None:
        """HV = V + C X' (H_z (X V')) for the W of the last fun_grad."""
        if self.z is None:
            raise TronError(-4, "SoftmaxHead.hv before fun_grad")
        if self._reach is None:   # bfloat16 has the range of 32 bits
            direction = V.to(self.X.dtype)
        else:
            scale = self._scale(V)
            C, direction = C / scale, _torch.mul(V, scale, out=_torch.empty_like(V, dtype=self.X.dtype))
        u = self._logits(direction)
        tron_distill_hv(self.z, self.lse, u, u, ids=self.ids, t=self.t, temperature=self.temperature, weight=self.weight)
        self._to_weights(u, C, V, HV)
