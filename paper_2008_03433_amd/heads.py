"""The operators of a multi-class softmax head and of the tokens at both its ends, as include/tron.h declares them, on torch CUDA tensors: argument marshalling only.

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
_FLOAT, _INT, _FLAG = [], [], []   # what lists of floats, of whole numbers and of flags are made of
_raw_stream = _raw_device = None   # torch's own functions behind current_stream and current_device, which cost 2 of the 11 microseconds of a small call


def _load():
    """The library, and torch (which the package does not import by itself)."""
    global _torch, _raw_stream, _raw_device
    lib = load_library()
    if _torch is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
        _raw_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        _types.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.float8_e4m3fn: 3, torch.int8: 4})
        _FLOAT[:], _INT[:], _FLAG[:] = [torch.float32], [torch.int32], [torch.bool, torch.uint8]
        _torch = torch
    return lib


def _refuse(text: str):
    raise TronError(EINVAL, text)


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
            self.address = _raw_stream(self.index)
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
            _refuse(f"{self.name}: {what} is of {t.dtype}; float32, bfloat16, float16, float8_e4m3fn and int8 are known")
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
        if _raw_device() == self.index:
            _check(function(*args))
        else:
            with _torch.cuda.device(self.device):
                _check(function(*args))


def tron_rms_norm(x, y, gain=None, eps=1e-6, residual=None, total=None, scale=None, rstd=None, stream=None) -> None:
    """y = s rstd gain with s = x + residual, written to `total` when given; rows of x.  y of x's type, or float8_e4m3fn or int8 with `scale`."""
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


def tron_layer_norm(x, y, gain=None, shift=None, eps=1e-5, residual=None, total=None, scale=None, mean=None, rstd=None, stream=None) -> None:
    """y = (s - mean) rstd gain + shift with s = x + residual, written to `total` when given; rows of x.  y of x's type, or float8_e4m3fn or int8
    with `scale`."""
    lib = _load()
    call = _Call("tron_layer_norm", x, stream)
    xp, m, d, ldx = call.matrix(x, "x")
    rp, _, _, ldr = call.matrix(residual, "residual", m, d, x.dtype)
    tp, _, _, ldt = call.matrix(total, "total", m, d, x.dtype)
    yp, _, _, ldy = call.matrix(y, "y", m, d)
    call.run(lib.tron_layer_norm, m, d, call.type(x, "x"), xp, ldx, rp, ldr, call.vector(gain, "gain", d), call.vector(shift, "shift", d), eps, tp, ldt,
             call.type(y, "y"), yp, ldy, call.vector(scale, "scale", m), call.vector(mean, "mean", m), call.vector(rstd, "rstd", m), call.address)


def tron_layer_norm_grad_work(m, d) -> int:
    return load_library().tron_layer_norm_grad_work(m, d)


def tron_layer_norm_grad(total, mean, rstd, dy, dx, gain=None, dtotal=None, dgain=None, dshift=None, work=None, stream=None) -> None:
    """dx, the gradient of x and of the residual, and dgain and dshift when given, from the forward call's total (x itself without a residual), mean and
    rstd."""
    lib = _load()
    call = _Call("tron_layer_norm_grad", total, stream)
    sp, m, d, lds = call.matrix(total, "total")
    dyp, _, _, lddy = call.matrix(dy, "dy", m, d, total.dtype)
    dtp, _, _, lddt = call.matrix(dtotal, "dtotal", m, d, total.dtype)
    dxp, _, _, lddx = call.matrix(dx, "dx", m, d, total.dtype)
    if mean is None or rstd is None:
        _refuse("tron_layer_norm_grad: mean and rstd are needed")
    space, wp, wb = call.work(work, lib.tron_layer_norm_grad_work(m, d) if dgain is not None or dshift is not None else 0)
    call.run(lib.tron_layer_norm_grad, m, d, call.type(total, "total"), sp, lds, call.vector(mean, "mean", m), call.vector(rstd, "rstd", m),
             call.vector(gain, "gain", d), dyp, lddy, dtp, lddt, dxp, lddx, call.vector(dgain, "dgain", d), call.vector(dshift, "dshift", d), wp, wb, call.address)


def tron_linear_work(m, n, k, dtype) -> int:
    lib = _load()
    return lib.tron_linear_work(m, n, k, _types.get(dtype, -1))


def tron_linear(x, w, y, bias=None, act=ACT_NONE, residual=None, pre=None, x_scale=None, w_scale=None, work=None, stream=None) -> None:
    """y = act(x w' + bias) + residual; the values before the activation go to `pre` when given.  x (m x k) and w (n x k) of one type:
    bfloat16, float16, or float8_e4m3fn or int8 with x_scale (m) and w_scale (n)."""
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


def _entries(call, t, what, shape, dtypes):
    """Address of a contiguous tensor of that shape and one of those types, or None."""
    if t is None:
        return None
    if t.get_device() != call.index:
        _refuse(f"{call.name}: {what} is on {t.device}, other arguments on {call.device}")
    if t.shape != shape or t.dtype not in dtypes or not t.is_contiguous():
        _refuse(f"{call.name}: {what} has to be {' x '.join(map(str, shape))} contiguous values of {' or '.join(map(str, dtypes))}")
    return t.data_ptr()


def tron_beam_select_work(batch, beams, V, picks) -> int:
    return load_library().tron_beam_select_work(batch, beams, V, picks)


def tron_beam_select(z, score, next_score, parent, token, ended=None, end=-1, next_ended=None, work=None, stream=None) -> None:
    """The step of a beam search: z (batch * beams x V) are the logits of beams with score (batch x beams); next_score, parent (rows of z) and token,
    batch x picks each, are the picks of largest log-probability.  ended and next_ended: bool or uint8.  next_score may be score, and next_ended ended, of as many picks
    as beams."""
    lib = _load()
    call = _Call("tron_beam_select", z, stream)
    zp, rows, V, ldz = call.matrix(z, "z")
    if score is None or next_score is None or score.dim() != 2 or next_score.dim() != 2 or score.shape[0] != next_score.shape[0]:
        _refuse("tron_beam_select: score (batch x beams) and next_score (batch x picks) have 2 dimensions")
    (batch, beams), picks = score.shape, next_score.shape[1]
    if rows != batch * beams:
        _refuse(f"tron_beam_select: z has {rows} rows, score {batch} x {beams}")
    space, wp, wb = call.work(work, lib.tron_beam_select_work(batch, beams, V, picks))
    call.run(lib.tron_beam_select, batch, beams, V, call.type(z, "z"), zp, ldz, _entries(call, score, "score", (batch, beams), _FLOAT),
             _entries(call, ended, "ended", (batch, beams), _FLAG), end, picks, _entries(call, next_score, "next_score", (batch, picks), _FLOAT),
             _entries(call, parent, "parent", (batch, picks), _INT), _entries(call, token, "token", (batch, picks), _INT),
             _entries(call, next_ended, "next_ended", (batch, picks), _FLAG), wp, wb, call.address)


def tron_beam_reorder(rows, states, out, lengths=None, stream=None) -> None:
    """out[:, i] = states[:, rows[i]] for states and out of layers x rows x positions x ..., whose positions lie one behind the other; rows: int32 of 1 or 2 dimensions
    (the parent of tron_beam_select, or its first columns).  lengths (int32, one a row of states): positions behind it are left as they were in out."""
    lib = _load()
    call = _Call("tron_beam_reorder", states, stream)
    if rows is None or rows.dtype != _torch.int32:
        _refuse("tron_beam_reorder: rows of int32 are needed")
    ip, batch, per, ldrows = call.matrix(rows, "rows")
    if out is None or states.dim() < 3 or out.dim() != states.dim() or out.dtype != states.dtype or out.shape[0] != states.shape[0] or out.shape[2:] != states.shape[2:]:
        _refuse("tron_beam_reorder: states and out have to be layers x rows x positions x ... of one type, alike but for the rows")
    if out.get_device() != call.index:
        _refuse(f"tron_beam_reorder: out is on {out.device}, other arguments on {call.device}")
    if out.shape[1] != batch * per:
        _refuse(f"tron_beam_reorder: out has {out.shape[1]} rows, expected {batch * per}")
    layers, rows_in, positions = states.shape[:3]
    size = step = states.element_size()
    for n in states.shape[3:]:
        step *= n
    if not (states.is_contiguous() and out.is_contiguous()):
        place = 1
        for i in range(states.dim() - 1, 1, -1):
            if states.shape[i] > 1 and not states.stride(i) == out.stride(i) == place:
                _refuse("tron_beam_reorder: the positions of a row of states or out are not contiguous")
            place *= max(1, states.shape[i])
    (src_layer, src_row), (dst_layer, dst_row) = states.stride()[:2], out.stride()[:2]
    call.run(lib.tron_beam_reorder, layers, batch, per, ip, ldrows, rows_in, states.data_ptr(), src_layer * size, src_row * size, out.data_ptr(),
             dst_layer * size, dst_row * size, positions, step, _entries(call, lengths, "lengths", (rows_in,), _INT), call.address)


def _ids(call, ids):
    """(address, count, bytes) of contiguous ids."""
    if ids is None or ids.get_device() != call.index:
        _refuse(f"{call.name}: ids are needed, on {call.device} as the other arguments")
    if ids.dtype not in (_torch.int32, _torch.int64) or ids.dim() != 1 or (ids.shape[0] > 1 and ids.stride(0) != 1):
        _refuse(f"{call.name}: ids have to be contiguous int32 or int64 values of one dimension")
    return ids.data_ptr(), ids.shape[0], 4 if ids.dtype == _torch.int32 else 8


def tron_embed(ids, table, y, scale=1.0, row_scale=None, stream=None) -> None:
    """y[i] = scale row_scale[ids[i]] table[ids[i]]; zeros where an id is not one of the table's rows.  table (V x d) of float32, bfloat16, float16, or float8_e4m3fn
    or int8 with row_scale (V); y of float32, bfloat16, float16."""
    lib = _load()
    call = _Call("tron_embed", table, stream)
    ip, m, ib = _ids(call, ids)
    if table.dim() != 2:
        _refuse("tron_embed: table has to have 2 dimensions")
    tp, V, d, ldt = call.matrix(table, "table")
    yp, _, _, ldy = call.matrix(y, "y", m, d)
    call.run(lib.tron_embed, m, d, V, ip, ib, call.type(table, "table"), tp, ldt, call.vector(row_scale, "row_scale", V), scale, call.type(y, "y"), yp, ldy, call.address)


def tron_embed_grad_work(m, d, V) -> int:
    return load_library().tron_embed_grad_work(m, d, V)


def tron_embed_grad(ids, dy, dtable, scale=1.0, add=False, work=None, stream=None) -> None:
    """dtable[v] = scale times the sum of the dy[i] with ids[i] = v, added to what is there with `add`.  dy (m x d) and dtable (V x d) of float32, bfloat16 or
    float16."""
    lib = _load()
    call = _Call("tron_embed_grad", dtable, stream)
    ip, m, ib = _ids(call, ids)
    if dtable.dim() != 2:
        _refuse("tron_embed_grad: dtable has to have 2 dimensions")
    tp, V, d, ldt = call.matrix(dtable, "dtable")
    dp, _, _, ldd = call.matrix(dy, "dy", m, d)
    space, wp, wb = call.work(work, lib.tron_embed_grad_work(m, d, V))
    call.run(lib.tron_embed_grad, m, d, V, ip, ib, call.type(dy, "dy"), dp, ldd, scale, int(add), call.type(dtable, "dtable"), tp, ldt, wp, wb, call.address)


# --------------------------------------------------------------------------- convenience wrapper
class SoftmaxHead:
    """The problem that a softmax head is trained on, with the calls of Dataset:

        f(W) = 1/2 W.W + C sum_i loss_i(z_i),   z = X W',   X = rms_norm(hidden + residual) gain

    or, with norm="layer", X = layer_norm(hidden + residual) gain + shift, for hidden states (m x d, bfloat16 or float16) and a teacher's ids and t (m x K).  W is n x d float32; the products take it rounded to
    the states' type.  fun_grad keeps the logits of its W for hv, as Dataset keeps D.

    hv is linear in its direction, whose size is the caller's (a gradient's, in the first product of a solve).  In float16 the products take it
    times a power of two, and the result by its reciprocal, so that neither the direction nor X V' leaves the type's range."""

    _LARGEST = 12   # log2 of a bound on |X V'|: four bits below float16's largest value, for weights and roundings

    def __init__(self, hidden, ids, t, gain=None, residual=None, eps=1e-6, temperature=1.0, weight=None, norm="rms", shift=None):
        _load()
        if norm not in ("rms", "layer") or (shift is not None and norm != "layer"):
            _refuse("SoftmaxHead: norm is 'rms' or 'layer', and the latter alone has a shift")
        self.m, self.d = hidden.shape
        self.ids, self.t, self.temperature, self.weight = ids, t, temperature, weight
        self.X = _torch.empty_like(hidden, memory_format=_torch.contiguous_format)
        if norm == "layer":
            tron_layer_norm(hidden, self.X, gain=gain, shift=shift, eps=eps, residual=residual)
        else:
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
