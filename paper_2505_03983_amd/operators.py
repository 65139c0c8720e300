"""The operators of a gated residual network (include/asd.h) on torch tensors: shapes, types and devices are checked here,
outputs and workspaces are allocated by torch, the kernels run on the tensors' device and its current stream.  With `stream` (a
torch stream of that device) a call is made as under `torch.cuda.stream(stream)`: new outputs are that stream's, and the inputs have
to be ready for it.  Matrices may have any row pitch; their columns lie next to each other.  Results carry no autograd history: the
gradients are the *_backward calls, and an argument that requires a gradient is refused where torch would record one (call under
torch.no_grad(), or from the forward of a torch.autograd.Function, whose backward makes the *_backward call).  There is no fallback:
without a GPU a call raises."""
import torch

from . import binding

_TYPE = {torch.float32: binding.ASD_F32, torch.bfloat16: binding.ASD_BF16, torch.float16: binding.ASD_F16,
         torch.int8: binding.ASD_I8}
_ACT = {"silu": binding.ASD_ACT_SILU, "gelu": binding.ASD_ACT_GELU}
_LARGEST = 2 ** 31 - 1   # (sizes are 32-bit integers in the library, and ctypes drops what is above)
_entries = {}


def _entry(name):
    f = _entries.get(name)
    if f is None:
        f = _entries[name] = getattr(binding.lib(), name)
    return f


def _refuse(message):
    raise binding.AsdError(binding.ASD_EINVAL, message)


def _matrix(t, name, dtype, device, rows, cols):
    """Address and row pitch of a matrix argument."""
    if t.shape != (rows, cols):
        _refuse("%s has shape %s, not %s" % (name, tuple(t.shape), (rows, cols)))
    if t.dtype is not dtype:
        _refuse("%s is %s, not %s" % (name, t.dtype, dtype))
    if t.device != device:
        _refuse("%s is on %s, not on %s" % (name, t.device, device))
    if t.requires_grad and torch.is_grad_enabled():
        _refuse("%s requires a gradient, and results carry no autograd history" % name)
    if t.is_contiguous():
        return t.data_ptr(), cols
    row, col = t.stride()
    if col != 1 and cols > 1:
        _refuse("the columns of %s do not lie next to each other" % name)
    if rows <= 1:
        row = cols
    elif row < cols:
        _refuse("the rows of %s overlap" % name)
    return t.data_ptr(), row


def _vector(t, name, dtype, device, n):
    if t is None:
        return None
    if t.shape != (n,):
        _refuse("%s has shape %s, not (%d,)" % (name, tuple(t.shape), n))
    if t.dtype is not dtype:
        _refuse("%s is %s, not %s" % (name, t.dtype, dtype))
    if t.device != device:
        _refuse("%s is on %s, not on %s" % (name, t.device, device))
    if t.requires_grad and torch.is_grad_enabled():
        _refuse("%s requires a gradient, and results carry no autograd history" % name)
    if not t.is_contiguous():
        _refuse("the elements of %s do not lie next to each other" % name)
    return t.data_ptr()


def _out(t, name, dtype, device, rows, cols, like=None):
    """An output matrix, a new one if none is given (like: a matrix of its shape; quicker): the tensor, its address and row
    pitch."""
    if t is None:
        if like is not None and like.is_contiguous():
            t = torch.empty_like(like, dtype=dtype)
        else:
            t = torch.empty((rows, cols), dtype=dtype, device=device)
        return t, t.data_ptr(), cols
    return (t, *_matrix(t, name, dtype, device, rows, cols))


def _out_vector(t, name, dtype, device, n):
    if t is None:
        t = torch.empty(n, dtype=dtype, device=device)
        return t, t.data_ptr()
    return t, _vector(t, name, dtype, device, n)


def _rows_of(x, name="x"):
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        _refuse("%s is no matrix" % name)
    rows, cols = x.shape
    if rows > _LARGEST or cols > _LARGEST:
        raise binding.AsdError(binding.ASD_EUNSUPPORTED, "%s has shape %s: up to %d rows and columns" % (name, tuple(x.shape), _LARGEST))
    if x.device.type != "cuda":
        _refuse("%s is on %s, not on a GPU" % (name, x.device))
    return rows, cols


def _on(stream, device):
    """The context of a call with a stream of its own."""
    if not isinstance(stream, torch.cuda.Stream) or stream.device != device:
        _refuse("the stream is no torch stream of %s" % device)
    return torch.cuda.stream(stream)


def _launch(name, args, device, workspace=True):
    """Runs an entry on the tensors' device; its workspace is torch's, which hands memory on in the order of the stream."""
    if torch.cuda.current_device() != device.index:
        with torch.cuda.device(device):
            return _launch(name, args, device, workspace)
    ws = None
    if workspace:
        need = _entry(name + "_workspace")(args)
        if need:
            ws = torch.empty(need, dtype=torch.uint8, device=device)
            args.workspace, args.workspace_bytes = ws.data_ptr(), need
    # (the raw handle: the stream object that torch.cuda.current_stream makes takes longer than a launch)
    s = _entry(name)(args, torch._C._cuda_getCurrentRawStream(device.index))
    if s != binding.ASD_OK:
        raise binding.AsdError(s, binding.last_error())


def rms_norm(x, gain=None, eps=1e-6, residual=None, out_type=None, out=None, scale=None, sum_out=None, rows_used=None,
             stream=None):
    """(out, scale, sum): the rows of x (+ residual) over their root mean square, times gain.  out_type torch.int8: 8-bit
    integers, and their scales; a number type (default x's): scale is None.  sum is x + residual as the next layer's residual
    stream (None without a residual, unless sum_out is given; sum_out may be x or residual)."""
    if stream is not None:
        with _on(stream, x.device):
            return rms_norm(x, gain, eps, residual, out_type, out, scale, sum_out, rows_used)
    rows, cols = _rows_of(x)
    dev, t = x.device, x.dtype
    out_type = out_type or t
    if t not in _TYPE or out_type not in _TYPE:
        _refuse("no such type: %s -> %s" % (t, out_type))
    a = binding.asd_norm(rows=rows, cols=cols, type=_TYPE[t], out_type=_TYPE[out_type], eps=eps)
    a.x, a.ld_x = _matrix(x, "x", t, dev, rows, cols)
    out, a.out, a.ld_out = _out(out, "out", out_type, dev, rows, cols, x)
    a.gain = _vector(gain, "gain", t, dev, cols)
    if residual is not None:
        a.residual, a.ld_residual = _matrix(residual, "residual", t, dev, rows, cols)
        if sum_out is None:
            sum_out, a.sum, a.ld_sum = _out(None, "sum_out", t, dev, rows, cols, x)
    if sum_out is not None and not a.sum:
        a.sum, a.ld_sum = _matrix(sum_out, "sum_out", t, dev, rows, cols)
    if out_type == torch.int8:
        scale, a.scale = _out_vector(scale, "scale", torch.float32, dev, rows)
    else:
        scale = None
    a.rows_used = _vector(rows_used, "rows_used", torch.int32, dev, 1)
    _launch("asd_rms_norm", a, dev, workspace=False)
    return out, scale, sum_out


def quantize_rows(x, out=None, scale=None, rows_used=None, stream=None):
    """(out, scale): the rows of x as 8-bit integers, out * scale[:, None] being x to half a step."""
    if stream is not None:
        with _on(stream, x.device):
            return quantize_rows(x, out, scale, rows_used)
    rows, cols = _rows_of(x)
    dev, t = x.device, x.dtype
    if t not in _TYPE:
        _refuse("no such type: %s" % t)
    a = binding.asd_norm(rows=rows, cols=cols, type=_TYPE[t], out_type=binding.ASD_I8)
    a.x, a.ld_x = _matrix(x, "x", t, dev, rows, cols)
    out, a.out, a.ld_out = _out(out, "out", torch.int8, dev, rows, cols, x)
    scale, a.scale = _out_vector(scale, "scale", torch.float32, dev, rows)
    a.rows_used = _vector(rows_used, "rows_used", torch.int32, dev, 1)
    _launch("asd_quantize_rows", a, dev, workspace=False)
    return out, scale


def rms_norm_backward(dy, total, gain=None, eps=1e-6, dsum=None, dx=None, dgain=None, stream=None):
    """(dx, dgain) from the gradient dy of the norm's output and total, the sum the norm was taken of (x itself without a
    residual).  dsum: the gradient that reaches the sum from elsewhere.  dx is the gradient of x and of residual."""
    if stream is not None:
        with _on(stream, total.device):
            return rms_norm_backward(dy, total, gain, eps, dsum, dx, dgain)
    rows, cols = _rows_of(total, "total")
    dev, t = total.device, total.dtype
    if t not in _TYPE:
        _refuse("no such type: %s" % t)
    a = binding.asd_norm_grad(rows=rows, cols=cols, type=_TYPE[t], eps=eps)
    a.sum, a.ld_sum = _matrix(total, "total", t, dev, rows, cols)
    a.dy, a.ld_dy = _matrix(dy, "dy", t, dev, rows, cols)
    if dsum is not None:
        a.dsum, a.ld_dsum = _matrix(dsum, "dsum", t, dev, rows, cols)
    a.gain = _vector(gain, "gain", t, dev, cols)
    dx, a.dx, a.ld_dx = _out(dx, "dx", t, dev, rows, cols, total)
    dgain, a.dgain = _out_vector(dgain, "dgain", t, dev, cols)
    _launch("asd_rms_norm_backward", a, dev)
    return dx, dgain


def linear_i8(x, x_scale, w, w_scale, bias=None, out_type=torch.bfloat16, out=None, rows_used=None, stream=None):
    """x_scale[:, None] * (x @ w.T) * w_scale + bias for int8 x [rows, cols] and w [channels, cols]."""
    if stream is not None:
        with _on(stream, x.device):
            return linear_i8(x, x_scale, w, w_scale, bias, out_type, out, rows_used)
    rows, cols = _rows_of(x)
    dev = x.device
    channels = _rows_of(w, "w")[0]
    if out_type not in _TYPE:
        _refuse("no such type: %s" % out_type)
    a = binding.asd_linear8(rows=rows, cols=cols, channels=channels, out_type=_TYPE[out_type])
    a.x, a.ld_x = _matrix(x, "x", torch.int8, dev, rows, cols)
    a.w, a.ld_w = _matrix(w, "w", torch.int8, dev, channels, cols)
    a.x_scale = _vector(x_scale, "x_scale", torch.float32, dev, rows)
    a.w_scale = _vector(w_scale, "w_scale", torch.float32, dev, channels)
    a.bias = _vector(bias, "bias", torch.float32, dev, channels)
    out, a.out, a.ld_out = _out(out, "out", out_type, dev, rows, channels)
    a.rows_used = _vector(rows_used, "rows_used", torch.int32, dev, 1)
    _launch("asd_linear_i8", a, dev)
    return out


def _gated_args(x, w_gate, w_up, act, out_type):
    rows, cols = _rows_of(x)
    dev, t = x.device, x.dtype
    if t not in _TYPE or out_type not in _TYPE:
        _refuse("no such type: %s -> %s" % (t, out_type))
    if act not in _ACT:
        _refuse("unknown activation %r" % (act,))
    channels = _rows_of(w_gate, "w_gate")[0]
    a = binding.asd_gated(rows=rows, cols=cols, channels=channels, type=_TYPE[t], out_type=_TYPE[out_type], act=_ACT[act])
    a.x, a.ld_x = _matrix(x, "x", t, dev, rows, cols)
    a.w_gate, a.ld_w_gate = _matrix(w_gate, "w_gate", t, dev, channels, cols)
    a.w_up, a.ld_w_up = _matrix(w_up, "w_up", t, dev, channels, cols)
    return a


def gated_ff(x, w_gate, w_up, act="silu", x_scale=None, gate_scale=None, up_scale=None, out_type=None, out=None,
             rows_used=None, stream=None):
    """act(x @ w_gate.T) * (x @ w_up.T) for bfloat16 or float16 x [rows, cols] and weights [channels, cols], or for int8 ones
    with their scales (out_type then bfloat16, the default, or float16).  act: "silu" or "gelu" (its tanh form)."""
    if stream is not None:
        with _on(stream, x.device):
            return gated_ff(x, w_gate, w_up, act, x_scale, gate_scale, up_scale, out_type, out, rows_used)
    out_type = out_type or (torch.bfloat16 if x.dtype == torch.int8 else x.dtype)
    a = _gated_args(x, w_gate, w_up, act, out_type)
    dev = x.device
    if x.dtype == torch.int8:
        a.x_scale = _vector(x_scale, "x_scale", torch.float32, dev, a.rows)
        a.gate_scale = _vector(gate_scale, "gate_scale", torch.float32, dev, a.channels)
        a.up_scale = _vector(up_scale, "up_scale", torch.float32, dev, a.channels)
    out, a.out, a.ld_out = _out(out, "out", out_type, dev, a.rows, a.channels)
    a.rows_used = _vector(rows_used, "rows_used", torch.int32, dev, 1)
    _launch("asd_gated_ff", a, dev)
    return out


def gated_ff_backward(dh, x, w_gate, w_up, act="silu", need_dx=True, need_dw=True, dx=None, dw_gate=None, dw_up=None,
                      stream=None):
    """(dx, dw_gate, dw_up) from dh, the gradient of gated_ff's result; None for what is not needed."""
    if stream is not None:
        with _on(stream, x.device):
            return gated_ff_backward(dh, x, w_gate, w_up, act, need_dx, need_dw, dx, dw_gate, dw_up)
    a = _gated_args(x, w_gate, w_up, act, x.dtype)
    dev, t = x.device, x.dtype
    a.dh, a.ld_dh = _matrix(dh, "dh", t, dev, a.rows, a.channels)
    if need_dx:
        dx, a.dx, a.ld_dx = _out(dx, "dx", t, dev, a.rows, a.cols, x)
    else:
        dx = None
    if need_dw:
        dw_gate, a.dw_gate, a.ld_dw_gate = _out(dw_gate, "dw_gate", t, dev, a.channels, a.cols)
        dw_up, a.dw_up, a.ld_dw_up = _out(dw_up, "dw_up", t, dev, a.channels, a.cols)
    else:
        dw_gate = dw_up = None
    _launch("asd_gated_ff_backward", a, dev)
    return dx, dw_gate, dw_up
