"""The layers of include/rnngraph_layers.h on torch tensors: argument marshalling, device memory and streams.

Frames x streams tensors are [T][N][heads][units] with any strides but 1 between a head's units; row tensors are
[..., units], rows evenly spaced.  Calls are queued on the current stream of the tensors' device; what a call needs
as workspace comes from torch's allocator, for that call and stream alone.  There is no CPU path.  Nothing is recorded
for torch.autograd, the gradients are calls of their own: a tensor that requires gradients is refused where they are
recorded, as in torch's functions with out= (use torch.no_grad(), detach() or a torch.autograd.Function)."""
from __future__ import annotations

import ctypes as C

import torch

from .binding import AddNormDesc, DropoutDesc, Frames, LinearAttentionDesc, RnnError, _check, load_library

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
INVALID_ARGUMENT = -1


def _invalid(why):
    return RnnError(INVALID_ARGUMENT, why)


class _On:
    """The tensors' device made current, if it is not."""

    def __init__(self, device):
        self.index = device.index
        self.before = None

    def __enter__(self):
        now = torch.cuda.current_device()
        if now != self.index:
            self.before = now
            torch.cuda.set_device(self.index)
        return torch._C._cuda_getCurrentRawStream(self.index)      # (current_stream(index).cuda_stream, which takes 1 us more of a call's 10)

    def __exit__(self, *exc):
        if self.before is not None:
            torch.cuda.set_device(self.before)


def _device(device):
    if not torch.cuda.is_available():
        raise RuntimeError("rnngraph needs a GPU: there is no CPU path")
    device = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device() if device.index is None else device.index)


def _int32(**sizes):
    """ctypes cuts numbers off without a word."""
    for name, n in sizes.items():
        if not -(1 << 31) <= n < 1 << 31:
            raise _invalid(f"{name} = {n} does not fit 32 bits")


def _dtype(dtype, allowed=DTYPES):
    if dtype not in allowed:
        raise _invalid(f"dtype {dtype} is not one of {', '.join(str(d) for d in allowed)}")
    return DTYPES[dtype]


def _no_record(name, x):
    if x.requires_grad and torch.is_grad_enabled():
        raise _invalid(f"{name} requires gradients, which are not recorded here")


def _tensor(name, x, shape, dtype, device):
    if x.dtype is not dtype or x.shape != shape or x.device != device:
        raise _invalid(f"{name}: expected {dtype} {list(shape)} on {device}, got {x.dtype} {list(x.shape)} on {x.device}")
    _no_record(name, x)
    return x


def _flat(name, x, shape, dtype, device):
    """Address of a contiguous tensor, or None."""
    if x is None:
        return None
    if not _tensor(name, x, shape, dtype, device).is_contiguous():
        raise _invalid(f"{name} must be contiguous")
    return x.data_ptr()


def _workspace(nbytes, device):
    """(tensor that owns it, address); torch aligns its blocks to 512 bytes."""
    if nbytes == 0:
        return None, None
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr()


class LinearAttention:
    """S(t) = exp(log_decay[h]) S(t - 1) + k(t) v(t)^T,  o(t) = scale S(t)^T q(t), for windows of T frames and N streams."""

    def __init__(self, T, N, heads, dim_k, dim_v, kv_heads=None, dtype=torch.bfloat16, scale=1.0, training=False, device="cuda:0"):
        kv_heads = heads if kv_heads is None else kv_heads
        _int32(T=T, N=N, heads=heads, kv_heads=kv_heads, dim_k=dim_k, dim_v=dim_v)
        self.lib = load_library()
        self.dev, self.dtype = _device(device), dtype
        self.desc = LinearAttentionDesc(T, N, heads, kv_heads, dim_k, dim_v, _dtype(dtype, (torch.float32, torch.bfloat16)), scale)
        self.ref = C.byref(self.desc)
        self.shapes = {"q": (T, N, heads, dim_k), "k": (T, N, kv_heads, dim_k), "v": (T, N, kv_heads, dim_v), "o": (T, N, heads, dim_v)}
        self.state_shape, self.N, self.heads = (N, heads, dim_k, dim_v), N, heads
        self.ws_bytes = [_check(self.lib.rnn_linear_attention_workspace_bytes(self.ref, 0)),
                         _check(self.lib.rnn_linear_attention_workspace_bytes(self.ref, 1)) if training else None]

    def _frames(self, name, x, like):
        if x is None:
            return None
        st, sn, sh, one = _tensor(name, x, self.shapes[like], self.dtype, self.dev).stride()
        if one != 1 and x.shape[3] > 1:
            raise _invalid(f"{name}: a head's units must lie next to each other")
        return Frames(x.data_ptr(), st, sn, sh)      # (ctypes passes its address)

    def _common(self, log_decay, lengths):
        return (_flat("log_decay", log_decay, (self.heads,), torch.float32, self.dev), _flat("lengths", lengths, (self.N,), torch.int32, self.dev))

    def _state(self, name, x):
        return _flat(name, x, self.state_shape, torch.float32, self.dev)

    def forward(self, q, k, v, log_decay, o=None, state=None, state_out=None, lengths=None):
        """Writes o and / or state_out (which may be state); returns o.  q may be None if o is."""
        with _On(self.dev) as stream:
            ws, ws_ptr = _workspace(self.ws_bytes[0], self.dev)
            a, n = self._common(log_decay, lengths)
            _check(self.lib.rnn_linear_attention_forward(
                self.ref, self._frames("q", q, "q"), self._frames("k", k, "k"), self._frames("v", v, "v"), a, n, self._state("state", state),
                self._state("state_out", state_out), self._frames("o", o, "o"), ws_ptr, self.ws_bytes[0], stream))
        return o

    def backward(self, q, k, v, log_decay, do, dq=None, dk=None, dv=None, state=None, dstate_out=None, dstate=None, lengths=None):
        """Writes the gradients that are given: dq, dk, dv, and dstate, the gradient of `state`."""
        if self.ws_bytes[1] is None:
            raise _invalid("the layer was made with training=False")
        with _On(self.dev) as stream:
            ws, ws_ptr = _workspace(self.ws_bytes[1], self.dev)
            a, n = self._common(log_decay, lengths)
            _check(self.lib.rnn_linear_attention_backward(
                self.ref, self._frames("q", q, "q"), self._frames("k", k, "k"), self._frames("v", v, "v"), a, n, self._state("state", state),
                self._frames("do", do, "o"), self._state("dstate_out", dstate_out), self._frames("dq", dq, "q"), self._frames("dk", dk, "k"),
                self._frames("dv", dv, "v"), self._state("dstate", dstate), ws_ptr, self.ws_bytes[1], stream))


def _rows(name, x, rows, dim, dtype, device):
    """(address, elements from a row to the next) of a tensor of `rows` evenly spaced rows; (None, 0) for None."""
    if x is None:
        return None, 0
    if x.dtype is not dtype or x.device != device or x.dim() < 1 or x.shape[-1] != dim or x.numel() != rows * dim:
        raise _invalid(f"{name}: expected {dtype}, {rows} rows of {dim} on {device}, got {x.dtype} {list(x.shape)} on {x.device}")
    _no_record(name, x)
    if x.is_contiguous():
        return x.data_ptr(), dim
    if dim > 1 and x.stride(-1) != 1:
        raise _invalid(f"{name}: a row's units must lie next to each other")
    ld, span = None, None
    for size, stride in zip(reversed(x.shape[:-1]), reversed(x.stride()[:-1])):
        if size == 1:
            continue
        if ld is None:
            ld, span = stride, size * stride
        elif stride != span:
            raise _invalid(f"{name}: its rows are not evenly spaced")
        else:
            span *= size
    return x.data_ptr(), dim if ld is None else ld


class AddNorm:
    """h = residual + dropout(x),  y = gain h / sqrt(mean(h^2) + eps), for `rows` rows of `dim` units."""

    def __init__(self, rows, dim, dtype=torch.bfloat16, eps=1e-6, dropout=0.0, seed=0, offset=0, d_offset=None, device="cuda:0"):
        _int32(dim=dim)
        self.lib = load_library()
        self.dev, self.dtype, self.rows, self.dim = _device(device), dtype, rows, dim
        self.d_offset = d_offset      # (kept: the descriptor has its address)
        self.desc = AddNormDesc(rows, dim, _dtype(dtype), eps, dropout, seed, offset, _flat("d_offset", d_offset, (1,), torch.int64, self.dev))
        self.ref = C.byref(self.desc)
        self.ws_bytes = _check(self.lib.rnn_add_norm_workspace_bytes(self.ref))

    def _rows(self, name, x, dtype=None):
        return _rows(name, x, self.rows, self.dim, dtype or self.dtype, self.dev)

    def _floats(self, name, x, shape):
        return _flat(name, x, shape, torch.float32, self.dev)

    def set_offset(self, offset):
        """The part of the generator's counter that tells calls apart (another one for every training step)."""
        self.desc.offset = offset

    def forward(self, x, y, residual=None, gain=None, h=None, rstd=None):
        with _On(self.dev) as stream:
            _check(self.lib.rnn_add_norm_forward(self.ref, *self._rows("x", x), *self._rows("residual", residual), self._floats("gain", gain, (self.dim,)),
                                                 *self._rows("h", h), *self._rows("y", y), self._floats("rstd", rstd, (self.rows,)), stream))
        return y

    def forward_e4m3(self, x, y, scales, residual=None, gain=None, h=None, rstd=None, group=128):
        """y: torch.float8_e4m3fn; scales: [rows][ceil(dim / 128)], or [rows][1] with group = 0."""
        _int32(group=group)
        blocks = -(-self.dim // 128) if group else 1
        with _On(self.dev) as stream:
            _check(self.lib.rnn_add_norm_e4m3(self.ref, *self._rows("x", x), *self._rows("residual", residual), self._floats("gain", gain, (self.dim,)),
                                              *self._rows("h", h), *self._rows("y", y, torch.float8_e4m3fn), self._floats("scales", scales, (self.rows, blocks)),
                                              group, self._floats("rstd", rstd, (self.rows,)), stream))
        return y

    def backward(self, dy, h, rstd, gain=None, dh=None, dx=None, dresidual=None, dgain=None):
        """h, rstd: as forward stored them; dh: gradient of h from elsewhere.  Writes those of dx, dresidual and dgain that are given."""
        with _On(self.dev) as stream:
            ws, ws_ptr = _workspace(self.ws_bytes if dgain is not None else 0, self.dev)
            _check(self.lib.rnn_add_norm_backward(
                self.ref, *self._rows("dy", dy), *self._rows("dh", dh), *self._rows("h", h), self._floats("rstd", rstd, (self.rows,)),
                self._floats("gain", gain, (self.dim,)), *self._rows("dx", dx), *self._rows("dresidual", dresidual), self._floats("dgain", dgain, (self.dim,)),
                ws_ptr, self.ws_bytes if ws_ptr else 0, stream))


def dropout(x, y, p, seed, offset=0, d_offset=None):
    """y = x / (1 - p) where the generator keeps an element, else 0; the same call on dy is the gradient.  y may be x."""
    dim = x.shape[-1] if x.dim() else 1
    _int32(dim=dim)
    lib = load_library()
    rows = x.numel() // dim if dim else 0
    px, ld_x = _rows("x", x, rows, dim, x.dtype, _device(x.device))
    py, ld_y = _rows("y", y, rows, dim, x.dtype, x.device)
    desc = DropoutDesc(rows, dim, _dtype(x.dtype), p, seed, offset, _flat("d_offset", d_offset, (1,), torch.int64, x.device))
    with _On(x.device) as stream:
        _check(lib.rnn_dropout(C.byref(desc), px, ld_x, py, ld_y, stream))
    return y
