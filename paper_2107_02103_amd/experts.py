"""Convenience objects of the routing and 8-bit calls: they check arguments and
allocate outputs as torch tensors.  All arithmetic happens in libdpc.

No call is recorded for torch's autograd: the outputs of tensors that require a
gradient do not.  Gradients are calls of their own, named at each method.

A call with few rows is over in microseconds, so these methods check what they
are given once and call the library by address, without the checks of the
binding's functions of the same names."""
import operator

import torch

from . import binding as B

_lib, _elem_of, _MOST = B._lib, B.elem_of, B.INT_MAX
_raw_stream = torch._C._cuda_getCurrentRawStream   # hipStream_t of a device's current stream
_current_device = torch._C._cuda_getDevice


def _check(status, where):
    if status:
        raise B.DpcError(status, where)


def _too_large(where):
    """Refuses a call with a size that is no C int (ctypes would drop its high bits)."""
    raise B.DpcError(B.DPC_ENOTSUP, where)


def _rows(x, name, n=None, width=None, dtype=None, device=None):
    """Checks a tensor of rows (unit stride inside a row, rows apart by any
    stride that does not make them overlap); returns its row stride."""
    shape = x.shape
    if len(shape) != 2 or (n is not None and shape[0] != n) or (width is not None and shape[1] != width):
        raise ValueError(f"{name} has shape {tuple(shape)}, expected [{'rows' if n is None else n}, "
                         f"{'width' if width is None else width}]")
    if dtype is not None and x.dtype != dtype:
        raise TypeError(f"{name} has dtype {x.dtype}, expected {dtype}")
    _on(x, device, name)
    n, w = shape
    between, inside = x.stride()
    if (w > 1 and inside != 1) or (n > 1 and between < w):
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return between if n > 1 else w or 1


def _on(x, device, name):
    """Checks that a tensor is on a GPU (that of the others)."""
    at = x.get_device()
    if at < 0:
        raise ValueError(f"{name} must be a tensor on a GPU device, not {x.device}")
    if device is not None and at != device:
        raise ValueError(f"{name} is on {x.device}, the others are on cuda:{device}")


def _fixed(name):
    """An attribute that stays what the constructor has checked: sizes and addresses
    of later calls follow from it."""
    return property(operator.attrgetter("_" + name))


def _layer_bias(bias, shape, device):
    """Address of the bias of layers, which may be another than the constructor's."""
    if bias is None:
        return None
    if bias.dtype != torch.float32 or bias.shape != shape or not bias.is_contiguous():
        raise ValueError("bias must be contiguous float32 [experts, outer]")
    _on(bias, device, "bias")
    return bias.data_ptr()


def _enter(device, stream):
    """Context for a call on tensors of `device`: the stream it is to run on, or
    that device where another is current (the library launches on the current one)."""
    if stream is None:
        return torch.cuda.device(device)
    if stream.device.index != device:
        raise ValueError(f"stream is on {stream.device}, the tensors are on cuda:{device}")
    return torch.cuda.stream(stream)                   # makes the device current too


class Route:
    """Plan that sends each token's row to the experts it chooses and back.

    expert   int32 [tokens, topk] (or [tokens]): expert of each choice; a choice
             outside [0, nexpert) is dropped
    offsets  int32 [nexpert + 1]: first row of each expert; offsets[nexpert] rows
             are in use
    rows     int32 [tokens * topk]: slot token * topk + j of each row, -1 for the
             empty rows at the end
    pos      int32 [tokens, topk]: row of each choice, -1 if it is dropped

    The three may be written into; others in their place take another object.

    A call runs on the GPU of its tensors, whichever is current.
    stream: a torch stream of that GPU that the call runs on, and for which its
    outputs are allocated (default: the current one)."""

    offsets, rows, pos, ntok, topk, nexpert = (_fixed(name) for name in ("offsets", "rows", "pos", "ntok", "topk", "nexpert"))

    def __init__(self, expert, nexpert, stream=None):
        if expert.dtype != torch.int32 or expert.dim() not in (1, 2) or not expert.is_contiguous():
            raise ValueError("expert must be contiguous int32 [tokens, topk] or [tokens]")
        _on(expert, None, "expert")
        self._device = dev = expert.get_device()
        if stream is not None or _current_device() != dev:
            with _enter(dev, stream):
                return Route.__init__(self, expert, nexpert)
        self._ntok, self._topk = expert.shape if expert.dim() == 2 else (expert.shape[0], 1)
        self._nexpert = int(nexpert)
        m, head = self._ntok * self._topk, max(self._nexpert, 0) + 1
        if m > _MOST or abs(self._nexpert) > _MOST:
            _too_large("dpc_route_plan")
        nb = _lib.dpc_route_workspace_bytes(self._ntok, self._topk, self._nexpert)
        # the three of the plan in one allocation
        buf = expert.new_empty(head + 2 * m)
        ws = expert.new_empty((nb + 3) // 4)
        self._offsets, self._rows, pos = buf.split_with_sizes((head, m, m))
        self._pos = pos.view(self._ntok, self._topk)
        first = buf.data_ptr()
        _check(_lib.dpc_route_plan(_raw_stream(dev), self._ntok, self._topk, self._nexpert, expert.data_ptr(),
                                   ws.data_ptr(), nb, first, first + 4 * head, first + 4 * (head + m)), "dpc_route_plan")

    @classmethod
    def from_plan(cls, offsets, rows, pos):
        """A plan made before (the three tensors of another Route)."""
        r = cls.__new__(cls)
        if pos.dim() != 2 or rows.dim() != 1 or offsets.dim() != 1 or rows.shape[0] != pos.numel() or len(offsets) < 2:
            raise ValueError("offsets, rows and pos do not belong together")
        r._device = pos.get_device()
        for name, t in (("offsets", offsets), ("rows", rows), ("pos", pos)):
            if t.dtype != torch.int32 or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous int32 tensor")
            _on(t, r._device, name)
        r._offsets, r._rows, r._pos = offsets, rows, pos
        r._ntok, r._topk = pos.shape
        r._nexpert = len(offsets) - 1
        if r._ntok > _MOST or r._topk > _MOST or r._nexpert > _MOST:
            _too_large("dpc_route_plan")
        return r

    def _weight(self, weight, x):
        """Address of the weights of a call on rows x."""
        if weight is None:
            return None
        want = torch.float64 if x.dtype == torch.float64 else torch.float32
        if weight.dtype != want or weight.shape != self._pos.shape or not weight.is_contiguous():
            raise ValueError(f"weight must be contiguous {want} [tokens, topk]")
        _on(weight, self._device, "weight")
        return weight.data_ptr()

    def gather(self, x, weight=None, out=None, stream=None):
        """[tokens * topk, width]: each row the token's row (times its weight),
        zeros in the empty rows.  With weights, the gradient of combine()."""
        if stream is not None or _current_device() != self._device:
            with _enter(self._device, stream):
                return self.gather(x, weight, out)
        dev, m = self._device, self._ntok * self._topk
        ldx, width = _rows(x, "x", self._ntok, None, None, dev), x.shape[1]
        if width > _MOST:
            _too_large("dpc_route_gather")
        if out is None:
            out, ldy = x.new_empty((m, width)), width or 1
        else:
            ldy = _rows(out, "out", m, width, x.dtype, dev)
        _check(_lib.dpc_route_gather(_raw_stream(dev), _elem_of(x.dtype), self._ntok, self._topk, width, x.data_ptr(), ldx,
                                     self._weight(weight, x), self._rows.data_ptr(), self._pos.data_ptr(),
                                     out.data_ptr(), ldy), "dpc_route_gather")
        return out

    def combine(self, x, weight=None, out=None, stream=None):
        """[tokens, width]: the sum of each token's rows (times their weights);
        without weights, the gradient of gather()."""
        if stream is not None or _current_device() != self._device:
            with _enter(self._device, stream):
                return self.combine(x, weight, out)
        dev = self._device
        ldx, width = _rows(x, "rows", self._ntok * self._topk, None, None, dev), x.shape[1]
        if width > _MOST:
            _too_large("dpc_route_combine")
        if out is None:
            out, ldy = x.new_empty((self._ntok, width)), width or 1
        else:
            ldy = _rows(out, "out", self._ntok, width, x.dtype, dev)
        _check(_lib.dpc_route_combine(_raw_stream(dev), _elem_of(x.dtype), self._ntok, self._topk, width, x.data_ptr(), ldx,
                                      self._weight(weight, x), self._pos.data_ptr(), out.data_ptr(), ldy),
               "dpc_route_combine")
        return out

    def combine_backward(self, x, dy, weight=None, need_rows=True, stream=None):
        """Gradient of combine(x, weight) from dE/dy: (dE/dx, dE/dweight); the
        second is None without weights, the first with need_rows=False."""
        if stream is not None or _current_device() != self._device:
            with _enter(self._device, stream):
                return self.combine_backward(x, dy, weight, need_rows)
        dev, m = self._device, self._ntok * self._topk
        ldx, width = _rows(x, "rows", m, None, None, dev), x.shape[1]
        if width > _MOST:
            _too_large("dpc_route_combine_bwd")
        lddy = _rows(dy, "dy", self._ntok, width, x.dtype, dev)
        w = self._weight(weight, x)
        if weight is None and not need_rows:
            return None, None
        dx = x.new_empty((m, width)) if need_rows else None
        dw = None if weight is None else weight.new_empty(weight.shape)
        _check(_lib.dpc_route_combine_bwd(_raw_stream(dev), _elem_of(x.dtype), self._ntok, self._topk, width, x.data_ptr(),
                                          ldx, w, self._rows.data_ptr(), self._pos.data_ptr(), dy.data_ptr(), lddy,
                                          None if dx is None else dx.data_ptr(), width or 1,
                                          None if dw is None else dw.data_ptr()), "dpc_route_combine_bwd")
        return dx, dw


class Int8Linear:
    """A layer y = x W^T + b on 8-bit codes, or one layer for each expert.

    Each product is off by about 1% of its norm.  Whether that will do is up to
    what follows: where tanh is saturated (pre-activations far above 1) forces
    taken through these layers can be wrong altogether.  A layer of the codes of
    W^T approximates the gradient in x; it is not the derivative of y.

    codes   int8 [experts, outer, i8_ld(inner)] (or [outer, ...] for one layer)
    scales  float32 [experts, outer];  bias float32 [experts, outer] or None
    All may be written into, and another bias may take the place of the first."""

    codes, scales, inner, outer, experts = (_fixed(name) for name in ("codes", "scales", "inner", "outer", "experts"))

    def __init__(self, codes, scales, inner, bias=None):
        if codes.dim() == 2:
            codes, scales = codes[None], scales[None]
            bias = None if bias is None else bias[None]
        self._inner = int(inner)
        shape = codes.shape
        if len(shape) != 3 or codes.dtype != torch.int8 or shape[2] != B.i8_ld(self._inner) or not codes.is_contiguous():
            raise ValueError("codes must be contiguous int8 [experts, outer, i8_ld(inner)]")
        self._device = codes.get_device()
        _on(codes, None, "codes")
        self._experts, self._outer = shape[:2]
        if self._inner > _MOST or self._experts > _MOST or self._outer > _MOST:
            _too_large("dpc_linear_i8")
        if scales.dtype != torch.float32 or scales.shape != shape[:2] or not scales.is_contiguous():
            raise ValueError("scales must be contiguous float32 [experts, outer]")
        _on(scales, self._device, "scales")
        _layer_bias(bias, shape[:2], self._device)
        self._codes, self._scales, self.bias = codes, scales, bias

    @classmethod
    def from_weight(cls, weight, bias=None, stream=None):
        """Codes the rows (output channels) of weight [experts, outer, inner] or
        [outer, inner]; bias of any floating type."""
        w = weight[None] if weight.dim() == 2 else weight
        if w.dim() != 3:
            raise ValueError("weight must be [experts, outer, inner] or [outer, inner]")
        _on(w, None, "weight")
        if stream is not None or _current_device() != w.get_device():
            with _enter(w.get_device(), stream):
                return cls.from_weight(weight, bias)
        g, n, k = w.shape
        if g * n > _MOST or k > _MOST:
            _too_large("dpc_quant_rows")
        w = w.contiguous()
        codes = torch.empty((g, n, B.i8_ld(k)), dtype=torch.int8, device=w.device)
        scales = torch.empty((g, n), dtype=torch.float32, device=w.device)
        _check(_lib.dpc_quant_rows(_raw_stream(w.get_device()), _elem_of(w.dtype), g * n, k, w.data_ptr(), k,
                                   codes.data_ptr(), scales.data_ptr()), "dpc_quant_rows")
        if bias is not None:
            bias = bias.to(torch.float32).reshape(g, n).contiguous()
        return cls(codes, scales, k, bias)

    def __call__(self, x, route=None, offsets=None, dtype=None, out=None, stream=None):
        """y [tokens, outer] of x [tokens, inner].  With a route, x holds the
        tokens and y its rows (each from its expert's layer); with offsets
        (int32 [experts + 1]), the rows of x are sorted by expert already.
        dtype: type of y (default: that of x)."""
        if stream is not None or _current_device() != self._device:
            with _enter(self._device, stream):
                return self(x, route, offsets, dtype, out)
        dev = self._device
        ldx = _rows(x, "x", None if route is None else route.ntok, self._inner, None, dev)
        ntok, topk, rows = x.shape[0], 1, None
        if ntok > _MOST:
            _too_large("dpc_linear_i8")
        if route is not None:
            if offsets is not None:
                raise ValueError("give a route or offsets, not both")
            topk, rows, offsets = route.topk, route.rows.data_ptr(), route.offsets
        if offsets is not None:
            if offsets.dtype != torch.int32 or not offsets.is_contiguous():
                raise TypeError("offsets must be contiguous int32")
            if len(offsets) != self._experts + 1:
                raise ValueError(f"offsets for {len(offsets) - 1} experts, layers for {self._experts}")
            _on(offsets, dev, "offsets")
            offsets = offsets.data_ptr()
        elif self._experts != 1:
            raise ValueError("layers of several experts need a route or offsets")
        if dtype is None:
            dtype = x.dtype
        if out is None:
            out, ldy = torch.empty((ntok * topk, self._outer), dtype=dtype, device=x.device), self._outer
        else:
            ldy = _rows(out, "out", ntok * topk, self._outer, dtype, dev)
        nb = _lib.dpc_linear_i8_workspace_bytes(ntok, self._inner)
        ws = self._codes.new_empty(nb)
        _check(_lib.dpc_linear_i8(_raw_stream(dev), _elem_of(x.dtype), _elem_of(dtype), ntok, topk, self._outer,
                                  self._inner, self._experts, x.data_ptr(), ldx, rows, offsets, self._codes.data_ptr(),
                                  self._scales.data_ptr(), _layer_bias(self.bias, (self._experts, self._outer), dev),
                                  ws.data_ptr(), nb, out.data_ptr(), ldy), "dpc_linear_i8")
        return out
