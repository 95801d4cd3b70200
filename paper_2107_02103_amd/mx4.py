"""Convenience objects of the calls in microscaled 4-bit floating point, beside
Int8Linear: they check arguments and allocate outputs; all arithmetic happens in
libdpc.  No call is recorded for torch's autograd."""
import torch

from . import binding as B
from .experts import (_MOST, _check, _current_device, _elem_of, _enter, _fixed, _layer_bias, _lib, _on, _raw_stream, _rows,
                      _too_large)


_U8 = torch.uint8


def _bytes(t, shape, name, device):
    if t.dtype != _U8 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous uint8 {list(shape)}")
    _on(t, device, name)


def _quantise(x, ldx, groups, n, dev, head=()):
    """Codes and scales (of shapes that `head` goes before) of rows x, `groups` matrices of n rows."""
    cols = x.shape[1]
    if groups * n > _MOST or cols > _MOST:
        _too_large("dpc_quant_mx4")
    ld = B.mx4_ld(cols)
    codes, scales = x.new_empty(head + (n, ld // 2), dtype=_U8), x.new_empty(head + (ld // 256, n, 8), dtype=_U8)
    _check(_lib.dpc_quant_mx4(_raw_stream(dev), _elem_of(x.dtype), groups, n, cols, x.data_ptr(), ldx, codes.data_ptr(),
                              scales.data_ptr()), "dpc_quant_mx4")
    return codes, scales


def _values(codes, scales, groups, n, cols, dtype, out, dev):
    """Rows that codes and scales of `groups` matrices of n rows stand for."""
    if out is None:
        out, ldy = codes.new_empty((groups * n, cols), dtype=dtype), cols
    else:
        ldy = _rows(out, "out", groups * n, cols, dtype, dev)
    _check(_lib.dpc_values_mx4(_raw_stream(dev), _elem_of(dtype), groups, n, cols, codes.data_ptr(), scales.data_ptr(),
                               out.data_ptr(), ldy), "dpc_values_mx4")
    return out


class Mx4Rows:
    """Rows in 4-bit floating-point codes with a power of two for every 32 columns.

    codes   uint8 [rows, mx4_ld(cols) / 2]: two columns in a byte
    scales  uint8 [mx4_ld(cols) / 256, rows, 8]: exponents, plus 127
    Both may be written into; others in their place take another object."""

    codes, scales, cols = _fixed("codes"), _fixed("scales"), _fixed("cols")

    def __init__(self, codes, scales, cols):
        self._cols = cols = int(cols)
        if cols < 1 or codes.dim() != 2:
            raise ValueError("codes must be contiguous uint8 [rows, mx4_ld(cols) / 2]")
        self._device, n, ld = codes.get_device(), codes.shape[0], B.mx4_ld(cols)
        if n > _MOST or cols > _MOST:
            _too_large("dpc_values_mx4")
        _bytes(codes, (n, ld // 2), "codes", None)
        _bytes(scales, (ld // 256, n, 8), "scales", self._device)
        self._codes, self._scales = codes, scales

    @classmethod
    def from_rows(cls, x, stream=None):
        """Codes the rows of x [rows, cols]."""
        ldx, dev = _rows(x, "x"), x.get_device()
        if stream is not None or _current_device() != dev:
            with _enter(dev, stream):
                return cls.from_rows(x)
        r = cls.__new__(cls)
        r._cols, r._device = x.shape[1], dev
        r._codes, r._scales = _quantise(x, ldx, 1, x.shape[0], dev)
        return r

    def values(self, dtype=torch.float32, out=None, stream=None):
        """[rows, cols]: what the codes stand for."""
        if stream is not None or _current_device() != self._device:
            with _enter(self._device, stream):
                return self.values(dtype, out)
        return _values(self.codes, self.scales, 1, self.codes.shape[0], self.cols, dtype, out, self._device)


class Mx4Linear:
    """A layer y = x W^T + b on 4-bit floating-point codes of x and W, or one layer
    for each expert: as Int8Linear, with half its bytes.

    Each product is off by 16 to 19% of its norm: for nets that were trained with
    these codes, and for searches.  A layer of the codes of W^T approximates the
    gradient in x; it is not the derivative of y.

    codes   uint8 [experts, outer, mx4_ld(inner) / 2] (or [outer, ...] for one)
    scales  uint8 [experts, mx4_ld(inner) / 256, outer, 8]
    bias    float32 [experts, outer] or None
    All may be written into, and another bias may take the place of the first."""

    codes, scales, inner, outer, experts = (_fixed(name) for name in ("codes", "scales", "inner", "outer", "experts"))

    def __init__(self, codes, scales, inner, bias=None):
        if codes.dim() == 2:
            codes, scales = codes[None], scales[None]
            bias = None if bias is None else bias[None]
        self._inner = inner = int(inner)
        if codes.dim() != 3 or inner < 1:
            raise ValueError("codes must be contiguous uint8 [experts, outer, mx4_ld(inner) / 2]")
        self._experts, self._outer = experts, outer = codes.shape[:2]
        if inner > _MOST or experts > _MOST or outer > _MOST:
            _too_large("dpc_linear_mx4")
        ld, self._device = B.mx4_ld(inner), codes.get_device()
        _bytes(codes, (experts, outer, ld // 2), "codes", None)
        _bytes(scales, (experts, ld // 256, outer, 8), "scales", self._device)
        _layer_bias(bias, (experts, outer), self._device)
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
        codes, scales = _quantise(w.contiguous().view(g * n, k), k, g, n, w.get_device(), (g,))
        if bias is not None:
            bias = bias.to(torch.float32).reshape(g, n).contiguous()
        return cls(codes, scales, k, bias)

    def weight(self, dtype=torch.float32, stream=None):
        """[experts, outer, inner]: the weights that the codes stand for."""
        if stream is not None or _current_device() != self._device:
            with _enter(self._device, stream):
                return self.weight(dtype)
        return _values(self._codes, self._scales, self._experts, self._outer, self._inner, dtype, None, self._device).view(
            self._experts, self._outer, self._inner)

    def __call__(self, x, route=None, offsets=None, dtype=None, out=None, stream=None):
        """y [tokens, outer] of x [tokens, inner], or of Mx4Rows (rows coded once for
        several layers).  With a route, x holds the tokens and y its rows (each from
        its expert's layer); with offsets (int32 [experts + 1]), the rows of x are
        sorted by expert already.  dtype: type of y (default: that of x; float32 for
        Mx4Rows)."""
        if stream is not None or _current_device() != self._device:
            with _enter(self._device, stream):
                return self(x, route, offsets, dtype, out)
        dev, coded = self._device, isinstance(x, Mx4Rows)
        ntok, topk, rows = x.codes.shape[0] if coded else x.shape[0], 1, None
        if coded:
            _on(x.codes, dev, "x")
            if x.cols != self._inner or (route is not None and ntok != route.ntok):
                raise ValueError(f"x has {ntok} rows of {x.cols} columns, expected "
                                 f"{'rows' if route is None else route.ntok} of {self._inner}")
        else:
            ldx = _rows(x, "x", None if route is None else route.ntok, self._inner, None, dev)
        if ntok > _MOST:
            _too_large("dpc_linear_mx4")
        if route is not None:
            if offsets is not None:
                raise ValueError("give a route or offsets, not both")
            _on(route.rows, dev, "route")
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
            dtype = torch.float32 if coded else x.dtype
        if out is None:
            out, ldy = self._codes.new_empty((ntok * topk, self._outer), dtype=dtype), self._outer
        else:
            ldy = _rows(out, "out", ntok * topk, self._outer, dtype, dev)
        tail = (rows, offsets, self._codes.data_ptr(), self._scales.data_ptr(),
                _layer_bias(self.bias, (self._experts, self._outer), dev))
        if coded:
            _check(_lib.dpc_matmul_mx4(_raw_stream(dev), _elem_of(dtype), ntok, topk, self._outer, self._inner, self._experts,
                                       x.codes.data_ptr(), x.scales.data_ptr(), *tail, out.data_ptr(), ldy), "dpc_matmul_mx4")
            return out
        nb = _lib.dpc_linear_mx4_workspace_bytes(ntok, self._inner)
        ws = self._codes.new_empty(nb)
        _check(_lib.dpc_linear_mx4(_raw_stream(dev), _elem_of(x.dtype), _elem_of(dtype), ntok, topk, self._outer, self._inner,
                                   self._experts, x.data_ptr(), ldx, *tail, ws.data_ptr(), nb, out.data_ptr(), ldy),
               "dpc_linear_mx4")
        return out
