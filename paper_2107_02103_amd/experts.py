"""Convenience objects of the routing and 8-bit calls: they check arguments and
allocate outputs as torch tensors.  All arithmetic happens in libdpc."""
import contextlib

import torch

from . import binding as B


_HERE = contextlib.nullcontext()


def _on(stream):
    """Outputs and workspaces are allocated for the stream that uses them."""
    return _HERE if stream is None else torch.cuda.stream(stream)


def _raw(stream, device):
    """hipStream_t of a torch stream, or of the device's current one."""
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _check(status, where):
    if status:
        raise B.DpcError(status, where)


def _elsewhere(t, device):
    raise ValueError(f"a tensor is on {t.device}, the others are on cuda:{device}")


def _matrix(x, name, rows=None, width=None, dtype=None):
    """Checks a tensor of rows (unit stride inside a row, rows apart by any
    stride that does not make them overlap); returns its row stride."""
    if x.dim() != 2 or (rows is not None and x.shape[0] != rows) or (width is not None and x.shape[1] != width):
        want = f"[{'rows' if rows is None else rows}, {'width' if width is None else width}]"
        raise ValueError(f"{name} has shape {tuple(x.shape)}, expected {want}")
    if dtype is not None and x.dtype != dtype:
        raise TypeError(f"{name} has dtype {x.dtype}, expected {dtype}")
    if not x.is_cuda:
        raise ValueError(f"{name} must be a tensor on a GPU device, not {x.device}")
    n, w = x.shape
    if (w > 1 and x.stride(1) != 1) or (n > 1 and x.stride(0) < w):
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return x.stride(0) if n > 1 else max(w, 1)


def _out(out, rows, width, like, name):
    if out is None:
        return torch.empty((rows, width), dtype=like.dtype, device=like.device)
    _matrix(out, name, rows, width, like.dtype)
    return out


class Route:
    """Plan that sends each token's row to the experts it chooses and back.

    expert   int32 [tokens, topk] (or [tokens]): expert of each choice; a choice
             outside [0, nexpert) is dropped
    offsets  int32 [nexpert + 1]: first row of each expert; offsets[nexpert] rows
             are in use
    rows     int32 [tokens * topk]: slot token * topk + j of each row, -1 for the
             empty rows at the end
    pos      int32 [tokens, topk]: row of each choice, -1 if it is dropped"""

    def __init__(self, expert, nexpert, stream=None):
        if expert.dtype != torch.int32 or expert.dim() not in (1, 2) or not expert.is_contiguous():
            raise ValueError("expert must be contiguous int32 [tokens, topk] or [tokens]")
        if not expert.is_cuda:
            raise ValueError(f"expert must be a tensor on a GPU device, not {expert.device}")
        self.ntok, self.topk = expert.shape[0], 1 if expert.dim() == 1 else expert.shape[1]
        self.nexpert = int(nexpert)
        m, dev = self.ntok * self.topk, expert.device
        with _on(stream):
            nb = B.dpc_route_workspace_bytes(self.ntok, self.topk, self.nexpert)
            # offsets, rows and positions in one allocation
            buf = torch.empty(max(self.nexpert, 0) + 1 + 2 * m, dtype=torch.int32, device=dev)
            self.offsets, self.rows = buf[:self.nexpert + 1], buf[self.nexpert + 1:self.nexpert + 1 + m]
            self.pos = buf[self.nexpert + 1 + m:].view(self.ntok, self.topk)
            ws = torch.empty(nb, dtype=torch.uint8, device=dev)
            at = buf.data_ptr()
            _check(B._lib.dpc_route_plan(_raw(stream, dev.index), self.ntok, self.topk, self.nexpert,
                                         expert.data_ptr(), ws.data_ptr(), nb, at, at + 4 * (self.nexpert + 1),
                                         at + 4 * (self.nexpert + 1 + m)), "dpc_route_plan")

    @classmethod
    def from_plan(cls, offsets, rows, pos):
        """A plan made before (the three tensors of another Route)."""
        r = cls.__new__(cls)
        if pos.dim() != 2 or rows.dim() != 1 or offsets.dim() != 1 or rows.shape[0] != pos.numel() or len(offsets) < 2:
            raise ValueError("offsets, rows and pos do not belong together")
        for name, t in (("offsets", offsets), ("rows", rows), ("pos", pos)):
            if t.dtype != torch.int32 or not t.is_contiguous() or not t.is_cuda:
                raise ValueError(f"{name} must be a contiguous int32 tensor on a GPU device")
        r.offsets, r.rows, r.pos = offsets, rows, pos
        r.ntok, r.topk = pos.shape
        r.nexpert = len(offsets) - 1
        return r

    def _weight(self, weight, x):
        if weight is None:
            return None
        want = torch.float64 if x.dtype == torch.float64 else torch.float32
        if weight.dtype != want or weight.shape != self.pos.shape or not weight.is_contiguous():
            raise ValueError(f"weight must be contiguous {want} [tokens, topk]")
        return weight

    def _call(self, name, stream, x, width, *args):
        """args: tensors are passed by address"""
        dev = self.pos.get_device()
        args = [a if a is None or isinstance(a, int) else a.data_ptr() if a.get_device() == dev else
                _elsewhere(a, dev) for a in args]
        _check(getattr(B._lib, name)(_raw(stream, dev), B.elem_of(x.dtype), self.ntok, self.topk, width, *args), name)

    def gather(self, x, weight=None, out=None, stream=None):
        """[tokens * topk, width]: each row the token's row (times its weight),
        zeros in the empty rows.  With weights, the gradient of combine()."""
        ldx = _matrix(x, "x", self.ntok)
        m, width = self.ntok * self.topk, x.shape[1]
        with _on(stream):
            y = _out(out, m, width, x, "out")
            self._call("dpc_route_gather", stream, x, width, x, ldx, self._weight(weight, x), self.rows, self.pos, y,
                       y.stride(0) if m > 1 else max(width, 1))
        return y

    def combine(self, x, weight=None, out=None, stream=None):
        """[tokens, width]: the sum of each token's rows (times their weights);
        without weights, the gradient of gather()."""
        m = self.ntok * self.topk
        ldx = _matrix(x, "rows", m)
        width = x.shape[1]
        with _on(stream):
            y = _out(out, self.ntok, width, x, "out")
            self._call("dpc_route_combine", stream, x, width, x, ldx, self._weight(weight, x), self.pos, y,
                       y.stride(0) if self.ntok > 1 else max(width, 1))
        return y

    def combine_backward(self, x, dy, weight=None, need_rows=True, stream=None):
        """Gradient of combine(x, weight) from dE/dy: (dE/dx, dE/dweight); the
        second is None without weights, the first with need_rows=False."""
        m = self.ntok * self.topk
        ldx = _matrix(x, "rows", m)
        width = x.shape[1]
        lddy = _matrix(dy, "dy", self.ntok, width, x.dtype)
        w = self._weight(weight, x)
        if w is None and not need_rows:
            return None, None
        with _on(stream):
            dx = torch.empty((m, width), dtype=x.dtype, device=x.device) if need_rows else None
            dw = None if w is None else torch.empty_like(w, memory_format=torch.contiguous_format)
            self._call("dpc_route_combine_bwd", stream, x, width, x, ldx, w, self.rows, self.pos, dy, lddy, dx,
                       max(width, 1), dw)
        return dx, dw


class Int8Linear:
    """A layer y = x W^T + b on 8-bit codes, or one layer for each expert.

    codes   int8 [experts, outer, i8_ld(inner)] (or [outer, ...] for one layer)
    scales  float32 [experts, outer];  bias float32 [experts, outer] or None"""

    def __init__(self, codes, scales, inner, bias=None):
        if codes.dim() == 2:
            codes, scales = codes[None], scales[None]
            bias = None if bias is None else bias[None]
        self.inner = int(inner)
        if codes.dim() != 3 or codes.dtype != torch.int8 or codes.shape[2] != B.i8_ld(self.inner):
            raise ValueError("codes must be int8 [experts, outer, i8_ld(inner)]")
        self.experts, self.outer = codes.shape[:2]
        for name, t in (("scales", scales), ("bias", bias)):
            if t is not None and (t.dtype != torch.float32 or t.shape != codes.shape[:2] or not t.is_contiguous()):
                raise ValueError(f"{name} must be contiguous float32 [experts, outer]")
        if not codes.is_contiguous() or not codes.is_cuda:
            raise ValueError("codes must be a contiguous tensor on a GPU device")
        self.codes, self.scales, self.bias = codes, scales, bias

    @classmethod
    def from_weight(cls, weight, bias=None, stream=None):
        """Codes the rows (output channels) of weight [experts, outer, inner] or
        [outer, inner]; bias of any floating type."""
        w = weight[None] if weight.dim() == 2 else weight
        if w.dim() != 3:
            raise ValueError("weight must be [experts, outer, inner] or [outer, inner]")
        g, n, k = w.shape
        with _on(stream):
            w = w.contiguous().view(g * n, k)
            codes = torch.empty((g, n, B.i8_ld(k)), dtype=torch.int8, device=w.device)
            scales = torch.empty((g, n), dtype=torch.float32, device=w.device)
            B.dpc_quant_rows(stream or torch.cuda.current_stream(w.device), B.elem_of(w.dtype), g * n, k, w, k,
                             codes, scales)
            if bias is not None:
                bias = bias.to(torch.float32).reshape(g, n).contiguous()
        return cls(codes, scales, k, bias)

    def __call__(self, x, route=None, offsets=None, dtype=None, out=None, stream=None):
        """y [tokens, outer] of x [tokens, inner].  With a route, x holds the
        tokens and y its rows (each from its expert's layer); with offsets
        (int32 [experts + 1]), the rows of x are sorted by expert already.
        dtype: type of y (default: that of x)."""
        ldx = _matrix(x, "x", None if route is None else route.ntok, self.inner)
        ntok, topk, rows = x.shape[0], 1, None
        if route is not None:
            if offsets is not None:
                raise ValueError("give a route or offsets, not both")
            topk, rows, offsets = route.topk, route.rows, route.offsets
        if offsets is not None and (offsets.dtype != torch.int32 or not offsets.is_contiguous()):
            raise TypeError("offsets must be contiguous int32")
        if offsets is not None and len(offsets) != self.experts + 1:
            raise ValueError(f"offsets for {len(offsets) - 1} experts, layers for {self.experts}")
        if offsets is None and self.experts != 1:
            raise ValueError("layers of several experts need a route or offsets")
        dtype = x.dtype if dtype is None else dtype
        with _on(stream):
            y = torch.empty((ntok * topk, self.outer), dtype=dtype, device=x.device) if out is None else out
            ldy = _matrix(y, "out", ntok * topk, self.outer, dtype)
            nb = B.dpc_linear_i8_workspace_bytes(ntok, self.inner)
            ws = torch.empty(nb, dtype=torch.uint8, device=x.device)
            dev = x.get_device()
            args = [a if a is None else a.data_ptr() if a.get_device() == dev else _elsewhere(a, dev)
                    for a in (rows, offsets, self.codes, self.scales, self.bias, y)]
            _check(B._lib.dpc_linear_i8(_raw(stream, dev), B.elem_of(x.dtype), B.elem_of(dtype), ntok, topk,
                                        self.outer, self.inner, self.experts, x.data_ptr(), ldx, *args[:5],
                                        ws.data_ptr(), nb, args[5], ldy), "dpc_linear_i8")
        return y
