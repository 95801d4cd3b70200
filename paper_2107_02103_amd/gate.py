"""Convenience objects of the calls before a routing: the choice of experts and
vectors of ids.  As Route's, their methods check arguments and allocate outputs;
all arithmetic happens in libdpc, and no call is recorded for torch's autograd:
gradients are methods of their own."""
import torch

from . import binding as B
from .experts import (_MOST, _check, _current_device, _elem_of, _enter, _lib, _on, _raw_stream, _rows, _too_large)

_Spec = B.dpc_gate_spec
_SCORES = {"softmax": B.DPC_SCORE_SOFTMAX, "sigmoid": B.DPC_SCORE_SIGMOID}


class Gate:
    """Which experts a token goes to, and with which weights, from its scores.

    nexpert, topk  experts, and how many of them a token is sent to
    score          "softmax" or "sigmoid" of the logits
    bias           float32 [nexpert] or None: added to the scores for the choice
                   alone, as what balances the experts' loads; another one may
                   take its place between calls
    groups, keep, best  the experts stand in `groups` groups of equal size, of
                   which a token keeps the `keep` with the largest sum of their
                   `best` (1 or 2) largest biased scores
    renormalise    the weights of a token are divided by their sum
    scale          factor of all weights

    An expert whose logit is -infinity is closed to the token; a token to which all
    are goes nowhere (padding atoms: scores of 0 are scores like any other)."""

    def __init__(self, nexpert, topk, score="softmax", groups=1, keep=1, best=1, bias=None, renormalise=False, scale=1.0):
        if score not in _SCORES:
            raise ValueError(f"score is softmax or sigmoid, not {score!r}")
        for v in (nexpert, topk, groups, keep, best):
            if not -_MOST <= v <= _MOST:
                _too_large("dpc_gate")
        self.spec = _Spec(int(nexpert), int(topk), _SCORES[score], int(groups), int(keep), int(best), bool(renormalise), scale)
        self.bias = bias
        self._bias(None)

    nexpert = property(lambda self: self.spec.nexpert)
    topk = property(lambda self: self.spec.topk)

    def _bias(self, dev):
        """Address of the bias, which may be another than the constructor's."""
        bias = self.bias
        if bias is None:
            return None
        if bias.dtype != torch.float32 or bias.shape != (self.spec.nexpert,) or not bias.is_contiguous():
            raise ValueError("bias must be contiguous float32 [nexpert]")
        _on(bias, dev, "bias")
        return bias.data_ptr()

    def _logits(self, logits, dev):
        ld = _rows(logits, "logits", None, self.spec.nexpert, None, dev)
        if logits.shape[0] > _MOST:
            _too_large("dpc_gate")
        return ld, torch.float64 if logits.dtype == torch.float64 else torch.float32

    def __call__(self, logits, stream=None):
        """Experts int32 [tokens, topk], the best first (-1: none left), and their
        weights [tokens, topk] (float64 for float64 logits, else float32): what
        Route and Route.combine take."""
        _on(logits, None, "logits")
        dev = logits.get_device()
        if stream is not None or _current_device() != dev:
            with _enter(dev, stream):
                return self(logits)
        ld, wt = self._logits(logits, None)
        bias, spec = self._bias(dev), self.spec
        n, elem = logits.shape[0], _elem_of(logits.dtype)
        shape = (n, max(spec.topk, 0))
        expert, weight = logits.new_empty(shape, dtype=torch.int32), logits.new_empty(shape, dtype=wt)
        _check(_lib.dpc_gate(_raw_stream(dev), elem, spec, n, logits.data_ptr(), ld, bias, expert.data_ptr(),
                             weight.data_ptr()), "dpc_gate")
        return expert, weight

    def backward(self, logits, expert, dweight, out=None, stream=None):
        """dE/dlogits from dE/dweight at the experts chosen (such as
        Route.combine_backward gives)."""
        _on(logits, None, "logits")
        dev = logits.get_device()
        if stream is not None or _current_device() != dev:
            with _enter(dev, stream):
                return self.backward(logits, expert, dweight, out)
        ld, wt = self._logits(logits, None)
        n, elem, spec = logits.shape[0], _elem_of(logits.dtype), self.spec
        for name, t, dt in (("expert", expert, torch.int32), ("dweight", dweight, wt)):
            if t.dtype != dt or t.shape != (n, spec.topk) or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous {dt} [tokens, topk]")
            _on(t, dev, name)
        if out is None:
            out, ldo = logits.new_empty((n, spec.nexpert)), spec.nexpert
        else:
            ldo = _rows(out, "out", n, spec.nexpert, logits.dtype, dev)
        _check(_lib.dpc_gate_bwd(_raw_stream(dev), elem, spec, n, logits.data_ptr(), ld, expert.data_ptr(),
                                 dweight.data_ptr(), out.data_ptr(), ldo), "dpc_gate_bwd")
        return out


def _ids(ids):
    if ids.dtype != torch.int32 or ids.dim() != 1 or not ids.is_contiguous():
        raise ValueError("ids must be contiguous int32 [tokens]")
    _on(ids, None, "ids")
    if ids.shape[0] > _MOST:
        _too_large("dpc_embed")
    return ids.get_device()


class Embedding:
    """A vector for each id (the species of an atom, a token), times a scale.

    table  [ids, width], rows of any stride; another one may take its place
    An id outside [0, ids) stands for nothing: its vector is zeros, and it has no
    part in the gradient."""

    def __init__(self, table, scale=1.0):
        self.table, self.scale = table, float(scale)
        self._read(table)

    def _read(self, table):
        """What a table is, its element type and the stride of its rows, checked."""
        ld, elem = _rows(table, "table"), _elem_of(table.dtype)
        if table.shape[0] > _MOST or table.shape[1] > _MOST:
            _too_large("dpc_embed")
        self._seen = seen = (table.shape, table.stride(), table.dtype, table.get_device()), elem, ld
        return seen

    @property
    def ids(self):
        return self.table.shape[0]

    @property
    def width(self):
        return self.table.shape[1]

    def __call__(self, ids, out=None, stream=None):
        """[tokens, width] of ids int32 [tokens]."""
        table, seen = self.table, self._seen
        dev = table.get_device()
        if (table.shape, table.stride(), table.dtype, dev) != seen[0]:  # another one, or changed as .data of a parameter is
            seen = self._read(table)
        if stream is not None or _current_device() != dev:
            with _enter(dev, stream):
                return self(ids, out)
        if _ids(ids) != dev:
            _on(ids, dev, "ids")
        (nid, width), (_, elem, ld), n = table.shape, seen, ids.shape[0]
        if out is None:
            out, ldy = table.new_empty((n, width)), width or 1
        else:
            ldy = _rows(out, "out", n, width, table.dtype, dev)
        _check(_lib.dpc_embed(_raw_stream(dev), elem, n, nid, width, ids.data_ptr(), table.data_ptr(), ld, self.scale,
                              out.data_ptr(), ldy), "dpc_embed")
        return out

    def backward(self, ids, dy, dtype=None, out=None, stream=None):
        """dE/dtable from dE/dy (see gradient)."""
        nid, width = self.table.shape
        if dy.dim() != 2 or dy.shape[1] != width:
            raise ValueError(f"dy has shape {tuple(dy.shape)}, expected [tokens, {width}]")
        _on(dy, self.table.get_device(), "dy")
        return Embedding.gradient(ids, dy, nid, self.scale, dtype, out, stream)

    @staticmethod
    def gradient(ids, dy, nid, scale=1.0, dtype=None, out=None, stream=None):
        """[nid, width]: scale times the sum of the rows of dy [tokens, width] of
        each id, in dy's type or (dtype=torch.float32) in float32."""
        dev = _ids(ids)
        if stream is not None or _current_device() != dev:
            with _enter(dev, stream):
                return Embedding.gradient(ids, dy, nid, scale, dtype, out)
        n, nid = ids.shape[0], int(nid)
        lddy, width = _rows(dy, "dy", n, None, None, dev), dy.shape[1]
        if abs(nid) > _MOST or width > _MOST:
            _too_large("dpc_embed_bwd")
        dtype = dy.dtype if dtype is None else dtype
        elem, elem_d = _elem_of(dy.dtype), _elem_of(dtype)
        if out is None:
            out, ldo = dy.new_empty((max(nid, 0), width), dtype=dtype), width or 1
        else:
            ldo = _rows(out, "out", nid, width, dtype, dev)
        nb = _lib.dpc_embed_bwd_workspace_bytes(elem, n, nid, width)
        ws = dy.new_empty(nb, dtype=torch.uint8)
        _check(_lib.dpc_embed_bwd(_raw_stream(dev), elem, elem_d, n, nid, width, ids.data_ptr(), dy.data_ptr(), lddy,
                                  float(scale), ws.data_ptr(), nb, out.data_ptr(), ldo), "dpc_embed_bwd")
        return out
