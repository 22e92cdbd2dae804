"""Python side of what lies between the looked-up rows and the next token (``include/qadam.h``, third part): layer norm with its gradient,
the product of tokens with weight codes in 8-bit integers, and sampling.  Argument checks and marshalling only, as in :mod:`.operators`:
every call enqueues on the given (default: current) stream, writes the buffers that it is given and does not synchronise.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

from . import binding
from .binding import QADAM_CODES8, _address, _device_and_stream, _Filters, _Status, _stream
from .operators import _F32, _Handle, _integer, _list_tensor, _on_device, _rows, _types


def _count(t, name, dim):
    """Rows of `dim` elements that a tensor stands for."""
    _on_device(t, name)
    if t.dim() < 2 or t.shape[-1] != dim:
        raise ValueError("%s: expected rows of %d elements, got shape %s" % (name, dim, tuple(t.shape)))
    return t.numel() // dim


def _type(t, name):
    types = _types()
    if t.dtype not in types:
        raise ValueError("%s: expected float32, bfloat16 or float16, got %s" % (name, t.dtype))
    return types[t.dtype]


def _vector(t, name, numel, like=None):
    """(address, element type) of an optional vector of a float type, that of `like` where there is one."""
    if t is None:
        return None, 0 if like is None else like
    _on_device(t, name)
    kind = _type(t, name)
    if like is not None and kind != like:
        raise ValueError("%s: expected the other vector's type, got %s" % (name, t.dtype))
    return _list_tensor(t, name, t.dtype, numel), kind


def _pair(a, b, names, numel):
    """(address of a, address of b, their type); None for the one that is missing."""
    at, kind = _vector(a, names[0], numel)
    bt, kind = _vector(b, names[1], numel, None if a is None else kind)
    return at, bt, kind


def _floats(t, name, numel):
    return None if t is None else _list_tensor(t, name, _F32(), numel)


class LayerNorm(_Handle):
    """Layer norm over rows of `dim` elements, and its gradient (qadam_layer_norm*)."""
    _destroy = "qadam_layer_norm_destroy"

    def __init__(self, dim: int, eps: float = 1e-5):
        super().__init__()
        self.dim, self.eps = _integer(int(dim), "dim", 32), float(eps)
        h = C.c_void_p()
        self._check(self._lib.qadam_layer_norm_init(C.byref(h), self.dim, self.eps))
        self._h = h
        self._plan = binding._native.layer_plan(h.value, self.dim, 0, _address(self._lib.qadam_layer_norm),
                                                _address(self._lib.qadam_layer_norm_grad))

    def forward(self, x, weight, bias, out, mean=None, rstd=None, stream=None):
        """out = (x - mean) rstd weight + bias, rows in any shape (..., dim); weight and bias of one type, or None.  `mean` and `rstd`:
        fp32 of each row, written for the gradient.  `out` may be `x`."""
        rc = binding._native.layer_norm(self._plan, *_device_and_stream(stream), x, weight, bias, out, mean, rstd)
        if rc is not None:
            return self._check(rc)
        n = _count(x, "x", self.dim)
        xs, os = _rows(x, "x", n, self.dim), _rows(out, "out", n, self.dim)
        w, b, kind = _pair(weight, bias, ("weight", "bias"), self.dim)
        self._check(self._lib.qadam_layer_norm(self._h, n, x.data_ptr(), _type(x, "x"), xs, w, b, kind, out.data_ptr(), _type(out, "out"), os,
                                               _floats(mean, "mean", n), _floats(rstd, "rstd", n), _stream(stream)))

    def grad(self, dout, x, weight, mean, rstd, dx, dweight=None, dbias=None, accumulate: bool = False, stream=None):
        """dx, and the sums over rows dweight and dbias (of one type; with `accumulate` added to what they hold), from the forward call's x,
        mean and rstd.  `dx` may be `dout` or `x`; `dout` may be an expanded row."""
        rc = binding._native.layer_norm_grad(self._plan, *_device_and_stream(stream), dout, x, weight, mean, rstd, dx, dweight, dbias, accumulate)
        if rc is not None:
            return self._check(rc)
        n = _count(x, "x", self.dim)
        xs, ds, gs = _rows(x, "x", n, self.dim), _rows(dout, "dout", n, self.dim), _rows(dx, "dx", n, self.dim)
        w, kind = _vector(weight, "weight", self.dim)
        dw, db, grad_kind = _pair(dweight, dbias, ("dweight", "dbias"), self.dim)
        self._check(self._lib.qadam_layer_norm_grad(
            self._h, n, dout.data_ptr(), _type(dout, "dout"), ds, x.data_ptr(), _type(x, "x"), xs, w, kind,
            _list_tensor(mean, "mean", _F32(), n), _list_tensor(rstd, "rstd", _F32(), n), dx.data_ptr(), _type(dx, "dx"), gs, dw, db, grad_kind,
            int(bool(accumulate)), _stream(stream)))


def _int8(t, name):
    import torch
    if t.dtype != torch.int8:
        raise ValueError("%s: expected int8, got %s" % (name, t.dtype))


class Linear8(_Handle):
    """Product of tokens with a matrix of `outputs` rows of `inputs` 8-bit integers, such as the weight codes that the quantized step emits
    (qadam_linear8_*).  `max_tokens`: the most tokens of one call."""
    _destroy = "qadam_linear8_destroy"

    def __init__(self, outputs: int, inputs: int, max_tokens: int):
        super().__init__()
        self.outputs, self.inputs, self.max_tokens = _integer(int(outputs), "outputs"), _integer(int(inputs), "inputs", 32), _integer(int(max_tokens), "max_tokens")
        h = C.c_void_p()
        self._check(self._lib.qadam_linear8_init(C.byref(h), self.outputs, self.inputs, self.max_tokens))
        self._h = h
        self._plan = binding._native.layer_plan(h.value, self.inputs, self.outputs, _address(self._lib.qadam_linear8_forward),
                                                _address(self._lib.qadam_linear8_quantize))

    def quantize(self, x, codes, scales, stream=None):
        """Tokens as 8-bit integers (int8) with a scale each (fp32), for several products."""
        rc = binding._native.linear8_quantize(self._plan, *_device_and_stream(stream), x, codes, scales)
        if rc is not None:
            return self._check(rc)
        n = _count(x, "x", self.inputs)
        xs, cs = _rows(x, "x", n, self.inputs), _rows(codes, "codes", n, self.inputs)
        _int8(codes, "codes")
        self._check(self._lib.qadam_linear8_quantize(self._h, n, x.data_ptr(), _type(x, "x"), xs, codes.data_ptr(), cs,
                                                     _list_tensor(scales, "scales", _F32(), n), _stream(stream)))

    def forward(self, x, weight, out, weight_scales=None, k_x: Optional[int] = None, x_scales=None, bias=None, stream=None):
        """out = x weight^T + bias.  `x`: floats, whose integers the call makes, or integers (int8) with their `x_scales`.  `weight`:
        (outputs, inputs) int8 with fp32 `weight_scales` of each output, or weight codes with their `k_x`."""
        rc = binding._native.linear8_forward(self._plan, *_device_and_stream(stream), x, weight, out, weight_scales, k_x, x_scales, bias)
        if rc is not None:
            return self._check(rc)
        n = _count(x, "x", self.inputs)
        xs, ws, os = _rows(x, "x", n, self.inputs), _rows(weight, "weight", self.outputs, self.inputs), _rows(out, "out", n, self.outputs)
        _int8(weight, "weight")
        if (weight_scales is None) == (k_x is None):
            raise ValueError("weight: expected weight_scales, or codes with k_x")
        if x_scales is None:
            kind = _type(x, "x")
        else:
            _int8(x, "x")
            kind = QADAM_CODES8
        b, bias_kind = _vector(bias, "bias", self.outputs)
        self._check(self._lib.qadam_linear8_forward(
            self._h, n, x.data_ptr(), kind, xs, _floats(x_scales, "x_scales", n), weight.data_ptr(), ws,
            _floats(weight_scales, "weight_scales", self.outputs), 0 if k_x is None else _integer(k_x, "k_x", 32), b, bias_kind, out.data_ptr(),
            _type(out, "out"), os, _stream(stream)))


class Sampler(_Handle):
    """One token per row of `vocab` logits, by given random numbers (qadam_sampler_*).  `max_rows`: the most rows of one call."""
    _destroy = "qadam_sampler_destroy"

    def __init__(self, vocab: int, max_rows: int):
        super().__init__()
        self.vocab, self.max_rows = _integer(int(vocab), "vocab"), _integer(int(max_rows), "max_rows")
        h = C.c_void_p()
        self._check(self._lib.qadam_sampler_init(C.byref(h), self.vocab, self.max_rows))
        self._h = h
        self._plan = binding._native.layer_plan(h.value, self.vocab, 0, _address(self._lib.qadam_sampler_sample), 0)

    def sample(self, logits, u, out, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, stream=None):
        """out[r] = the token of row r: the filters of ``include/qadam.h`` in their order, then the token that u[r] (fp32 in [0, 1)) falls
        on in the descending order of the logits.  -1 for a row without a token (status bit QADAM_STATUS_NO_TOKEN).  Filters: a number
        for all rows, or a tensor of one per row (fp32, top_k int32).  `out`: int32 or int64."""
        rc = binding._native.sample(self._plan, *_device_and_stream(stream), logits, u, out, temperature, top_k, top_p, min_p)
        if rc is not None:
            return self._check(rc)
        import torch
        n = _count(logits, "logits", self.vocab)
        ls, kind = _rows(logits, "logits", n, self.vocab), _type(logits, "logits")
        _on_device(out, "out")
        if out.dtype not in (torch.int32, torch.int64):
            raise ValueError("out: expected int32 or int64, got %s" % out.dtype)
        f = _Filters()
        for name, value, dtype in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                                   ("min_p", min_p, torch.float32)):
            if isinstance(value, torch.Tensor):
                setattr(f, name + "s", _list_tensor(value, name, dtype, n))
            else:
                setattr(f, name, _integer(value, name, 32) if name == "top_k" else float(value))
        self._check(self._lib.qadam_sampler_sample(self._h, n, logits.data_ptr(), kind, ls, _list_tensor(u, "u", _F32(), n), C.byref(f),
                                                   _list_tensor(out, "out", out.dtype, n), out.element_size(), _stream(stream)))

    def get_status(self, clear=False, stream=None) -> int:
        st = _Status()
        self._check(self._lib.qadam_sampler_get_status(self._h, C.byref(st), int(clear), _stream(stream)))
        return int(st.flags)
