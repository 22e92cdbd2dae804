"""Python side of the operators beside the step (``include/qadam.h``, second part): AdamW over a list of tensors, the norm that clips
their gradients, embedding lookup and its gradient.  Argument checks and marshalling only, as in :mod:`.binding`: every call enqueues on
the given (default: current) stream and does not synchronise.  Buffers are written in place behind autograd's back: their version
counters stay, so a backward pass that saved a tensor before a call has changed it is not refused.
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import Optional, Sequence

from . import binding
from .binding import (QADAM_BF16, QADAM_CODES16, QADAM_CODES8, QADAM_F16, QADAM_F32, QADAM_OK, QADAM_STATE_BLOCK, QAdamError, _AdamWConfig,
                      _AdamWTensor, _Status, _address, _device_and_stream, _stream)


def _types():
    import torch
    return {torch.float32: QADAM_F32, torch.bfloat16: QADAM_BF16, torch.float16: QADAM_F16}


def _on_device(t, name):
    import torch
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s: expected a tensor, got %s" % (name, type(t).__name__))
    if not t.is_cuda:
        raise ValueError("%s: expected a device tensor" % name)
    if t.device.index != torch.cuda.current_device():
        raise ValueError("%s lives on %s, the current device is %d" % (name, t.device, torch.cuda.current_device()))


def _list_tensor(t, name, dtype, numel):
    """Address of a contiguous device tensor of this type and size."""
    _on_device(t, name)
    if not t.is_contiguous():
        raise ValueError("%s: expected a contiguous tensor" % name)
    if t.dtype != dtype:
        raise ValueError("%s: expected %s, got %s" % (name, dtype, t.dtype))
    if t.numel() != numel:
        raise ValueError("%s holds %d elements, expected %d" % (name, t.numel(), numel))
    return t.data_ptr()


def _rows(t, name, rows, dim):
    """Elements from one row to the next of a device tensor that stands for `rows` rows of `dim` elements: its last dimension is a
    row, the others are the rows in order, at one distance."""
    _on_device(t, name)
    if t.dim() < 2 or t.shape[-1] != dim or t.numel() != rows * dim:
        raise ValueError("%s: expected %d rows of %d elements, got shape %s" % (name, rows, dim, tuple(t.shape)))
    if rows == 0 or t.is_contiguous():
        return dim
    if dim > 1 and t.stride(-1) != 1:
        raise ValueError("%s: expected the elements of a row one behind the other" % name)
    step, length = None, 1
    for d in range(t.dim() - 2, -1, -1):
        if t.shape[d] == 1:
            continue
        if step is None:
            step = t.stride(d)
        elif t.stride(d) != step * length:
            raise ValueError("%s: expected all rows at one distance" % name)
        length *= t.shape[d]
    return dim if step is None else step


def _integer(value, name, bits=64):
    """`value` where the boundary takes an integer of so many bits: ctypes drops what lies above them."""
    if not -(1 << (bits - 1)) <= value < 1 << (bits - 1):
        raise ValueError("%s: %d does not fit %d bits" % (name, value, bits))
    return value


class _Handle:
    """Owner of one handle of the library."""
    _destroy = None

    def __init__(self):
        self._lib = binding.load_library()
        self._h = self._plan = None

    def _check(self, rc: int):
        if rc != QADAM_OK:
            raise QAdamError(rc, (self._lib.qadam_last_error() or b"").decode())

    def close(self):
        if self._h is not None:
            getattr(self._lib, self._destroy)(self._h)
            self._h = self._plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _TensorList(_Handle):
    """What AdamW and GradNorm share: a list of gradients of known types and sizes."""

    def _expect(self, numels, grad_dtypes, entry):
        types = _types()
        self._numels, self._grad_dtypes = numels, grad_dtypes
        self._table = C.c_void_p * max(1, len(numels))
        # as in the quantized step's binding: tensors of the common form are checked natively, any other call goes through the checks here
        self._plan = binding._native.list_plan(self._h.value, _address(entry), list(numels), [types[t] for t in grad_dtypes])

    def _grads(self, grads):
        if len(grads) != len(self._numels):
            raise ValueError("grads: expected %d tensors, got %d" % (len(self._numels), len(grads)))
        return self._table(*[None if g is None else _list_tensor(g, "grads[%d]" % i, self._grad_dtypes[i], self._numels[i])
                             for i, g in enumerate(grads)])


def _per_tensor(value, count, name):
    values = list(value) if isinstance(value, (list, tuple)) else [value] * count
    if len(values) != count:
        raise ValueError("%s: expected %d values, got %d" % (name, count, len(values)))
    return values


@dataclass
class AdamWConfig:
    beta1: float = 0.9
    beta2: float = 0.999
    eps: float = 1e-8
    state_bits: int = 32


def adamw_state(cfg: AdamWConfig, params: Sequence) -> dict:
    """Moments of a run that begins: the keyword arguments m, v (and m_scales, v_scales) of AdamW, all zero."""
    import torch
    dtype = torch.float32 if cfg.state_bits == 32 else torch.float8_e4m3fn
    state = {n: [torch.zeros(p.numel(), dtype=dtype, device=p.device) for p in params] for n in ("m", "v")}
    if cfg.state_bits == 8:
        for n in ("m_scales", "v_scales"):
            state[n] = [torch.zeros(-(-p.numel() // QADAM_STATE_BLOCK), dtype=torch.float32, device=p.device) for p in params]
    return state


class AdamW(_TensorList):
    """AdamW over a list of tensors (qadam_adamw_*): fp32, bfloat16 or float16 weights, moments in 32 or 8 bits.

    The handle steps the tensors that it is made with, in place: `params`, `m`, `v`, with 8-bit states (torch.float8_e4m3fn)
    `m_scales`, `v_scales`, and where given `copies`, the weights in another type (None for a tensor without one).  They must be
    contiguous and stay where they are.  `weight_decay` and `grad_dtype`: one for all, or one per tensor.  8-bit second moments do not
    follow gradients that shrink against others of their block of 256 (``include/qadam.h`` has figures).
    """
    _destroy = "qadam_adamw_destroy"

    def __init__(self, cfg: AdamWConfig, params: Sequence, m: Sequence, v: Sequence, m_scales: Optional[Sequence] = None,
                 v_scales: Optional[Sequence] = None, copies: Optional[Sequence] = None, weight_decay=0.0, grad_dtype=None):
        super().__init__()
        import torch
        types = _types()
        n = len(params)
        self.cfg = cfg
        state8 = cfg.state_bits == 8
        lists = dict(m=m, v=v, **(dict(m_scales=m_scales, v_scales=v_scales) if state8 else {}))
        for name, ts in lists.items():
            if ts is None or len(ts) != n:
                raise ValueError("%s: expected %d tensors" % (name, n))
        copies = _per_tensor(copies, n, "copies")
        decays = _per_tensor(weight_decay, n, "weight_decay")
        dtypes = _per_tensor(torch.float32 if grad_dtype is None else grad_dtype, n, "grad_dtype")
        self.kept = (list(params), {k: list(ts) for k, ts in lists.items()}, copies)    # the buffers live as long as the handle
        table = (_AdamWTensor * max(1, n))()
        for i, p in enumerate(params):
            r = table[i]
            _on_device(p, "params[%d]" % i)
            if p.dtype not in types or dtypes[i] not in types:
                raise ValueError("params[%d], grad_dtype: expected float32, bfloat16 or float16" % i)
            r.numel = p.numel()
            r.param, r.param_type, r.grad_type = _list_tensor(p, "params[%d]" % i, p.dtype, r.numel), types[p.dtype], types[dtypes[i]]
            for name, ts in lists.items():
                scales = name.endswith("scales")
                setattr(r, name, _list_tensor(ts[i], "%s[%d]" % (name, i), torch.float8_e4m3fn if state8 and not scales else torch.float32,
                                              -(-r.numel // QADAM_STATE_BLOCK) if scales else r.numel))
            if copies[i] is not None:
                _on_device(copies[i], "copies[%d]" % i)
                if copies[i].dtype not in types:
                    raise ValueError("copies[%d]: expected bfloat16 or float16" % i)
                r.copy, r.copy_type = _list_tensor(copies[i], "copies[%d]" % i, copies[i].dtype, r.numel), types[copies[i].dtype]
            r.weight_decay = decays[i]
        c = _AdamWConfig(C.sizeof(_AdamWConfig), _integer(cfg.state_bits, "state_bits", 32), cfg.beta1, cfg.beta2, cfg.eps)
        h = C.c_void_p()
        self._check(self._lib.qadam_adamw_init(C.byref(h), C.byref(c), table, n))
        self._h = h
        self._expect([p.numel() for p in params], dtypes, self._lib.qadam_adamw_step)

    def step(self, step: int, lr: float, grads: Sequence, grad_scale=None, stream=None):
        """One step with these gradients (None: that tensor rests).  `grad_scale`: one fp32 on the device that all gradients are
        multiplied with, such as GradNorm's out[1:]; where it is NaN or infinite nothing changes."""
        rc = binding._native.adamw_step(self._plan, *_device_and_stream(stream), step, lr, grads, grad_scale)
        if rc is not None:
            return self._check(rc)
        factor = None if grad_scale is None else _list_tensor(grad_scale, "grad_scale", _F32(), 1)
        self._check(self._lib.qadam_adamw_step(self._h, _integer(step, "step"), lr, self._grads(grads), factor, _stream(stream)))


def _F32():
    import torch
    return torch.float32


class GradNorm(_TensorList):
    """Norm of a list of gradients, and the factor that clips it (qadam_grad_norm_*).  `grad_dtype`: one for all, or one per tensor."""
    _destroy = "qadam_grad_norm_destroy"

    def __init__(self, numels: Sequence[int], grad_dtype=None):
        super().__init__()
        types = _types()
        numels = [_integer(int(n), "numels") for n in numels]
        dtypes = _per_tensor(_F32() if grad_dtype is None else grad_dtype, len(numels), "grad_dtype")
        for t in dtypes:
            if t not in types:
                raise ValueError("grad_dtype: expected float32, bfloat16 or float16")
        n = len(numels)
        h = C.c_void_p()
        self._check(self._lib.qadam_grad_norm_init(C.byref(h), (C.c_int64 * max(1, n))(*numels),
                                                   (C.c_int32 * max(1, n))(*[types[t] for t in dtypes]), n))
        self._h = h
        self._expect(numels, dtypes, self._lib.qadam_grad_norm)

    def grad_norm(self, grads: Sequence, max_norm: float, out, stream=None):
        """out[0] = norm, out[1] = max_norm / norm where the norm is beyond max_norm, else 1; NaN where the norm is not finite."""
        rc = binding._native.grad_norm(self._plan, *_device_and_stream(stream), grads, max_norm, out)
        if rc is not None:
            return self._check(rc)
        self._check(self._lib.qadam_grad_norm(self._h, self._grads(grads), max_norm, _list_tensor(out, "out", _F32(), 2), _stream(stream)))


def _padding(index):
    return -1 if index is None else _integer(index, "padding_idx")


class Embedding(_Handle):
    """A matrix of `rows` rows of `dim` elements, looked up by tokens, and its gradient (qadam_embedding_*).  `max_tokens`: the most
    tokens of one gradient."""
    _destroy = "qadam_embedding_destroy"

    def __init__(self, rows: int, dim: int, max_tokens: int):
        super().__init__()
        self.rows, self.dim, self.max_tokens = _integer(int(rows), "rows"), _integer(int(dim), "dim", 32), _integer(int(max_tokens), "max_tokens")
        h = C.c_void_p()
        self._check(self._lib.qadam_embedding_init(C.byref(h), self.rows, self.dim, self.max_tokens))
        self._h = h
        self._plan = binding._native.embedding_plan(h.value, self.rows, self.dim, _address(self._lib.qadam_embedding_lookup),
                                                    _address(self._lib.qadam_embedding_grad))

    def _tokens(self, tokens):
        import torch
        _on_device(tokens, "tokens")
        if tokens.dtype not in (torch.int32, torch.int64):
            raise ValueError("tokens: expected int32 or int64, got %s" % tokens.dtype)
        if not tokens.is_contiguous():
            raise ValueError("tokens: expected a contiguous tensor")
        return tokens.data_ptr(), tokens.element_size(), tokens.numel()

    def lookup(self, weight, tokens, out, scale: float = 1.0, k_x: Optional[int] = None, padding_idx: Optional[int] = None, stream=None):
        """out[t] = scale * weight[tokens[t]]; zeros for the padding and for tokens out of range (status bit QADAM_STATUS_TOKEN_RANGE).
        torch's embedding returns the row of its padding_idx: for that, give it to `grad` alone.
        `weight`: (rows, dim) in float32, bfloat16, float16, or weight codes in int8 or int16 with their `k_x`."""
        rc = binding._native.embedding_lookup(self._plan, *_device_and_stream(stream), weight, tokens, out, scale, k_x, padding_idx)
        if rc is not None:
            return self._check(rc)
        import torch
        types = _types()
        at, size, n = self._tokens(tokens)
        ws = _rows(weight, "weight", self.rows, self.dim)
        if k_x is not None:
            if weight.dtype not in (torch.int8, torch.int16):
                raise ValueError("weight: expected codes in int8 or int16, got %s" % weight.dtype)
            wt = QADAM_CODES8 if weight.dtype == torch.int8 else QADAM_CODES16
        elif weight.dtype not in types:
            raise ValueError("weight: expected float32, bfloat16, float16, or codes with k_x, got %s" % weight.dtype)
        else:
            wt = types[weight.dtype]
        os = _rows(out, "out", n, self.dim)
        if out.dtype not in types:
            raise ValueError("out: expected float32, bfloat16 or float16, got %s" % out.dtype)
        self._check(self._lib.qadam_embedding_lookup(
            self._h, weight.data_ptr(), wt, 0 if k_x is None else _integer(k_x, "k_x", 32), ws, at, size, n, _padding(padding_idx), scale,
            out.data_ptr(), types[out.dtype], os, _stream(stream)))

    def grad(self, tokens, dout, grad, scale: float = 1.0, padding_idx: Optional[int] = None, accumulate: bool = False, stream=None):
        """grad[r] = scale * sum of dout[t] over the t with tokens[t] = r, for every row; with `accumulate` added to what grad holds.
        `dout` may be an expanded row."""
        rc = binding._native.embedding_grad(self._plan, *_device_and_stream(stream), tokens, dout, grad, scale, padding_idx, accumulate)
        if rc is not None:
            return self._check(rc)
        types = _types()
        at, size, n = self._tokens(tokens)
        ds, gs = _rows(dout, "dout", n, self.dim), _rows(grad, "grad", self.rows, self.dim)
        if dout.dtype not in types or grad.dtype not in types:
            raise ValueError("dout, grad: expected float32, bfloat16 or float16")
        self._check(self._lib.qadam_embedding_grad(
            self._h, at, size, n, _padding(padding_idx), scale, dout.data_ptr(), types[dout.dtype], ds,
            grad.data_ptr(), types[grad.dtype], gs, int(bool(accumulate)), _stream(stream)))

    def get_status(self, clear=False, stream=None) -> int:
        st = _Status()
        self._check(self._lib.qadam_embedding_get_status(self._h, C.byref(st), int(clear), _stream(stream)))
        return int(st.flags)
