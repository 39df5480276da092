"""Routed products: a router's choice, the grouping by it, products with matrices in 4 bits, the weighted sum.

The torch front of the calls of ``include/vbr_spmm.h`` that start with ``route_`` and ``q4_`` (their comments there say what each
computes).  As in ``binding``, everything the C ABI cannot see of a tensor is checked here before anything is launched, work goes to torch's
current stream of the operands' device, and there is no fallback.

    ids, weights = route_topk(logits, k, score="sigmoid", bias=bias, n_groups=8, top_groups=4)
    up = Q4(codes, scales, zeros, group=128, gated=True).upload()      # [experts, 2 F, K / 2] codes
    down = Q4(codes2, scales2, zeros2, group=128).upload()             # [experts, K, F / 2]
    out = experts_forward(x, ids, weights, up, down)

or step by step: ``plan = route_plan(ids, n_experts)``, ``h = up.mm_routed(x, plan)``, ``y = down.mm_routed(h, plan)``,
``out = route_combine(y, ids, weights)``.

Autograd does not see any of it: where gradients are recorded, the calls forward refuse operands that require one instead of giving results that are
cut off from them.  ``route_topk_grad`` and ``route_combine_grad`` are the router's and the sum's gradients, to be called with gradients
off (inside a ``torch.autograd.Function``, for instance); matrices in 4 bits are frozen, and their products pass none on to ``x``.
"""
from __future__ import annotations

import ctypes
from functools import lru_cache

import torch

from .binding import VbrError, _Route, _current_device, _lib, _raw_stream

_TYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_SCORES = {"softmax": 0, "sigmoid": 1}


def _call(what, fn, device, *args):
    """The C call on torch's current stream of the device, which is made the current one if it is not."""
    if device < 0:
        raise ValueError("%s: operands must be on the GPU" % what)
    if _current_device() == device:
        rc = fn(*args, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _raw_stream(device))
    if rc != 0:
        raise VbrError(rc, what)


def _rows(what, name, t, n_rows, n_cols, types):
    """A 2-D operand whose rows do not overlap, of one of `types`; returns its row stride."""
    shape, stride = t.shape, t.stride()
    if t.dtype not in types or len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError("%s: %s must be a 2-D tensor of %s with unit column stride" % (what, name, " or ".join(str(x) for x in types)))
    if (n_rows is not None and shape[0] != n_rows) or (n_cols is not None and shape[1] != n_cols):
        raise ValueError("%s: %s must be of shape (%s, %s), not %s" % (what, name, n_rows, n_cols, tuple(shape)))
    if shape[0] <= 1:
        return max(stride[0], shape[1])
    if stride[0] < shape[1]:
        raise ValueError("%s: rows of %s must not overlap" % (what, name))
    return stride[0]


def _cut_off(what):
    if torch.is_grad_enabled():
        raise ValueError("%s: an operand requires a gradient, which autograd would not get through this call: detach it, or call under torch.no_grad()" % what)


def _dense(what, name, t, shape, dtype):
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s: %s must be a contiguous %s tensor of shape %s" % (what, name, dtype, tuple(shape)))


def _new(n_rows, n_cols, dtype, device):
    return torch.empty_strided((n_rows, n_cols), (n_cols, 1), dtype=dtype, device=device)      # (torch.empty takes 0.4 us longer)


def _together(what, device, *others):
    for t in others:
        if t is not None and t.get_device() != device:
            raise ValueError("%s: operands must be on one device" % what)


@lru_cache(maxsize=256)
def _route(n_experts, k, score, n_groups, top_groups, renormalise, scale):
    if score not in _SCORES:
        raise ValueError("score must be 'softmax' or 'sigmoid'")
    return ctypes.byref(_Route(n_experts, k, _SCORES[score], n_groups, top_groups, int(bool(renormalise)), scale))


def route_topk(logits, k, *, score="softmax", bias=None, n_groups=1, top_groups=1, renormalise=True, scale=1.0, ids=None, weights=None):
    """The ``k`` experts of every row of ``logits`` [T, E] (float32, bfloat16 or float16; row stride free) and their weights: int32 and float32
    [T, k], allocated here unless given.  ``bias``: float32 [E], added to the scores for the choice alone."""
    what = "route_topk"
    if logits.requires_grad:
        _cut_off(what)
    ld = _rows(what, "logits", logits, None, None, _TYPES)
    n_rows, n_experts = logits.shape
    device = logits.get_device()
    if bias is not None:
        _dense(what, "bias", bias, (n_experts,), torch.float32)
    if ids is None:
        ids = _new(n_rows, k, torch.int32, logits.device)
    else:
        _dense(what, "ids", ids, (n_rows, k), torch.int32)
    if weights is None:
        weights = _new(n_rows, k, torch.float32, logits.device)
    else:
        _dense(what, "weights", weights, (n_rows, k), torch.float32)
    _together(what, device, bias, ids, weights)
    _call(what, _lib.route_topk, device, _route(n_experts, int(k), score, int(n_groups), int(top_groups), renormalise, float(scale)), logits.data_ptr(), ld,
          _TYPES[logits.dtype], None if bias is None else bias.data_ptr(), n_rows, ids.data_ptr(), weights.data_ptr())
    return ids, weights


def route_topk_grad(logits, ids, dweights, *, score="softmax", renormalise=True, scale=1.0, dlogits=None):
    """The gradient to ``logits`` of the weights that ``route_topk`` gave with the same arguments, for ``dweights`` [T, k]; in logits' type."""
    what = "route_topk_grad"
    ld = _rows(what, "logits", logits, None, None, _TYPES)
    n_rows, n_experts = logits.shape
    device = logits.get_device()
    if ids.dim() != 2:
        raise ValueError("%s: ids must be of shape (T, k)" % what)
    k = ids.shape[1]
    _dense(what, "ids", ids, (n_rows, k), torch.int32)
    _dense(what, "dweights", dweights, (n_rows, k), torch.float32)
    if dlogits is None:
        dlogits, ldd = _new(n_rows, n_experts, logits.dtype, logits.device), n_experts
    else:
        ldd = _rows(what, "dlogits", dlogits, n_rows, n_experts, (logits.dtype,))
    _together(what, device, ids, dweights, dlogits)
    _call(what, _lib.route_topk_grad, device, _route(n_experts, k, score, 1, 1, renormalise, float(scale)), logits.data_ptr(), ld, _TYPES[logits.dtype],
          ids.data_ptr(), dweights.data_ptr(), n_rows, dlogits.data_ptr(), ldd)
    return dlogits


class RoutePlan:
    """The pairs of ``ids`` grouped by expert: ``offsets`` int32 [E + 1], ``order`` int32 [T k] (views of the plan's buffer)."""

    def __init__(self, buf, n_rows, top_k, n_experts):
        self._buf, self._at = buf, buf.data_ptr()
        self.n_rows, self.top_k, self.n_pairs, self.n_experts = n_rows, top_k, n_rows * top_k, n_experts

    @property
    def offsets(self):
        return self._buf.as_strided((self.n_experts + 1,), (1,), 0)

    @property
    def order(self):
        return self._buf.as_strided((self.n_pairs,), (1,), _lib.route_plan_order(self.n_pairs, self.n_experts) // 4)


@lru_cache(maxsize=1024)
def _plan_bytes(n_pairs, n_experts):
    n = int(_lib.route_plan_bytes(n_pairs, n_experts))
    if n == 0:
        raise VbrError(-1, "route_plan")
    return n


def route_plan(ids, n_experts) -> RoutePlan:
    """Group the pairs of ``ids`` (int32 [T, k]) by expert.  Ids outside [0, n_experts) belong to none."""
    what = "route_plan"
    if ids.dim() != 2:
        raise ValueError("%s: ids must be of shape (T, k)" % what)
    _dense(what, "ids", ids, ids.shape, torch.int32)
    n_rows, k = ids.shape
    n_experts = int(n_experts)
    buf = torch.empty(_plan_bytes(n_rows * k, n_experts) // 4, dtype=torch.int32, device=ids.device)
    plan = RoutePlan(buf, n_rows, k, n_experts)
    _call(what, _lib.route_plan, ids.get_device(), ids.data_ptr(), n_rows * k, n_experts, plan._at)
    return plan


_ANY = 2 ** 31 - 1


def route_combine(y, ids, weights, out=None, *, out_dtype=None, n_experts=_ANY):
    """out[t] = sum over j of weights[t, j] * y[t k + j], in ``out_dtype`` (y's, if not given).  Pairs whose id is negative, or not below
    ``n_experts``, are left out."""
    what = "route_combine"
    if y.requires_grad or weights.requires_grad:
        _cut_off(what)
    n_rows, k, n_cols, ldy, device = _sum_operands(what, y, ids, weights)
    if out_dtype is not None and (out_dtype not in _TYPES or (out is not None and out.dtype is not out_dtype)):
        raise ValueError("%s: out_dtype must be float32, bfloat16 or float16, and out's" % what)
    if out is None:
        out, ldo = _new(n_rows, n_cols, out_dtype or y.dtype, y.device), n_cols
    else:
        ldo = _rows(what, "out", out, n_rows, n_cols, _TYPES)
    _together(what, device, ids, weights, out)
    _call(what, _lib.route_combine, device, y.data_ptr(), ldy, _TYPES[y.dtype], ids.data_ptr(), weights.data_ptr(), n_rows, k, n_experts, n_cols, out.data_ptr(), ldo,
          _TYPES[out.dtype])
    return out


def _sum_operands(what, y, ids, weights):
    if ids.dim() != 2:
        raise ValueError("%s: ids must be of shape (T, k)" % what)
    n_rows, k = ids.shape
    _dense(what, "ids", ids, ids.shape, torch.int32)
    _dense(what, "weights", weights, ids.shape, torch.float32)
    ldy = _rows(what, "y", y, n_rows * k, None, _TYPES)
    return n_rows, k, y.shape[1], ldy, y.get_device()


def route_combine_grad(dout, y, ids, weights, dy=None, dweights=None, *, n_experts=_ANY):
    """The gradients of ``route_combine`` for ``dout`` [T, D]: (dy in y's type, dweights float32 [T, k])."""
    what = "route_combine_grad"
    n_rows, k, n_cols, ldy, device = _sum_operands(what, y, ids, weights)
    ldo = _rows(what, "dout", dout, n_rows, n_cols, _TYPES)
    if dy is None:
        dy, lddy = _new(n_rows * k, n_cols, y.dtype, y.device), n_cols
    else:
        lddy = _rows(what, "dy", dy, n_rows * k, n_cols, (y.dtype,))
    if dweights is None:
        dweights = _new(n_rows, k, torch.float32, y.device)
    else:
        _dense(what, "dweights", dweights, (n_rows, k), torch.float32)
    _together(what, device, dout, ids, weights, dy, dweights)
    _call(what, _lib.route_combine_grad, device, dout.data_ptr(), ldo, _TYPES[dout.dtype], y.data_ptr(), ldy, _TYPES[y.dtype], ids.data_ptr(), weights.data_ptr(),
          n_rows, k, n_experts, n_cols, dy.data_ptr(), lddy, dweights.data_ptr())
    return dy, dweights


class Q4:
    """Matrices in 4 bits.  ``codes`` uint8 [M, N, K / 2] or [N, K / 2], ``scales`` float16 or bfloat16 [M, N, ceil(K / group)], ``zeros`` uint8 of the
    same shape or None (8 everywhere); ``gated``: the first N / 2 rows gate the others.  ``upload`` lays them out on the GPU they are on,
    after which the tensors given are not needed."""

    def __init__(self, codes, scales, zeros=None, *, group, gated=False):
        what = "Q4"
        self._h = ctypes.c_void_p(None)
        if codes.dtype is not torch.uint8 or codes.dim() not in (2, 3) or scales.dim() != codes.dim():
            raise ValueError("%s: codes must be uint8 [M, N, K / 2] or [N, K / 2], scales with as many dimensions" % what)
        if scales.dtype not in (torch.float16, torch.bfloat16):
            raise ValueError("%s: scales must be float16 or bfloat16" % what)
        n_rows, n_cols, group = codes.shape[-2], 2 * codes.shape[-1], int(group)
        n_mats = codes.shape[0] if codes.dim() == 3 else 1
        shape = tuple(codes.shape[:-1]) + ((n_cols + group - 1) // group if group > 0 else 0,)
        if tuple(scales.shape) != shape:
            raise ValueError("%s: scales must be of shape %s, not %s" % (what, shape, tuple(scales.shape)))
        if zeros is not None and (zeros.dtype is not torch.uint8 or tuple(zeros.shape) != shape):
            raise ValueError("%s: zeros must be uint8 of shape %s" % (what, shape))
        _together(what, codes.get_device(), scales, zeros)
        h = ctypes.c_void_p()
        rc = _lib.q4_create(n_mats, n_rows, n_cols, group, _TYPES[scales.dtype], int(zeros is not None), int(bool(gated)), ctypes.byref(h))
        if rc != 0:
            raise VbrError(rc, "q4_create")
        self._h = h
        self.dtype, self.group, self.gated = scales.dtype, group, bool(gated)
        self.n_mats, self.n_rows, self.n_cols = n_mats, n_rows, n_cols
        self.n_out = n_rows // 2 if gated else n_rows
        self._given = (codes, scales, zeros)
        self._dev = None

    def close(self):
        if self._h:
            _lib.q4_free(self._h)
            self._h = ctypes.c_void_p(None)
            self._dev = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def device_bytes(self) -> int:
        return int(_lib.q4_device_bytes(self._h))

    def upload(self):
        if self._given is None:
            raise VbrError(-4, "q4_upload")
        codes, scales, zeros = (None if t is None else t.contiguous() for t in self._given)
        if codes.data_ptr() % 4:                     # a view that begins between words
            codes = codes.clone()
        if codes.get_device() < 0:
            raise ValueError("q4_upload: the matrices must be on the GPU")
        buf = torch.empty(self.device_bytes(), dtype=torch.uint8, device=codes.device)
        _call("q4_upload", _lib.q4_upload, codes.get_device(), self._h, codes.data_ptr(), scales.data_ptr(), None if zeros is None else zeros.data_ptr(),
              buf.data_ptr())
        self._dev, self._given = buf, None
        return self

    def _operands(self, what, x, n_out, y, y_dtype):
        if x.requires_grad:
            _cut_off(what)
        ldx = _rows(what, "x", x, None, self.n_cols, (self.dtype,))
        if y is None:
            if y_dtype is not None and y_dtype is not self.dtype and y_dtype is not torch.float32:
                raise ValueError("%s: y must be of the matrix's type or float32" % what)
            y, ldy = _new(n_out, self.n_out, y_dtype or self.dtype, x.device), self.n_out
        else:
            if y_dtype is not None and y.dtype is not y_dtype:
                raise ValueError("%s: y is not of y_dtype" % what)
            ldy = _rows(what, "y", y, n_out, self.n_out, (self.dtype, torch.float32))
        if self._dev is None:
            raise VbrError(-4, what)
        device = self._dev.get_device()
        _together(what, device, x, y)
        return ldx, y, ldy, device

    def mm(self, x, y=None, *, y_dtype=None):
        """y = x W^T: ``x`` [T, K] in the matrix's type (row stride free, a multiple of 8), ``y`` [T, N] (N / 2 gated) in that type or
        float32, allocated here unless given."""
        what = "q4_mm"
        ldx, y, ldy, device = self._operands(what, x, x.shape[0], y, y_dtype)
        _call(what, _lib.q4_mm, device, self._h, x.data_ptr(), ldx, y.data_ptr(), ldy, _TYPES[y.dtype], x.shape[0])
        return y

    def mm_routed(self, x, plan, y=None, *, y_dtype=None):
        """y[t k + j] = x[t] (or x[t k + j], if ``x`` has a row for every pair) times the matrix of the pair's expert, transposed.  Rows of y
        of pairs without an expert are left as they are."""
        what = "q4_mm_routed"
        if plan.n_experts != self.n_mats:
            raise ValueError("%s: the plan is for %d experts, there are %d matrices" % (what, plan.n_experts, self.n_mats))
        n_x = x.shape[0]
        if n_x != plan.n_rows and n_x != plan.n_pairs:
            raise ValueError("%s: x has %d rows, the plan is for %d rows and %d pairs" % (what, n_x, plan.n_rows, plan.n_pairs))
        ldx, y, ldy, device = self._operands(what, x, plan.n_pairs, y, y_dtype)
        _together(what, device, plan._buf)
        _call(what, _lib.q4_mm_routed, device, self._h, plan._at, plan.n_pairs, x.data_ptr(), ldx, n_x, y.data_ptr(), ldy, _TYPES[y.dtype])
        return y


def experts_forward(x, ids, weights, up, down, out=None):
    """A layer of experts: out[t] = sum over j of weights[t, j] * down_e(up_e(x[t])), e = ids[t, j]; ``up`` is gated.  What ``up`` gives is rounded to the
    matrices' type, which the second product multiplies; its results stay in float32 until they are summed."""
    if not up.gated or up.n_out != down.n_cols or up.n_mats != down.n_mats or down.gated or up.dtype is not down.dtype:
        raise ValueError("experts_forward: up must be gated, and down take what it gives, of as many experts and the same type")
    what = "experts_forward"
    if x.requires_grad or weights.requires_grad:
        _cut_off(what)
    if ids.dim() != 2:
        raise ValueError("%s: ids must be of shape (T, k)" % what)
    n_rows, k = ids.shape
    ldx = _rows(what, "x", x, n_rows, up.n_cols, (up.dtype,))
    _dense(what, "ids", ids, ids.shape, torch.int32)
    _dense(what, "weights", weights, ids.shape, torch.float32)
    if out is None:
        out, ldo = _new(n_rows, down.n_out, x.dtype, x.device), down.n_out
    else:
        ldo = _rows(what, "out", out, n_rows, down.n_out, _TYPES)
    if up._dev is None or down._dev is None:
        raise VbrError(-4, what)
    device = up._dev.get_device()
    _together(what, device, down._dev, x, ids, weights, out)
    n_bytes = int(_lib.experts_work_bytes(up._h, down._h, n_rows, k))
    if n_bytes == 0:
        raise VbrError(-1, what)
    work = torch.empty(n_bytes, dtype=torch.uint8, device=x.device)
    _call(what, _lib.experts_forward, device, up._h, down._h, x.data_ptr(), ldx, n_rows, ids.data_ptr(), weights.data_ptr(), k, out.data_ptr(), ldo,
          _TYPES[out.dtype], work.data_ptr())
    return out
