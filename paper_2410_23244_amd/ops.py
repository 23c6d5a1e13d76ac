"""Binding of the second part of libbart (include/bart_ops.h): log
probabilities of given classes with entropy, best alternatives and gradients,
and AdamW steps over many tensors.

Argument marshalling only, as in :mod:`paper_2410_23244_amd.bart`: torch
tensors give memory and the current stream, every computation is a HIP kernel
of libbart.so, and there is no CPU fallback.  Definitions, and what happens in
rows that need a rule, are in the header.

Results carry no graph of torch's automatic differentiation, also where scores
require a gradient: scores.backward(r.grad) goes on from here.  Tensors that are
written in place (weights, grad_out) count as modified.

    r = logprob(scores, labels, k=3, entropy=True)       # answers
    r.logp, r.entropy, r.top_class, r.top_logp

    r = logprob(scores, labels, grad_logp=-weights)      # a loss and its gradient
    loss, r.grad                                         # loss = -(weights * r.logp).sum()

    r = logprob(scores, labels, norm=True, entropy=True) # weights known only later
    grad = logprob_grad(scores, labels, r.norm, w, entropy=r.entropy, grad_entropy=h)

    opt = AdamW([W, b], [dW, db], lr=1e-2, weight_decay=[1e-3, 0.0])
    opt.step()
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

import torch
from torch.autograd.graph import increment_version

from . import bart
from .bart import BART_EINVAL, BartError, _check

BART_F32, BART_F16, BART_BF16 = 0, 1, 2
BART_MAX_TOP = 64
MAX_CLASSES = 1 << 30
STATE_BLOCK = 256
_DTYPES = {torch.float32: BART_F32, torch.float16: BART_F16, torch.bfloat16: BART_BF16}


class Rows(C.Structure):
    _fields_ = [("x", C.c_void_p), ("n", C.c_int64), ("ld", C.c_int64), ("n_class", C.c_int32),
                ("dtype", C.c_int32), ("label", C.c_void_p), ("label_stride", C.c_int64),
                ("mask", C.c_void_p), ("ld_mask", C.c_int64), ("temperature", C.c_double)]


class RowsGrad(C.Structure):
    _fields_ = [("w_logp", C.c_void_p), ("w_logp_stride", C.c_int64), ("w_entropy", C.c_void_p),
                ("w_entropy_stride", C.c_int64), ("grad", C.c_void_p), ("ld_grad", C.c_int64)]


class RowsOut(C.Structure):
    _fields_ = [("logp", C.c_void_p), ("entropy", C.c_void_p), ("norm", C.c_void_p),
                ("k", C.c_int32), ("top_logp", C.c_void_p), ("top_class", C.c_void_p)]


class AdamwTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("master", C.c_void_p),
                ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("n", C.c_int64), ("param_dtype", C.c_int32),
                ("grad_dtype", C.c_int32), ("weight_decay", C.c_float), ("lr_scale", C.c_float)]


class AdamwHyper(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double),
                ("eps", C.c_double), ("grad_scale", C.c_double), ("step", C.c_int64)]


_lib = None


def lib():
    global _lib
    if _lib is None:
        L = bart.lib()
        vp, P = C.c_void_p, C.POINTER
        L.bart_logprob_workspace_bytes.argtypes = [P(Rows), P(RowsOut), P(RowsGrad)]
        L.bart_logprob_workspace_bytes.restype = C.c_size_t
        L.bart_logprob.argtypes = [P(Rows), P(RowsOut), P(RowsGrad), vp, C.c_size_t, vp]
        L.bart_logprob_grad.argtypes = [P(Rows), vp, vp, P(RowsGrad), vp]
        L.bart_adamw_workspace_bytes.argtypes = [P(AdamwTensor), C.c_int32, C.c_int32]
        L.bart_adamw_workspace_bytes.restype = C.c_size_t
        L.bart_adamw_init.argtypes = [P(AdamwTensor), C.c_int32, C.c_int32, vp, C.c_size_t, vp,
                                      P(vp)]
        L.bart_adamw_step.argtypes = [vp, P(AdamwHyper), vp]
        L.bart_adamw_destroy.argtypes = [vp]
        L.bart_adamw_destroy.restype = None
        for f in ("bart_logprob", "bart_logprob_grad", "bart_adamw_init", "bart_adamw_step"):
            getattr(L, f).restype = C.c_int
        _lib = L
    return _lib


def _refuse(msg: str):
    raise BartError(BART_EINVAL, msg)


# ------------------------------------------------------------- rows of scores

class LogProb(NamedTuple):
    """What :func:`logprob` computed; None where it was not asked for."""
    logp: Optional[torch.Tensor]       # f32 [n]
    entropy: Optional[torch.Tensor]    # f32 [n]
    norm: Optional[torch.Tensor]       # f32 [n, 2], for logprob_grad
    top_logp: Optional[torch.Tensor]   # f32 [n, k]
    top_class: Optional[torch.Tensor]  # i32 [n, k]
    grad: Optional[torch.Tensor]       # scores' dtype [n, classes]


def _new(shape, strides, dtype, device):
    # the quickest of torch's allocations, by 0.4 us of the 14 that a small call takes
    return torch.empty_strided(shape, strides, dtype=dtype, device=device)


def _stride0(t: torch.Tensor, n: int) -> int:
    return t.stride(0) if n > 1 else 1


def _rows(scores, labels, mask, temperature) -> Rows:
    if scores.dim() != 2:
        _refuse(f"scores must be [rows, classes], not of {scores.dim()} dimensions")
    n, c = scores.shape
    dtype = _DTYPES.get(scores.dtype)
    if dtype is None:
        _refuse(f"scores must be float32, float16 or bfloat16, not {scores.dtype}")
    if not scores.is_cuda:
        _refuse("scores must be on a HIP device")
    if not 1 <= c <= MAX_CLASSES:   # the library's field is narrower than a tensor's size
        _refuse(f"scores must have 1 to 2^30 classes, not {c}")
    if c > 1 and scores.stride(1) != 1:
        _refuse("the classes of a row must be next to each other (stride 1)")
    r = Rows(scores.data_ptr(), n, scores.stride(0) if n > 1 else c, c, dtype, None, 0, None, 0,
             temperature)
    if labels is not None:
        if labels.dtype != torch.int64 or labels.shape != (n,) or labels.device != scores.device:
            _refuse(f"labels must be int64 [{n}] on the scores' device")
        r.label, r.label_stride = labels.data_ptr(), _stride0(labels, n)
    if mask is not None:
        if mask.dtype not in (torch.bool, torch.uint8) or mask.device != scores.device:
            _refuse("mask must be bool or uint8 on the scores' device")
        if mask.shape == (c,):
            ld = 0
        elif mask.shape == (n, c):
            ld = mask.stride(0) if n > 1 else c
        else:
            _refuse(f"mask must be [{c}] or [{n}, {c}]")
        if c > 1 and mask.stride(-1) != 1:
            _refuse("the classes of a mask's row must be next to each other (stride 1)")
        r.mask, r.ld_mask = mask.data_ptr(), ld
    return r


def _rows_grad(scores, grad_logp, grad_entropy, out):
    n = scores.shape[0]
    if out is None:
        out = _new(scores.shape, (scores.shape[1], 1), scores.dtype, scores.device)
    elif out.shape != scores.shape or out.dtype != scores.dtype or out.device != scores.device:
        _refuse("grad_out must have the scores' shape, dtype and device")
    elif scores.shape[1] > 1 and out.stride(1) != 1:
        _refuse("the classes of a row of grad_out must be next to each other (stride 1)")
    g = RowsGrad(None, 0, None, 0, out.data_ptr(), out.stride(0) if n > 1 else scores.shape[1])
    for name, w in (("w_logp", grad_logp), ("w_entropy", grad_entropy)):
        if w is None:
            continue
        if w.dtype != torch.float32 or w.device != scores.device or w.shape not in ((n,), ()):
            _refuse(f"the weights of a gradient must be float32 [{n}] or one number, "
                    "on the scores' device")
        setattr(g, name, w.data_ptr())
        setattr(g, name + "_stride", 0 if w.dim() == 0 else _stride0(w, n))
    return g, out


def _call(device, f, *args):
    """f on the tensors' device, given its current stream as the last argument."""
    if device.index == torch.cuda.current_device():
        _check(f(*args, torch.cuda.current_stream(device.index).cuda_stream))
    else:
        with torch.cuda.device(device):
            _check(f(*args, torch.cuda.current_stream(device).cuda_stream))


class Held:
    """Device memory that calls use and whose user does not see it: the allocator
    is told of every other stream it is used on than the one it was made on, so
    that memory dropped behind such a call is not handed out before the call is
    done."""

    def __init__(self, tensors, device):
        self.tensors = [t for t in tensors if t is not None and t.numel()]
        self.streams = {torch.cuda.current_stream(device).cuda_stream}

    def use(self, device, handle: int) -> None:
        """handle: that of the device's current stream."""
        if handle not in self.streams:
            stream = torch.cuda.current_stream(device)
            for t in self.tensors:
                t.record_stream(stream)
            self.streams.add(handle)


def logprob(scores, labels=None, *, mask=None, temperature: float = 1.0, k: int = 0,
            entropy: bool = False, norm: bool = False, grad_logp=None, grad_entropy=None,
            grad_out=None) -> LogProb:
    """Log probabilities of rows of scores.

    scores: [n, classes] float32, float16 or bfloat16, any row stride.  labels:
    int64 [n], negative where a row has none (without labels, no logp).  mask:
    the allowed classes, bool [classes] or [n, classes].  k: alternatives per
    row, at most 64.  entropy, norm: whether to return them.  grad_logp,
    grad_entropy: float32 [n] or a 0-dim tensor; given one of them, grad is
    the gradient of sum(grad_logp * logp + grad_entropy * entropy) with respect
    to the scores, in grad_out (which may be the scores themselves) or a new
    tensor."""
    L = lib()
    r = _rows(scores, labels, mask, temperature)
    if not 0 <= k <= BART_MAX_TOP:
        _refuse(f"k must be in [0, {BART_MAX_TOP}]")
    n, dev = r.n, scores.device
    got_logp = _new((n,), (1,), torch.float32, dev) if labels is not None else None
    got_entropy = _new((n,), (1,), torch.float32, dev) if entropy else None
    got_norm = _new((n, 2), (2, 1), torch.float32, dev) if norm else None
    top_logp = _new((n, k), (k, 1), torch.float32, dev) if k else None
    top_class = _new((n, k), (k, 1), torch.int32, dev) if k else None
    o = RowsOut(got_logp.data_ptr() if got_logp is not None else None,
                got_entropy.data_ptr() if entropy else None,
                got_norm.data_ptr() if norm else None, k,
                top_logp.data_ptr() if k else None, top_class.data_ptr() if k else None)
    g, grad = None, None
    if grad_logp is not None or grad_entropy is not None:
        g, grad = _rows_grad(scores, grad_logp, grad_entropy, grad_out)
    elif grad_out is not None:
        _refuse("grad_out needs grad_logp or grad_entropy")
    need = L.bart_logprob_workspace_bytes(r, o, g)
    ws = _new((need,), (1,), torch.uint8, dev) if need else None
    _call(dev, L.bart_logprob, r, o, g, ws.data_ptr() if need else None, need)
    if grad_out is not None:
        increment_version(grad_out)
    return LogProb(got_logp, got_entropy, got_norm, top_logp, top_class, grad)


def logprob_grad(scores, labels, norm, grad_logp, *, entropy=None, grad_entropy=None, mask=None,
                 temperature: float = 1.0, grad_out=None) -> torch.Tensor:
    """The gradient of sum(grad_logp * logp + grad_entropy * entropy) with
    respect to the scores, from the norm (and entropy, where grad_entropy is
    given) that :func:`logprob` returned for the same scores, mask and
    temperature."""
    r = _rows(scores, labels, mask, temperature)
    n = r.n
    if norm is None:
        _refuse("the gradient alone needs the norm that logprob returned")
    for name, t, shape in (("norm", norm, (n, 2)), ("entropy", entropy, (n,))):
        if t is not None and (t.dtype != torch.float32 or t.shape != shape or
                              t.device != scores.device or not t.is_contiguous()):
            _refuse(f"{name} must be contiguous float32 {list(shape)} on the scores' device")
    g, grad = _rows_grad(scores, grad_logp, grad_entropy, grad_out)
    _call(scores.device, lib().bart_logprob_grad, r, norm.data_ptr(),
          entropy.data_ptr() if entropy is not None else None, g)
    if grad_out is not None:
        increment_version(grad_out)
    return grad


# ---------------------------------------------------------------------- AdamW

def _dense(t: torch.Tensor) -> bool:
    """Whether the elements fill one stretch of memory, in any order of dimensions."""
    if t.numel() == 0:
        return True
    need = 1
    for size, stride in sorted(((s, st) for s, st in zip(t.shape, t.stride()) if s != 1),
                               key=lambda q: q[1]):
        if stride != need:
            return False
        need *= size
    return True


def _same_layout(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether two dense tensors of one shape hold their elements in one order."""
    return a.shape == b.shape and (a.stride() == b.stride() or a.numel() == 0 or all(
        s == 1 or x == y for s, x, y in zip(a.shape, a.stride(), b.stride())))


def _ptr(t):
    return None if t is None or t.numel() == 0 else t.data_ptr()


class AdamW:
    """AdamW over a list of tensors, one launch per step for tensors of equal types.

    params, grads: lists of dense tensors, pairwise of one shape and layout,
    on one device and apart from each other (a shared weight is given once);
    params float32, float16 or bfloat16, grads of the param's dtype or float32.
    They are updated and read in place: a step uses what the grads hold when it
    runs.  masters: None, or for 16-bit params a list of float32 tensors that hold
    the weights, of which the params are then rounded copies ("new" makes them
    from the params).  weight_decay, lr_scale: a number, or one for each tensor.

    state_bits 32: float32 moments, state[i]["m"] and ["v"].  state_bits 8:
    float8_e4m3fn state[i]["m"] and ["r"] (the ROOT of the second moment),
    flat in the param's memory order, with float32 scales of each 256 elements
    in ["m_scale"] and ["r_scale"]: m = code * scale, v = (code * scale)^2.
    state: such a list to go on from (used in place), after `steps` steps."""

    def __init__(self, params, grads, *, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.0, lr_scale=1.0, state_bits: int = 32, masters=None, state=None,
                 steps: int = 0):
        params, grads = list(params), list(grads)
        if not params or len(params) != len(grads):
            _refuse("params and grads must be lists of the same length, at least 1")
        if state_bits not in (8, 32):
            _refuse("state_bits must be 32 or 8")
        self.device = dev = params[0].device
        if dev.type != "cuda":
            _refuse("params must be on a HIP device")
        n = len(params)
        self.params, self.grads, self.state_bits, self.steps = params, grads, state_bits, int(steps)
        self.lr, self.betas, self.eps = float(lr), (float(betas[0]), float(betas[1])), float(eps)
        made = []
        if isinstance(masters, str):
            if masters != "new":
                _refuse('masters must be None, "new" or a list')
            masters = [p.float() if p.dtype != torch.float32 else None for p in params]
            made += masters
        self.masters = list(masters) if masters is not None else [None] * n
        wd = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * n
        scale = list(lr_scale) if hasattr(lr_scale, "__len__") else [lr_scale] * n
        if state is None:
            state = [self._new_state(p) for p in params]
            made += [t for s in state for t in s.values()]
        self.state = list(state)
        if not n == len(self.masters) == len(wd) == len(scale) == len(self.state):
            _refuse("masters, weight_decay, lr_scale and state must have one entry per tensor")
        table = (AdamwTensor * n)()
        for i, (p, g, w, s) in enumerate(zip(params, grads, self.masters, self.state)):
            self._check_tensor(i, p, g, w, s)
            small = state_bits == 8
            table[i] = AdamwTensor(_ptr(p), _ptr(g), _ptr(w), _ptr(s["m"]),
                                   _ptr(s["r" if small else "v"]),
                                   _ptr(s["m_scale"]) if small else None,
                                   _ptr(s["r_scale"]) if small else None, p.numel(),
                                   _DTYPES[p.dtype], _DTYPES[g.dtype], wd[i], scale[i])
        L = lib()
        need = L.bart_adamw_workspace_bytes(table, n, state_bits)
        self.ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
        self._held = Held(made + [self.ws], dev)
        self._weights = params + [w for w in self.masters if w is not None]
        self.h, h = None, C.c_void_p()
        with torch.cuda.device(dev):
            _check(L.bart_adamw_init(table, n, state_bits, self.ws.data_ptr(), need,
                                     torch.cuda.current_stream(dev).cuda_stream, C.byref(h)))
        self.h = h.value

    def _new_state(self, p):
        n, nb = p.numel(), (p.numel() + STATE_BLOCK - 1) // STATE_BLOCK
        if self.state_bits == 32:
            return dict(m=torch.zeros_like(p, dtype=torch.float32),
                        v=torch.zeros_like(p, dtype=torch.float32))

        def zeros(k, dtype):
            return torch.zeros(k, dtype=dtype, device=p.device)

        return dict(m=zeros(n, torch.uint8).view(torch.float8_e4m3fn),
                    r=zeros(n, torch.uint8).view(torch.float8_e4m3fn),
                    m_scale=zeros(nb, torch.float32), r_scale=zeros(nb, torch.float32))

    def _check_tensor(self, i, p, g, w, s):
        def same(t, dtype):
            return t.dtype == dtype and _same_layout(t, p) and t.device == self.device

        def flat(t, dtype, n):
            return (t.dtype == dtype and t.shape == (n,) and t.is_contiguous() and
                    t.device == self.device)

        if p.dtype not in _DTYPES:
            _refuse(f"param {i} must be float32, float16 or bfloat16, not {p.dtype}")
        if p.device != self.device or not _dense(p):
            _refuse(f"param {i} must be dense and on the device of the first one")
        if g.dtype not in (p.dtype, torch.float32) or not same(g, g.dtype):
            _refuse(f"grad {i} must have its param's shape, layout and device, and its dtype or "
                    "float32")
        if w is not None and (p.dtype == torch.float32 or not same(w, torch.float32)):
            _refuse(f"master {i} must be float32, of the shape and layout of its 16-bit param")
        n, nb = p.numel(), (p.numel() + STATE_BLOCK - 1) // STATE_BLOCK
        if self.state_bits == 32:
            ok = all(k in s and same(s[k], torch.float32) for k in ("m", "v"))
        else:
            ok = (all(k in s and flat(s[k], torch.float8_e4m3fn, n) for k in ("m", "r")) and
                  all(k in s and flat(s[k], torch.float32, nb) for k in ("m_scale", "r_scale")))
        if not ok:
            _refuse(f"state {i} does not fit its param and state_bits = {self.state_bits}")

    def step(self, lr: Optional[float] = None, grad_scale: float = 1.0) -> None:
        """One step on the current stream (lr: of this step alone).  A graph that
        captured it repeats this one step, with its number, lr and grad_scale, at
        every replay, and needs this object as long as it is replayed: train by
        calls, not by replays."""
        y = AdamwHyper(self.lr if lr is None else lr, self.betas[0], self.betas[1], self.eps,
                       grad_scale, self.steps + 1)
        # the handle alone: a stream's object takes 1.1 us of the 5 of a small step
        stream = torch._C._cuda_getCurrentRawStream(self.device.index)
        self._held.use(self.device, stream)
        _check(lib().bart_adamw_step(self.h, y, stream))
        increment_version(self._weights)
        self.steps += 1

    def close(self) -> None:
        if getattr(self, "h", None):
            lib().bart_adamw_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
