"""Operators of a token model's potential (``Sampler`` has them as methods):
embedding, linear layer, gated block and categorical likelihood, each with its
gradient, in fp32 or bf16 on device tensors.

Every call enqueues HIP kernels on torch's current stream and returns without
waiting (so it can be captured into a graph).  Matrices are 2-D with unit column stride (any row stride);
gradients are functions of their own, so a potential's gradient is written as
the calls in reverse.
"""
from __future__ import annotations

import ctypes


class _Torch:
    """torch, imported at the first use (the rest of the package does without)."""

    def __getattr__(self, name):
        import torch as t
        v = getattr(t, name)
        setattr(self, name, v)
        return v


torch = _Torch()
NUTS_F32, NUTS_BF16 = 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "sigmoid": 2, "silu": 3, "gelu": 4}
NUTS_ROUND_DZ = 256

_P, _i64, _i32, _dbl = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double


def _record(name, fields):
    kinds = {"p": _P, "n": _i64, "i": _i32, "d": _dbl}
    return type(name, (ctypes.Structure,), {"_fields_": [(f[2:], kinds[f[0]]) for f in fields.split()]})


_Embedding = _record("_Embedding", "i:dtype i:_reserved n:N n:V n:D p:ids p:table n:ld_table d:scale p:out n:ld_out")
_EmbeddingGrad = _record("_EmbeddingGrad", "i:dtype i:_reserved n:N n:V n:D p:ids p:dout n:ld_dout d:scale p:dtable "
                                           "n:ld_dtable")
_Linear = _record("_Linear", "i:dtype i:act n:M n:N n:K p:x n:ldx p:w n:ldw p:bias p:residual n:ldr p:y n:ldy p:pre")
_LinearGrad = _record("_LinearGrad", "i:dtype i:act n:M n:N n:K p:dy n:lddy p:x n:ldx p:w n:ldw p:pre p:dx n:lddx "
                                     "p:dw n:lddw p:dbias")
_Gated = _record("_Gated", "i:dtype i:act n:M n:F n:K p:x n:ldx p:wg n:ldwg p:wu n:ldwu p:y n:ldy p:pre")
_GatedGrad = _record("_GatedGrad", "i:dtype i:act n:M n:F n:K p:dy n:lddy p:x n:ldx p:wg n:ldwg p:wu n:ldwu p:pre "
                                   "p:dx n:lddx p:dwg n:lddwg p:dwu n:lddwu")
_Categorical = _record("_Categorical", "i:dtype i:_reserved n:M n:V p:logits n:ld_logits p:targets d:scale p:nll "
                                       "p:total p:dlogits n:ld_dlogits")

_CALLS = {"nuts_embedding": (_Embedding, False), "nuts_embedding_grad": (_EmbeddingGrad, True),
          "nuts_linear": (_Linear, True), "nuts_linear_grad": (_LinearGrad, True),
          "nuts_gated": (_Gated, True), "nuts_gated_grad": (_GatedGrad, True),
          "nuts_categorical": (_Categorical, False)}
# What include/nuts_token.h declares.
EXPORTED = list(_CALLS) + [name + "_workspace" for name, (_, space) in _CALLS.items() if space]


def declare(L):
    """Declare the library's functions; {name: (function, its workspace's size)}."""
    calls = {}
    for name, (args, space) in _CALLS.items():
        fn = getattr(L, name)
        fn.argtypes = [_P, ctypes.POINTER(args)] + ([_P, _i64] if space else []) + [_P]
        fn.restype = ctypes.c_int
        if space:
            fn = getattr(L, name + "_workspace")
            fn.argtypes = [ctypes.POINTER(args)]
            fn.restype = _i64
        calls[name] = (getattr(L, name), fn if space else None)
    return calls


def _type(t, name):
    if t.dtype is torch.bfloat16:
        return NUTS_BF16
    if t.dtype is torch.float32:
        return NUTS_F32
    raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")


def _matrix(t, name, dtype, rows=None, cols=None):
    """(pointer, row stride) of a 2-D tensor with unit column stride (of a
    single row: its length, whatever the tensor says)."""
    if t.dim() != 2 or t.dtype != dtype:
        raise TypeError(f"{name} must be a 2-D {dtype} tensor, got {t.dim()}-D {t.dtype}")
    R, C = t.shape
    if (rows is not None and R != rows) or (cols is not None and C != cols):
        raise ValueError(f"{name} must have shape ({rows}, {cols}), got {tuple(t.shape)}")
    ld, step = t.stride()
    if C > 1 and step != 1:
        raise ValueError(f"{name}: columns must be adjacent in memory (strides {t.stride()})")
    return t.data_ptr(), (ld if R > 1 else C)


def _vector(t, name, dtype, n):
    if t.dim() != 1 or t.dtype != dtype or t.shape[0] != n:
        raise TypeError(f"{name} must be a {dtype} vector of {n}, got {tuple(t.shape)} {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _act(name):
    try:
        return ACTIVATIONS[name]
    except KeyError:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, got {name!r}") from None


class TokenOps:
    """Methods of ``Sampler`` (which provides ``_h``, ``_check`` and
    ``_token_calls``)."""

    def _call(self, name, args, device):
        """Enqueue, with the workspace that the call asks for."""
        ref = ctypes.byref(args)
        # (host tensors are refused by the library)
        stream = torch._C._cuda_getCurrentRawStream(device.index) if device.type == "cuda" else None
        fn, space = self._token_calls[name]
        if space is None:
            self._check(fn(self._h, ref, stream))
            return
        need = space(ref)
        if need > 0:
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
            self._check(fn(self._h, ref, workspace.data_ptr(), need, stream))
        else:  # (a refusal comes with its message)
            self._check(fn(self._h, ref, None, 0, stream))

    # ------------------------------------------------------------------
    def embedding(self, ids, table, *, scale=1.0, out=None):
        """out[i] = scale table[ids[i]]: [N, D] for ids [N] (int64) and table
        [V, D]; a row of zeros where ids[i] lies outside [0, V)."""
        V, D = table.shape
        N = ids.shape[0]
        if out is None:
            out = torch.empty(N, D, dtype=table.dtype, device=table.device)
        t = table.dtype
        self._call("nuts_embedding", _Embedding(
            _type(table, "table"), 0, N, V, D, _vector(ids, "ids", torch.int64, N), *_matrix(table, "table", t),
            scale, *_matrix(out, "out", t, N, D)), table.device)
        return out

    def embedding_grad(self, ids, dout, V, *, scale=1.0, out=None):
        """Gradient [V, D] of ``embedding``'s table for dout [N, D]: scale
        times the sum of dout over the positions of each token."""
        N, D = dout.shape
        if out is None:
            out = torch.empty(V, D, dtype=dout.dtype, device=dout.device)
        t = dout.dtype
        self._call("nuts_embedding_grad", _EmbeddingGrad(
            _type(dout, "dout"), 0, N, V, D, _vector(ids, "ids", torch.int64, N), *_matrix(dout, "dout", t),
            scale, *_matrix(out, "out", t, V, D)), dout.device)
        return out

    def linear(self, x, w, *, bias=None, act="none", residual=None, save=False, out=None):
        """act(x w^T + bias) + residual: [M, N] for x [M, K], w [N, K].  act is
        one of none, relu, sigmoid, silu, gelu.  out may be residual.  With
        save=True returns (y, pre): pre is x w^T + bias in fp32, which
        ``linear_grad`` reads (None with act="none": it needs none)."""
        (M, K), N, t = x.shape, w.shape[0], x.dtype
        if out is None:
            out = torch.empty(M, N, dtype=t, device=x.device)
        pre = None
        if save and act != "none":
            pre = torch.empty(M, N, dtype=torch.float32, device=x.device)
        r = (None, 0) if residual is None else _matrix(residual, "residual", t, M, N)
        self._call("nuts_linear", _Linear(
            _type(x, "x"), _act(act), M, N, K, *_matrix(x, "x", t), *_matrix(w, "w", t, N, K),
            None if bias is None else _vector(bias, "bias", t, N), *r, *_matrix(out, "out", t, M, N),
            None if pre is None else pre.data_ptr()), x.device)
        return (out, pre) if save else out

    def linear_grad(self, dy, x, w, *, act="none", pre=None, bias=True, dx=True, dw=True, rounded=False):
        """Gradients (dx [M, K], dw [N, K], dbias [N]) of ``linear`` for dy
        [M, N]; None where not asked for.  The residual's gradient is dy.  With
        bf16 and an activation, rounded=True rounds dy act'(z) to bf16 for the
        two products: half of their work, and 1.4 times the outputs' error."""
        (M, K), N, t = x.shape, w.shape[0], dy.dtype
        empty = lambda *shape: torch.empty(*shape, dtype=t, device=dy.device)  # noqa: E731
        gx, gw = empty(M, K) if dx else None, empty(N, K) if dw else None
        gb = empty(N) if bias else None
        code = _act(act) | (NUTS_ROUND_DZ if rounded else 0)
        if pre is not None:
            pre, _ = _matrix(pre, "pre", torch.float32, M, N) if pre.is_contiguous() else _refuse("pre")
        elif act != "none":
            raise ValueError("the gradient through an activation needs pre (linear(..., save=True))")
        self._call("nuts_linear_grad", _LinearGrad(
            _type(dy, "dy"), code, M, N, K, *_matrix(dy, "dy", t, M, N), *_matrix(x, "x", t), *_matrix(w, "w", t, N, K),
            pre, *((None, 0) if gx is None else (gx.data_ptr(), K)), *((None, 0) if gw is None else (gw.data_ptr(), K)),
            None if gb is None else gb.data_ptr()), dy.device)
        return gx, gw, gb

    def gated(self, x, wg, wu, *, act="silu", save=False, out=None):
        """act(x wg^T) * (x wu^T): [M, F] for x [M, K] and wg, wu [F, K], both
        products in one kernel.  With save=True returns (y, pre): pre [2, M, F]
        holds the two products in fp32, which ``gated_grad`` reads."""
        (M, K), F, t = x.shape, wg.shape[0], x.dtype
        if out is None:
            out = torch.empty(M, F, dtype=t, device=x.device)
        pre = torch.empty(2, M, F, dtype=torch.float32, device=x.device) if save else None
        self._call("nuts_gated", _Gated(
            _type(x, "x"), _act(act), M, F, K, *_matrix(x, "x", t), *_matrix(wg, "wg", t, F, K),
            *_matrix(wu, "wu", t, F, K), *_matrix(out, "out", t, M, F), None if pre is None else pre.data_ptr()),
            x.device)
        return (out, pre) if save else out

    def gated_grad(self, dy, x, wg, wu, pre, *, act="silu", dx=True, dw=True, rounded=False):
        """Gradients (dx [M, K], dwg [F, K], dwu [F, K]) of ``gated`` for dy
        [M, F]; None where not asked for.  With bf16, rounded=True rounds the
        gradients of the two products' results to bf16: half of the work, and
        1.4 times the outputs' error."""
        (M, K), F, t = x.shape, wg.shape[0], dy.dtype
        empty = lambda *shape: torch.empty(*shape, dtype=t, device=dy.device)  # noqa: E731
        gx = empty(M, K) if dx else None
        gg, gu = (empty(F, K), empty(F, K)) if dw else (None, None)
        if pre.dtype != torch.float32 or tuple(pre.shape) != (2, M, F) or not pre.is_contiguous():
            _refuse("pre")
        at = lambda g: (None, 0) if g is None else (g.data_ptr(), K)  # noqa: E731
        self._call("nuts_gated_grad", _GatedGrad(
            _type(dy, "dy"), _act(act) | (NUTS_ROUND_DZ if rounded else 0), M, F, K, *_matrix(dy, "dy", t, M, F), *_matrix(x, "x", t),
            *_matrix(wg, "wg", t, F, K), *_matrix(wu, "wu", t, F, K), pre.data_ptr(), *at(gx), *at(gg), *at(gu)),
            dy.device)
        return gx, gg, gu

    def categorical(self, logits, targets, *, grad=False, scale=1.0, out=None):
        """Negative log-likelihood nll [M] (fp32) of targets [M] (int64) under
        softmax(logits [M, V]) by row.  With grad=True returns (nll, total,
        dlogits): their sum (a float64 scalar tensor) and scale times its
        gradient (out may be logits itself).  A target outside [0, V) marks a
        row without an observation: 0, and a zero gradient."""
        (M, V), t = logits.shape, logits.dtype
        nll = torch.empty(M, dtype=torch.float32, device=logits.device)
        total = None
        o = (None, 0)
        if grad:
            total = torch.empty((), dtype=torch.float64, device=logits.device)
            if out is None:
                out = torch.empty(M, V, dtype=t, device=logits.device)
            o = _matrix(out, "out", t, M, V)
        self._call("nuts_categorical", _Categorical(
            _type(logits, "logits"), 0, M, V, *_matrix(logits, "logits", t), _vector(targets, "targets", torch.int64, M),
            scale, nll.data_ptr(), None if total is None else total.data_ptr(), *o), logits.device)
        return (nll, total, out) if grad else nll


def _refuse(name):
    raise ValueError(f"{name} must be the contiguous float32 tensor that the forward call returned")
