"""ctypes binding of the layer norm and of distillation into a linear head, in the manner of ``binding``: argument checks and marshalling only."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as b


def _teacher(index: torch.Tensor, teacher: torch.Tensor, teacher_lse: Optional[torch.Tensor], N: int):
    if index.dtype != torch.int64 or index.ndim != 2 or teacher.shape != index.shape or index.shape[0] != N:
        raise ValueError("index must be int64 [tokens, K], teacher of its shape")
    ip, ldi = b._mat(index, "index")
    tp, ldt = b._mat(teacher, "teacher")
    return ip, ldi, tp, b._dt(teacher), ldt, None if teacher_lse is None else b._tokens(teacher_lse, N, torch.float32, "teacher_lse")


def _distill_workspace(op: int, X: torch.Tensor, W: torch.Tensor, K: int, wp: int, ldw: int) -> torch.Tensor:
    op |= b.OP_F32 if X.dtype == torch.float32 else 0
    return b.velora_workspace_alloc(b.velora_workspace_bytes(op, X.shape[0], X.shape[1], W.shape[0], K, b._odd_rows(W, wp, ldw)), X.device)


def velora_head_distill(X: torch.Tensor, W: torch.Tensor, index: torch.Tensor, teacher: torch.Tensor, temperature: float = 1.0,
                        teacher_lse: Optional[torch.Tensor] = None, loss: Optional[torch.Tensor] = None,
                        lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Divergence of every token's distribution under the linear head W from a teacher's K likeliest columns ``index`` with logits ``teacher``
    (index < 0: no entry), without the student's logits: (loss, lse), both fp32 [N]."""
    if stream is not None and (loss is None or lse is None or ws is None):
        return b._on(stream, velora_head_distill, X, W, index, teacher, temperature, teacher_lse, loss, lse, ws)
    xp, ldx, wp, ldw = b._head(X, W)
    N, D = X.shape
    V = W.shape[0]
    lists = _teacher(index, teacher, teacher_lse, N)
    K = index.shape[1]
    if loss is None:
        loss = torch.empty(N, dtype=torch.float32, device=X.device)
    if lse is None:
        lse = torch.empty(N, dtype=torch.float32, device=X.device)
    lp, sp = b._tokens(loss, N, torch.float32, "loss"), b._tokens(lse, N, torch.float32, "lse")
    b._here(X, W, index, teacher, loss, lse, *([] if teacher_lse is None else [teacher_lse]))
    if ws is None:
        ws = _distill_workspace(b.OP_HEAD_DISTILL, X, W, K, wp, ldw)
    rc = b.lib().velora_head_distill(xp, ldx, wp, ldw, *lists, temperature, K, lp, sp, b._dt(X), N, D, V, *b._room(ws), b._stream(stream))
    b._check(rc, "velora_head_distill")
    return loss, lse


def velora_head_distill_backward(X: torch.Tensor, W: torch.Tensor, index: torch.Tensor, teacher: torch.Tensor, lse: torch.Tensor, dloss: torch.Tensor,
                                 temperature: float = 1.0, teacher_lse: Optional[torch.Tensor] = None, dX: Optional[torch.Tensor] = None,
                                 dW: Optional[torch.Tensor] = None, need_dX: bool = True, need_dW: bool = True, dw_dtype=None, beta: int = 0,
                                 ws: Optional[torch.Tensor] = None, stream=None):
    """(dX, dW) of velora_head_distill, given the gradient of every token's loss and the lse it returned."""
    if stream is not None and (ws is None or (need_dX and dX is None) or (need_dW and dW is None)):
        return b._on(stream, velora_head_distill_backward, X, W, index, teacher, lse, dloss, temperature, teacher_lse, dX, dW, need_dX, need_dW,
                   dw_dtype, beta, ws)
    xp, ldx, wp, ldw = b._head(X, W)
    N, D = X.shape
    V = W.shape[0]
    lists = _teacher(index, teacher, teacher_lse, N)
    K = index.shape[1]
    sp, gp = b._tokens(lse, N, torch.float32, "lse"), b._tokens(dloss, N, torch.float32, "dloss")
    if need_dX and dX is None:
        dX = torch.empty((N, D), dtype=X.dtype, device=X.device)
    if need_dW and dW is None:
        if beta:
            raise ValueError("beta = 1 adds to a dW that is passed in")
        dW = torch.empty((V, D), dtype=dw_dtype or X.dtype, device=X.device)
    if (need_dX and (dX.shape != X.shape or dX.dtype != X.dtype)) or (need_dW and dW.shape != W.shape):
        raise ValueError("dX must be like X, dW of W's shape")
    dxp, lddx = b._mat(dX, "dX") if need_dX else (None, D)
    dwp, lddw = b._mat(dW, "dW") if need_dW else (None, D)
    b._here(X, W, index, teacher, lse, dloss, *([] if teacher_lse is None else [teacher_lse]), *([dX] if need_dX else []), *([dW] if need_dW else []))
    if ws is None:
        ws = _distill_workspace(b.OP_HEAD_DISTILL_BACKWARD, X, W, K, wp, ldw)
    rc = b.lib().velora_head_distill_backward(xp, ldx, wp, ldw, *lists, temperature, K, sp, gp, dxp, lddx, dwp, b._dt(dW) if need_dW else b.F32, lddw, beta,
                                            b._dt(X), N, D, V, *b._room(ws), b._stream(stream))
    b._check(rc, "velora_head_distill_backward")
    return dX, dW


def _rows_like(t: torch.Tensor, X: torch.Tensor, name: str):
    """Address and pitch of a matrix like X."""
    if t.shape != X.shape or t.dtype != X.dtype:
        raise ValueError("%s must have the rows' shape and type" % name)
    return b._mat(t, name)


def _columns(t: torch.Tensor, D: int, name: str) -> int:
    if t.ndim != 1 or t.shape[0] != D or not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor with one element per column" % name)
    return t.data_ptr()


def velora_layer_norm(X: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                      residual: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None, H: Optional[torch.Tensor] = None,
                      mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None, stream=None):
    """Layer norm of the rows of H = X + residual (of X without one): (Y, H, mean, rstd), the last three for the backward pass.  H is X itself
    where nothing is added, and None where Y is written over it: then nothing is left for the backward pass."""
    if stream is not None and (Y is None or mean is None or rstd is None or (residual is not None and H is None)):
        return b._on(stream, velora_layer_norm, X, weight, bias, eps, residual, Y, H, mean, rstd)
    xp, ldx = b._mat(X, "X")
    N, D = X.shape
    given = [X]                                               # what is made here needs no look
    rp, ldr, hp, ldh, wp, bp, p_dtype = None, D, None, D, None, None, b.F32
    if residual is not None:
        rp, ldr = _rows_like(residual, X, "residual")
        given.append(residual)
        if H is None:
            H = torch.empty_like(X, memory_format=torch.contiguous_format)
            hp = H.data_ptr()
        else:
            hp, ldh = _rows_like(H, X, "H")
            given.append(H)
    elif H is None or H is X:
        H = X
    else:
        raise ValueError("H is X where nothing is added")
    if weight is not None:
        wp, p_dtype = _columns(weight, D, "weight"), b._dt(weight)
        given.append(weight)
    if bias is not None:
        if weight is not None and weight.dtype != bias.dtype:
            raise ValueError("weight and bias must have one type")
        bp, p_dtype = _columns(bias, D, "bias"), b._dt(bias)
        given.append(bias)
    if Y is None:
        Y = torch.empty_like(X, memory_format=torch.contiguous_format)
        yp, ldy = Y.data_ptr(), D
    else:
        yp, ldy = _rows_like(Y, X, "Y")
        given.append(Y)
        if residual is None and N and yp == xp:
            H = None
    if mean is None:
        mean = torch.empty(N, dtype=torch.float32, device=X.device)
        mp = mean.data_ptr()
    else:
        mp = b._tokens(mean, N, torch.float32, "mean")
        given.append(mean)
    if rstd is None:
        rstd = torch.empty(N, dtype=torch.float32, device=X.device)
        sp = rstd.data_ptr()
    else:
        sp = b._tokens(rstd, N, torch.float32, "rstd")
        given.append(rstd)
    b._here(*given)
    rc = b.lib().velora_layer_norm(xp, ldx, rp, ldr, wp, bp, p_dtype, eps, hp, ldh, yp, ldy, mp, sp, b._dt(X), N, D, b._stream(stream))
    b._check(rc, "velora_layer_norm")
    return Y, H, mean, rstd


def velora_layer_norm_backward(dY: torch.Tensor, H: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor] = None,
                               dH: Optional[torch.Tensor] = None, dX: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None,
                               dbias: Optional[torch.Tensor] = None, need_dX: bool = True, need_dweight: bool = True, need_dbias: bool = True,
                               dw_dtype=None, beta: int = 0, ws: Optional[torch.Tensor] = None, stream=None):
    """(dX, dweight, dbias) of velora_layer_norm, given what it returned and the gradients of Y and, where H went on to another layer, of H."""
    if stream is not None and ((need_dX and dX is None) or (need_dweight and dweight is None) or (need_dbias and dbias is None) or ws is None):
        return b._on(stream, velora_layer_norm_backward, dY, H, mean, rstd, weight, dH, dX, dweight, dbias, need_dX, need_dweight, need_dbias,
                     dw_dtype, beta, ws)
    if H is None:
        raise ValueError("H is None: velora_layer_norm wrote Y over it")
    hp, ldh = b._mat(H, "H")
    N, D = H.shape
    yp, lddy = _rows_like(dY, H, "dY")
    mp, sp = b._tokens(mean, N, torch.float32, "mean"), b._tokens(rstd, N, torch.float32, "rstd")
    given = [dY, H, mean, rstd]                               # what is made here needs no look
    wp, p_dtype, gp, lddh, xp, lddx, dwp, dbp = None, b.F32, None, D, None, D, None, None
    if weight is not None:
        wp, p_dtype = _columns(weight, D, "weight"), b._dt(weight)
        given.append(weight)
    if dH is not None:
        gp, lddh = _rows_like(dH, H, "dH")
        given.append(dH)
    if not need_dX:
        dX = None
    elif dX is None:
        dX = torch.empty_like(H, memory_format=torch.contiguous_format)
        xp = dX.data_ptr()
    else:
        xp, lddx = _rows_like(dX, H, "dX")
        given.append(dX)
    dweight, dbias = dweight if need_dweight else None, dbias if need_dbias else None
    if dweight is not None and dbias is not None and dweight.dtype != dbias.dtype:
        raise ValueError("dweight and dbias must have one type")
    if (need_dweight and dweight is None) or (need_dbias and dbias is None):
        if beta:
            raise ValueError("beta = 1 adds to a dweight and a dbias that are passed in")
        kind = dweight.dtype if dweight is not None else dbias.dtype if dbias is not None else dw_dtype or (torch.float32 if weight is None else weight.dtype)
    if need_dweight:
        if dweight is None:
            dweight = torch.empty(D, dtype=kind, device=H.device)
            dwp = dweight.data_ptr()
        else:
            dwp = _columns(dweight, D, "dweight")
            given.append(dweight)
    if need_dbias:
        if dbias is None:
            dbias = torch.empty(D, dtype=kind, device=H.device)
            dbp = dbias.data_ptr()
        else:
            dbp = _columns(dbias, D, "dbias")
            given.append(dbias)
    b._here(*given)
    sums, room = dweight if need_dweight else dbias, (None, 0)
    if ws is None and sums is not None:
        ws = b.velora_workspace_alloc(b.velora_workspace_bytes(b.OP_LAYER_NORM_BACKWARD, N, D, 1, 1, False), H.device)
    if ws is not None:
        room = b._room(ws)
    rc = b.lib().velora_layer_norm_backward(yp, lddy, hp, ldh, mp, sp, wp, p_dtype, gp, lddh, xp, lddx, dwp, dbp,
                                            b.F32 if sums is None else b._dt(sums), beta, b._dt(H), N, D, *room, b._stream(stream))
    b._check(rc, "velora_layer_norm_backward")
    return dX, dweight, dbias
