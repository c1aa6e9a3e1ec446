"""The operators around the experts of a block (argument marshalling only): dropout with a residual, the
balance loss of a router, the dense product with its epilogue.

Every step runs in libecmoe.so; include/ecmoe.h has the definitions. Tensors are contiguous and on the
context's device. Calls run on the current stream of the current device; given another stream they make
it the current one, so that the tensors they allocate belong to it.
"""
from __future__ import annotations

import torch

from . import (EC_ACTIVATIONS, EC_OK, ECError, _check, check_site, ec_balance_ctx_create,
               ec_linear_ctx_create, load)
from .layer import _DT, Context, check_tensor

_CODE = {t: code for code, t in _DT.values()}


def _stream_on(dev):
    """Handle of the current stream. Launches go to the current device, so tensors of another one are
    refused. (Device and stream are asked for without torch.cuda's wrappers: 1.5 us of a call's host
    time.)"""
    cur = torch._C._cuda_getDevice()
    if cur != dev.index:
        raise ValueError(f"tensors on {dev}, but the current device is {cur}")
    return torch._C._cuda_getCurrentRawStream(cur)


def _ptr(t):
    return None if t is None else t.data_ptr()


def dropout(X, p, rng, site=0, R=None, Y=None, stream=None):
    """Y = R + drop(X) (R None: 0), elements counted along X. X bf16 or f32 of any shape; R and Y like X,
    each may be X itself. rng: int64 device tensor {seed, step}. The gradient with respect to X is the
    same call on dY without R."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return dropout(X, p, rng, site, R, Y)
    check_site(site)
    dev = X.device
    if X.dtype not in _CODE or not X.is_contiguous() or dev.type != "cuda":
        raise ValueError(f"X: a contiguous bf16 or f32 CUDA tensor is wanted, got {X.dtype} on {dev}, "
                         f"strides {X.stride()}")
    check_tensor("rng", rng, (2,), torch.int64, dev)
    if R is not None:
        check_tensor("R", R, X.shape, X.dtype, dev)
    if Y is None:
        Y = torch.empty_like(X)
    else:
        check_tensor("Y", Y, X.shape, X.dtype, dev)
    st, n = _stream_on(dev), X.numel()
    if n:
        status = load().ec_dropout(_CODE[X.dtype], n, X.data_ptr(), _ptr(R), Y.data_ptr(), p,
                                   rng.data_ptr(), site, st)
        if status != EC_OK:
            raise ECError(status, "ec_dropout rejected the call")
    return Y


class BalanceLoss(Context):
    """Balance loss over N tokens in sequences `group_off` (None: one), E experts, k choices a token."""

    def __init__(self, N, E, k, group_off=None, device="cuda"):
        self.N, self.E, self.k = int(N), int(E), int(k)
        group_off = [0, self.N] if group_off is None else group_off
        self.G = len(group_off) - 1
        self.device = torch.device(device)
        self.ctx = ec_balance_ctx_create(self.N, self.E, self.k, group_off)
        self._attach()

    def forward(self, S, choice, mask=None, stream=None):
        """S [N][E] f32 scores, choice [N][k] int32, mask [N] uint8 (0: token left out). Returns (loss [1]
        f32, count [G][E] int32)."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.forward(S, choice, mask)
        dev = self.device
        check_tensor("S", S, (self.N, self.E), torch.float32, dev)
        check_tensor("choice", choice, (self.N, self.k), torch.int32, dev)
        if mask is not None:
            check_tensor("mask", mask, (self.N,), torch.uint8, dev)
        loss = torch.empty(1, dtype=torch.float32, device=dev)
        count = torch.empty((self.G, self.E), dtype=torch.int32, device=dev)
        st = _stream_on(dev)
        if self.N:
            _check(self.ctx, load().ec_balance_forward(self.ctx, S.data_ptr(), choice.data_ptr(),
                                                       _ptr(mask), loss.data_ptr(), count.data_ptr(),
                                                       st))
        else:   # torch gives empty tensors no address, and the answer is zeros
            loss.zero_()
            count.zero_()
        return loss, count

    def backward(self, S, mask=None, dloss=None, dZ=None, stream=None):
        """Gradient of dloss * loss (dloss [1] f32, None: 1) of the last forward with respect to the
        logits behind S, which is passed again with its mask."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.backward(S, mask, dloss, dZ)
        dev = self.device
        check_tensor("S", S, (self.N, self.E), torch.float32, dev)
        if mask is not None:
            check_tensor("mask", mask, (self.N,), torch.uint8, dev)
        if dloss is not None:
            check_tensor("dloss", dloss, (1,), torch.float32, dev)
        if dZ is None:
            dZ = torch.empty((self.N, self.E), dtype=torch.float32, device=dev)
        else:
            check_tensor("dZ", dZ, (self.N, self.E), torch.float32, dev)
        st = _stream_on(dev)
        if self.N:
            _check(self.ctx, load().ec_balance_backward(self.ctx, S.data_ptr(), _ptr(mask), _ptr(dloss),
                                                        dZ.data_ptr(), st))
        return dZ


class Linear(Context):
    """Y = R + drop(act(X W + b)) for up to `rows` rows and W [K][N]; act "none", "relu", "gelu" (tanh
    form) or "silu". train=False leaves out the workspace of backward()."""

    def __init__(self, rows, K, N, act="none", dtype="bf16", train=True, device="cuda"):
        self.rows, self.K, self.N, self.act = int(rows), int(K), int(N), act
        self.train = bool(train)
        self.code, self.tdtype = _DT[dtype]
        self.device = torch.device(device)
        self.ctx = ec_linear_ctx_create(self.rows, self.K, self.N, EC_ACTIVATIONS[act], self.code,
                                        self.train)
        self._attach()

    def _rows(self, X):
        m = X.shape[0]
        if m > self.rows:
            raise ValueError(f"{m} rows: the context has room for {self.rows}")
        return m

    def forward(self, X, W, b=None, R=None, save=None, Y=None, P=None, stream=None):
        """X [m][K], W [K][N], b [N], R [m][N]. Returns (Y [m][N], P): P is the pre-activation that
        backward() needs, or None with save=False (default: save where the context trains) and where
        there is no activation."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.forward(X, W, b, R, save, Y, P)
        m, dt, dev = self._rows(X), self.tdtype, self.device
        check_tensor("X", X, (m, self.K), dt, dev)
        check_tensor("W", W, (self.K, self.N), dt, dev)
        if b is not None:
            check_tensor("b", b, (self.N,), dt, dev)
        if R is not None:
            check_tensor("R", R, (m, self.N), dt, dev)
        if Y is None:
            Y = torch.empty((m, self.N), dtype=dt, device=dev)
        else:
            check_tensor("Y", Y, (m, self.N), dt, dev)
        if P is not None:
            check_tensor("P", P, (m, self.N), dt, dev)
        elif (self.train if save is None else save) and self.act != "none":
            P = torch.empty((m, self.N), dtype=dt, device=dev)
        _check(self.ctx, load().ec_linear_forward(self.ctx, m, X.data_ptr(), W.data_ptr(), _ptr(b),
                                                  _ptr(R), _ptr(P), Y.data_ptr(),
                                                  _stream_on(dev)))
        return Y, P

    def backward(self, dY, X, W, P=None, need_dX=True, need_dW=True, with_bias=True, stream=None):
        """Gradients of <dY, Y>: a dict of dX, dW and db in the layer's dtype (None where not asked
        for). The residual's gradient is dY itself."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.backward(dY, X, W, P, need_dX, need_dW, with_bias)
        m, dt, dev = self._rows(dY), self.tdtype, self.device
        check_tensor("dY", dY, (m, self.N), dt, dev)
        check_tensor("X", X, (m, self.K), dt, dev)
        check_tensor("W", W, (self.K, self.N), dt, dev)
        if P is not None:
            check_tensor("P", P, (m, self.N), dt, dev)
        elif self.act != "none" and m:
            raise ValueError("P is wanted: the pre-activation that forward() returns with save=True")
        g = {"dX": torch.empty((m, self.K), dtype=dt, device=dev) if need_dX else None,
             "dW": torch.empty((self.K, self.N), dtype=dt, device=dev) if need_dW else None,
             "db": torch.empty(self.N, dtype=dt, device=dev) if with_bias else None}
        _check(self.ctx, load().ec_linear_backward(self.ctx, m, dY.data_ptr(), X.data_ptr(), W.data_ptr(),
                                                   _ptr(P), _ptr(g["dX"]), _ptr(g["dW"]), _ptr(g["db"]),
                                                   _stream_on(dev)))
        return g
