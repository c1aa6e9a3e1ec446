"""Dense products whose sums are long: weight gradients over millions of rows, products with K or N up to
2^20, where what an accumulator of the tensor cores cuts off, or a chain of fp32 sums rounds, adds up.

Numbers of one sign, so that every cut goes the same way, with columns of different scales, so that the
results lie anywhere between two bf16 numbers. u = 2^-24.
bf16: an accumulator takes 256 steps of 16 products, each off by 2 u of the sum at most; a chain of register
sums n u. The mean of the signed errors over n results, each rounded to bf16 (2^-8 at most, evenly spread:
2^-8 / sqrt(3) in the mean square), has a standard deviation of 2^-8 / sqrt(3 n), and four of them are given.
fp32: four steps of a k-slice add numbers of its size (2 u each), what the planes leave out is 4 u, joining
and rounding 3 u; rounding errors of a chain of n sums of like numbers have the root mean square
u / sqrt(3) sqrt(n / 3): chains of 256 k-slices, whose errors spread over m blocks, and of m.
"""
import math

import pytest
import torch

from paper_2604_01622_gb300.block import Linear
from tests.test_gpu_linear import _check_forward, _inputs

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _positive(rows, cols, dtype, seed, across=1):
    """rows x cols positive numbers; `across`: the dimension along which the scales differ."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.rand(rows, cols, device="cuda", generator=g)
    x += 0.5
    shape = (1, cols) if across else (rows, 1)
    x *= 0.5 + torch.rand(shape, device="cuda", generator=g)
    return x.to(DT[dtype])


def _exact(A, B_, step=1 << 18):
    """A^T B in 64 bits over the first dimension."""
    out = torch.zeros(A.shape[1], B_.shape[1], dtype=torch.float64, device="cuda")
    for i in range(0, A.shape[0], step):
        out += A[i:i + step].double().t() @ B_[i:i + step].double()
    return out


def _bf16_bias(got, want, slices):
    err = ((got.double() - want) / want).flatten()
    n = err.numel()
    tol = 256 * 2 * U + slices / 64 * U + 4 * 2.0 ** -8 / math.sqrt(3 * n)
    assert abs(float(err.mean())) <= tol, (float(err.mean()), tol)
    assert float(err.abs().max()) <= 1.01 * 2.0 ** -8 + tol


def _f32_rms(got, want, chain):
    err = ((got.double() - want) / want).flatten()
    m = max(chain / 256, 1)
    tol = (4 * 2 + 4 + 3) * U + U / math.sqrt(3) * (math.sqrt(256 / 3 / m) + math.sqrt(m / 3))
    rms = float(err.square().mean().sqrt())
    assert rms <= tol, (rms, tol)


@pytest.mark.parametrize("rows,K,N", [(2 ** 22 + 77, 64, 64), (300001, 2048, 1032)])
def test_bf16_weight_gradient_over_many_rows(rows, K, N):
    X, dY = _positive(rows, K, "bf16", 1), _positive(rows, N, "bf16", 2)
    W = _positive(K, N, "bf16", 3)
    lin = Linear(rows, K, N)
    g = lin.backward(dY, X, W)
    lin.check()
    cols = slice(0, min(N, 256))
    _bf16_bias(g["dW"][:, cols], _exact(X, dY[:, cols]), rows / 64 / (8 if K == 64 else 1))
    # beside it, dX and db
    pick = torch.arange(0, rows, rows // 50, device="cuda")
    want = dY[pick].double() @ W.double().t()
    assert (g["dX"][pick].double() - want).abs().le(want * (1.01 * 2.0 ** -8 + N * 2 * U)).all()
    want = _exact(dY, torch.ones(rows, 1, device="cuda"))[:, 0]
    assert (g["db"].double() - want).abs().le(want * (1.01 * 2.0 ** -8 + 1e-5)).all()


@pytest.mark.parametrize("form", ["forward", "dX"])
def test_bf16_products_with_a_long_inner_dimension(form):
    m, n, L = 1000, 1032, 2 ** 20
    A = _positive(m, L, "bf16", 4, across=0)
    if form == "forward":
        W = _positive(L, n, "bf16", 5)
        lin = Linear(m, L, n, train=False)
        got, _ = lin.forward(A, W)
        rows = W[:, :256]
    else:
        W = _positive(n, L, "bf16", 5, across=0)
        lin = Linear(m, n, L)
        X = torch.zeros(m, n, device="cuda", dtype=torch.bfloat16)
        got = lin.backward(A, X, W, need_dW=False, with_bias=False)["dX"]
        rows = W[:256].t()
    lin.check()
    want = torch.zeros(256, 256, dtype=torch.float64, device="cuda")
    for i in range(0, L, 1 << 16):
        want += A[:256, i:i + (1 << 16)].double() @ rows[i:i + (1 << 16)].double()
    _bf16_bias(got[:256, :256], want, L / 64)


def test_f32_weight_gradient_over_many_rows():
    rows, K, N = 2 ** 23, 32, 32
    X, dY = _positive(rows, K, "f32", 6), _positive(rows, N, "f32", 7)
    lin = Linear(rows, K, N, dtype="f32")
    g = lin.backward(dY, X, torch.zeros(K, N, device="cuda"), need_dX=False, with_bias=False)
    lin.check()
    _f32_rms(g["dW"], _exact(X, dY), rows / 64 / 4)


def test_f32_product_with_a_long_inner_dimension():
    m, K, N = 200, 2 ** 20, 68
    X, W = _positive(m, K, "f32", 8, across=0), _positive(K, N, "f32", 9)
    lin = Linear(m, K, N, dtype="f32", train=False)
    Y, _ = lin.forward(X, W)
    lin.check()
    want = torch.zeros(m, N, dtype=torch.float64, device="cuda")
    for i in range(0, K, 1 << 18):
        want += X[:, i:i + (1 << 18)].double() @ W[i:i + (1 << 18)].double()
    _f32_rms(Y, want, K / 64 / 4)


# both sides of the limits: 256 k-slices of fp32 in up to four blocks of K, 512 of bf16
@pytest.mark.parametrize("dtype,m,K,N", [("f32", 60, 16384, 36), ("f32", 60, 65536, 36),
                                         ("f32", 60, 65600, 36), ("f32", 300, 70004, 132),
                                         ("f32", 1500, 20004, 1032), ("bf16", 600, 33000, 520),
                                         ("bf16", 1100, 40000, 1032),
                                         ("bf16", 70, 524296, 72)])
def test_long_sums_with_the_whole_epilogue(dtype, m, K, N):
    t = _inputs(m, K, N, dtype, seed=K)
    lin = Linear(m, K, N, act="gelu", dtype=dtype)
    rng = torch.tensor([2 ** 50 + 3, 11], dtype=torch.int64, device="cuda")
    lin.set_dropout(0.1, rng, 5)
    Y, P = lin.forward(t["X"], t["W"], t["b"], t["R"])
    lin.check()
    _check_forward(t, "gelu", dtype, Y, P, (0.1, 2 ** 50 + 3, 11, 5))


@pytest.mark.parametrize("dtype,rows,K,N", [("bf16", 2 ** 22 + 333, 72, 136), ("f32", 70001, 68, 132),
                                            ("bf16", 270000, 1032, 2056), ("bf16", 32768, 1032, 2056),
                                            ("bf16", 32769, 1032, 2056), ("bf16", 32769, 264, 520),
                                            ("bf16", 600001, 264, 520), ("bf16", 50000, 8, 8)])
def test_weight_gradients_of_any_sign(dtype, rows, K, N):
    """Ragged sizes, against 64 bits: each step of a sum off by 2 u of the absolute sums, bf16 dP = dY."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    X, dY = (torch.randn(rows, c, device="cuda", generator=g).to(DT[dtype]) for c in (K, N))
    W = torch.randn(K, N, device="cuda", generator=g).to(DT[dtype])
    lin = Linear(rows, K, N, dtype=dtype)
    got = lin.backward(dY, X, W)
    again = lin.backward(dY, X, W)
    lin.check()
    assert all(torch.equal(got[k], again[k]) for k in got)
    want, size = _exact(X, dY), _exact(X.abs(), dY.abs())
    half = 2.0 ** -8 if dtype == "bf16" else U
    # bf16: an accumulator of up to 32768 rows, or 256 steps and a chain of sums
    steps = min(rows, 32768) / 16 + rows / 4096 if dtype == "bf16" else 40 + 256 + rows / 16384
    err = (got["dW"].double() - want).abs()
    assert (err <= 1.01 * half * want.abs() + steps * 2 * U * size).all()
    assert torch.isfinite(got["dX"].float()).all()


def test_the_bound_tells():
    """The tolerance above is below what one accumulator of all rows would lose: 1e-7 of the sum for every
    16 of K, as measured."""
    slices = (2 ** 22 + 77) / 64 / 8
    assert 256 * 2 * U + slices / 64 * U + 4 * 2.0 ** -8 / math.sqrt(3 * 64 * 64) < 0.1 * 1e-7 * slices * 4
