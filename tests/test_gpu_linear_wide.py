"""fp32 dense products of few rows over wide weights (above 2^20 elements: their planes at full size), and
operands near the smallest numbers. Tolerances: tests/test_gpu_linear.py."""
import pytest
import torch

from paper_2604_01622_gb300.block import Linear
from tests.test_gpu_linear import U, _both

pytestmark = pytest.mark.gpu


# the last rows of the row kernel, the first of the tiles, several of its row counts; ragged columns
@pytest.mark.parametrize("m", [1, 7, 16, 17, 24, 64, 130])
@pytest.mark.parametrize("K,N", [(1032, 4100), (4100, 1028), (520, 8196)])
def test_few_rows(m, K, N):
    _both(m, K, N, "f32", ("gelu", "silu")[m % 2], p=0.1 if m % 3 == 0 else 0.0, bias=m != 17, res=m > 16)


@pytest.mark.parametrize("m", [4, 64])
@pytest.mark.parametrize("e", [-100, -112, -116, -120, -125])
def test_operands_near_the_smallest_numbers(m, e):
    """An operand's last bf16 part is a multiple of 2^-133, so half of that may be left out of it, beside
    the planes' 4 u and the sums' 2 K u of the absolute sums."""
    g = torch.Generator(device="cuda").manual_seed(m)
    X, W = ((torch.randn(s, device="cuda", generator=g).double() * 2.0 ** x).float()
            for s, x in (((m, 64), e), ((64, 64), 90)))
    lin = Linear(m, 64, 64, dtype="f32")
    Y, _ = lin.forward(X, W)
    lin.check()
    a, b = X.double(), W.double()
    tol = (2 * 64 + 4 + 2) * U * (a.abs() @ b.abs()) + 2.0 ** -134 * b.abs().sum(0)
    assert ((Y.double() - a @ b).abs() <= tol).all()
