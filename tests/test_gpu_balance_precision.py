"""The logit gradient of a balance loss whose counts are nearly equal: the small difference of nearly equal
numbers keeps fp32's precision.

With h = f0 + h' (f0 the mean over the experts) the gradient is dloss S (h' - <S, h'> + f0 (1 - sum S)).
Tolerance: h' has three roundings; a term of <S, h'> passes at most 16 sums of a lane, 5 of the lanes and
the last three, each 2^-24 of max|h'|; f0 (1 - sum S) is held with the scores' parts below 2^-22, E
numbers of 2^-23 at most which add up with a relative error of E 2^-24, so to f0 E^2 2^-47, and 2 roundings
of its own, and |1 - sum S| is at most E 2^-24: in all |dloss| S (32 2^-24 max|h'| + 4 E^2 2^-48 f0). A sum that is
rounded to fp32 would err by about 2^-24 f0, several times that.
"""
import numpy as np
import pytest
import torch

from oracle import block as B
from paper_2604_01622_gb300.block import BalanceLoss
from tests._util import host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E,k", [(8, 2), (33, 3), (60, 4), (64, 8), (130, 5), (255, 2), (256, 8), (509, 4)])
def test_nearly_equal_counts(E, k):
    # as many tokens as keep the counts near 500: one choice more or less is 0.2% of them
    N = (500 * E + k - 1) // k
    g = torch.Generator(device="cuda").manual_seed(E)
    S = torch.softmax(1.5 * torch.randn(N, E, device="cuda", generator=g), 1)
    pair = torch.arange(N * k, device="cuda").view(N, k)
    choice = (pair % E).int()
    choice[0, 0] = (choice[0, 0] + 1) % E
    h = BalanceLoss(N, E, k)
    h.forward(S, choice)
    dZ = host(h.backward(S))
    s = host(S)
    _, _, hh = B.balance(s, choice.cpu().numpy(), None, [0, N])
    want = B.balance_grad(s, None, [0, N], hh)
    f0 = hh.mean()
    small = np.abs(hh - f0).max()
    tol = s * (32 * 2.0 ** -24 * small + 4 * E * E * 2.0 ** -48 * f0)
    assert 5 * tol.max() < s.max() * 2.0 ** -24 * f0    # a rounded sum would show
    bad = ~(np.abs(dZ - want) <= tol)
    assert not bad.any(), (int(bad.sum()), float((np.abs(dZ - want) / tol).max()))


def test_scores_of_any_sum():
    """The gradient is that of the definition for scores that are no softmax."""
    N, E, k = 300, 40, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    S = torch.rand(N, E, device="cuda", generator=g) * 3
    choice = torch.topk(S, k, 1).indices.int()
    h = BalanceLoss(N, E, k, [0, 100, N])
    h.forward(S, choice)
    s = host(S)
    _, _, hh = B.balance(s, choice.cpu().numpy(), None, [0, 100, N])
    want = B.balance_grad(s, None, [0, 100, N], hh)
    # sums of E products of at most 3 max|h|, and a dozen roundings
    hmax = np.repeat(np.abs(hh).max(1), [100, 200])[:, None]
    tol = s * hmax * 2.0 ** -24 * (2 * E + 16) * (s.sum(1, keepdims=True) + 2)
    assert (np.abs(host(h.backward(S)) - want) <= tol).all()
