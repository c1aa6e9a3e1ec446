"""Balance-loss calls whose outputs lie in their inputs are refused on the host, before any launch."""
import pytest
import torch

import paper_2604_01622_gb300 as ec
from paper_2604_01622_gb300.block import BalanceLoss

pytestmark = pytest.mark.gpu


def test_loss_and_counts_in_an_input_or_in_each_other():
    N, E, k = 96, 8, 2
    S = torch.softmax(torch.randn(N, E, device="cuda"), 1)
    choice = torch.topk(S, k, 1).indices.int()
    mask = torch.ones(N, dtype=torch.uint8, device="cuda")
    out = torch.zeros(256, dtype=torch.int32, device="cuda")
    h = BalanceLoss(N, E, k, [0, 32, N])
    s, c, m, o = (t.data_ptr() for t in (S, choice, mask, out))
    st = torch.cuda.current_stream().cuda_stream
    before = [t.clone() for t in (S, choice, mask, out)]
    launches = h.launches
    for loss, count in ((s, o), (s + 4 * (N * E - 1), o), (c + 4 * (N * k - 1), o), (m + N - 4, o),
                        (o, s + 4), (o, c - 4 * 2 * E + 4), (o, m), (o + 8, o), (o + 4 * (2 * E - 1), o)):
        with pytest.raises(ec.ECError) as e:
            ec.ec_balance_forward(h.ctx, s, c, m, loss, count, st)
        assert e.value.status == ec.EC_ERR_INVALID_ARG
    assert h.launches == launches
    assert all(torch.equal(a, b) for a, b in zip(before, (S, choice, mask, out)))
    # next to each other they are taken
    ec.ec_balance_forward(h.ctx, s, c, m, o + 4 * 2 * E, o, st)
    h.check()
    loss, count = h.forward(S, choice, mask)
    assert torch.equal(out[:2 * E].view(2, E), count)
    assert torch.equal(out[2 * E:2 * E + 1].view(torch.float32), loss)
