"""What a context is left with when attaching its workspace fails (CPU: there is no device to attach it on)."""
import os

import pytest
import torch

import paper_2604_01622_gb300 as ec
from paper_2604_01622_gb300 import build as B

ADDR = [0x10000000 + i * 0x1000000 for i in range(4)]   # made-up aligned addresses, far apart


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ec.LIB_PATH):
        B.build()
    return ec.load()


@pytest.mark.skipif(torch.cuda.is_available(), reason="the address must not reach a device")
def test_a_workspace_that_was_not_prepared_is_not_attached():
    """The kernels follow tables and count tickets that attaching writes into the workspace: where that
    failed, a call must find none attached."""
    bal = ec.ec_balance_ctx_create(256, 8, 2, [0, 256])
    lin = ec.ec_linear_ctx_create(64, 64, 64, 0, ec.EC_BF16)
    moe = ec.ec_ctx_create(256, 64, 8, 128, 1, [0, 256], [16], ec.EC_BF16)
    for c in (bal, lin, moe):
        with pytest.raises(ec.ECError) as e:
            ec.ec_ctx_set_workspace(c, 0x40000000, ec.ec_workspace_bytes(c))
        assert e.value.status == ec.EC_ERR_CUDA
    for call in (lambda: ec.ec_balance_forward(bal, ADDR[0], ADDR[1], None, ADDR[2], None, None),
                 lambda: ec.ec_linear_forward(lin, 4, *ADDR[:3], None, None, ADDR[3], None),
                 lambda: ec.ec_route(moe, ADDR[0], ADDR[1], None, None, None, ADDR[2], ADDR[3], None)):
        with pytest.raises(ec.ECError) as e:
            call()
        assert e.value.status == ec.EC_ERR_WORKSPACE
    for c in (bal, lin, moe):
        ec.ec_ctx_destroy(c)
