"""What a context is left with when attaching its workspace fails (CPU: there is no device to attach it on)."""
import os

import pytest
import torch

import paper_2604_01622_gb300 as ec
from paper_2604_01622_gb300 import build as B
from paper_2604_01622_gb300 import layer as layer_mod

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


def test_dropout_whose_workspace_could_not_be_allocated_may_be_set_again(monkeypatch):
    """The larger workspace of the first dropout fails to be allocated once: the old one has been given
    back by then, and the next set_dropout attaches one."""
    attached, alive = [], []

    class Layer(layer_mod.Context):
        def __init__(self):
            self.device, self.code, self.tdtype = torch.device("cpu"), ec.EC_BF16, torch.bfloat16
            self.ctx = ec.ec_linear_ctx_create(64, 64, 64, 0, ec.EC_BF16)
            self._attach()

    class Stream:
        def synchronize(self):
            pass

    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream())
    monkeypatch.setattr(layer_mod, "ec_ctx_set_workspace", lambda c, p, n: attached.append(n))
    lay = Layer()
    assert attached == [lay.ws_bytes]
    rng = torch.zeros(2, dtype=torch.int64)
    empty = torch.empty

    def fails(*a, **kw):
        alive.append(lay.ws is not None)
        raise torch.OutOfMemoryError("no memory")

    monkeypatch.setattr(torch, "empty", fails)
    with pytest.raises(torch.OutOfMemoryError):
        lay.set_dropout(0.1, rng)
    monkeypatch.setattr(torch, "empty", empty)
    assert alive == [False] and len(attached) == 1
    lay.set_dropout(0.1, rng)
    assert len(attached) == 2 and attached[1] == lay.ws_bytes == ec.ec_workspace_bytes(lay.ctx)
    assert lay.ws.numel() == lay.ws_bytes > attached[0]
    lay.set_dropout(0.2, rng)
    assert len(attached) == 2
