"""The first dropout of a layer gives it a larger workspace: what calls have left in the old one stays in
force."""
import numpy as np
import pytest
import torch

import paper_2604_01622_gb300 as ec
from oracle import ecmoe as O
from paper_2604_01622_gb300 import inputs as I
from paper_2604_01622_gb300.layer import ECMoELayer
from tests._util import dev, host

pytestmark = pytest.mark.gpu


def _layer(dtype):
    w = (I.scaled(I.WORKLOADS["tiny_f32"], G=4, L=96, d=64, E=8, d_ff=64, k_base=12) if dtype == "f32"
         else I.scaled(I.WORKLOADS["ec_d2048_e64"], G=4, L=96, d=128, E=8, d_ff=64, k_base=12))
    inp = I.make_inputs(w)
    L = inp.layers[0]
    lay = ECMoELayer(w.N, w.d, w.E, w.d_ff, inp.group_off, inp.k_g, dtype=w.dtype)
    return lay, inp, (dev(inp.X), dev(L.Wr), None, dev(L.Wg), dev(L.Wu), dev(L.Wd))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_capacities_set_on_the_device_stay(dtype):
    lay, inp, args = _layer(dtype)
    k_g = np.asarray(inp.k_g, np.int32) + np.array([5, -5, -7, 7], np.int32)
    lay.set_capacity_async(torch.from_numpy(k_g).cuda())
    rng = torch.tensor([1, 2], dtype=torch.int64, device="cuda")
    lay.set_dropout(0.25, rng)
    _, idx, _, S = lay.forward(*args)
    lay.check()
    want, _ = O.ec_select(host(S).T, inp.group_off, k_g)
    assert np.array_equal(idx.cpu().numpy(), want)
    # those set on the host afterwards count again
    lay.set_capacity(inp.k_g)
    _, idx, _, S = lay.forward(*args)
    want, _ = O.ec_select(host(S).T, inp.group_off, inp.k_g)
    assert np.array_equal(idx.cpu().numpy(), want)


def test_a_status_that_nobody_has_read_stays():
    lay, inp, args = _layer("bf16")
    bad = np.asarray(inp.k_g, np.int32) + np.array([1, 0, 0, 0], np.int32)   # another sum
    lay.set_capacity_async(torch.from_numpy(bad).cuda())
    lay.set_dropout(0.25, torch.tensor([1, 2], dtype=torch.int64, device="cuda"))
    with pytest.raises(ec.ECError) as e:
        lay.check()
    assert e.value.status == ec.EC_ERR_SHAPE
    lay.check()                          # reported once
    _, idx, _, S = lay.forward(*args)
    lay.check()
    want, _ = O.ec_select(host(S).T, inp.group_off, inp.k_g)
    assert np.array_equal(idx.cpu().numpy(), want)
