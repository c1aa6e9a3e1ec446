"""Sizes, offsets and dropout sites that do not fit the 32 bits the library takes them in are refused, not
cut off (CPU: the addresses are never followed)."""
import os

import numpy as np
import pytest
import torch

import paper_2604_01622_gb300 as ec
from paper_2604_01622_gb300 import block
from paper_2604_01622_gb300 import build as B

ADDR = [0x10000000 + i * 0x1000000 for i in range(6)]
WRAP = 1 << 32


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ec.LIB_PATH):
        B.build()
    return ec.load()


@pytest.mark.parametrize("args", [(WRAP + 64, 64, 64), (64, WRAP + 64, 64), (64, 64, WRAP + 64),
                                  (64 - WRAP, 64, 64)])
def test_dense_product_sizes(args):
    with pytest.raises(ValueError, match="is not in"):
        ec.ec_linear_ctx_create(*args, 0, ec.EC_BF16)


def test_dense_product_rows_of_a_call():
    c = ec.ec_linear_ctx_create(64, 64, 64, 0, ec.EC_BF16)
    with pytest.raises(ValueError, match="rows"):
        ec.ec_linear_forward(c, WRAP + 4, *ADDR[:3], None, None, ADDR[3], None)
    with pytest.raises(ValueError, match="rows"):
        ec.ec_linear_backward(c, WRAP + 4, *ADDR[:3], None, ADDR[3], None, None, None)
    ec.ec_ctx_destroy(c)


@pytest.mark.parametrize("args", [(WRAP + 256, 8, 2, [0, 256]), (256, WRAP + 8, 2, [0, 256]),
                                  (256, 8, WRAP + 2, [0, 256]),
                                  (256, 8, 2, np.array([0, WRAP + 256])),
                                  (256, 8, 2, np.array([-WRAP, 256])),
                                  (256, 8, 2, torch.tensor([0, WRAP + 256]))])
def test_balance_sizes_and_offsets(args):
    with pytest.raises(ValueError, match="is not in"):
        ec.ec_balance_ctx_create(*args)


def test_offsets_that_fit_are_taken_in_any_form():
    for off in ([0, 256], (0, 100, 256), np.array([0, 256]), np.array([0, 256], np.int16),
                torch.tensor([0, 256])):
        ec.ec_ctx_destroy(ec.ec_balance_ctx_create(256, 8, 2, off))


@pytest.mark.parametrize("site", [-1, WRAP, WRAP + 3])
def test_dropout_sites(site):
    c = ec.ec_linear_ctx_create(64, 64, 64, 0, ec.EC_BF16)
    with pytest.raises(ValueError, match="site"):
        ec.ec_ctx_set_dropout(c, 0.1, ADDR[0], site)
    with pytest.raises(ValueError, match="site"):
        ec.ec_dropout(ec.EC_BF16, 64, *ADDR[:3], 0.1, ADDR[3], site, None)
    with pytest.raises(ValueError, match="site"):
        block.dropout(torch.zeros(8), 0.1, torch.zeros(2, dtype=torch.int64), site=site)
    ec.ec_ctx_set_dropout(c, 0.1, ADDR[0], WRAP - 1)
    ec.ec_ctx_destroy(c)
