"""The head's gradients with a factor on the device, without a GPU: what the C entry point and the binding refuse, before any launch."""
import os

import pytest
import torch

from paper_2502_04416_amd import binding
from test_training_operators_cpu import FIELDS, M


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return binding.load()


@pytest.mark.parametrize("factor,change,msg", [
    (30 * M + 2, {}, "factor is not aligned"), (6 * M + 4, {}, "dx overlaps factor"), (7 * M, {}, "dweight overlaps factor"), (20 * M + 64, {}, "workspace overlaps factor"),
    (30 * M, dict(x=0), "null"), (30 * M, dict(size=8), "version"),
])
def test_refusals(lib, factor, change, msg):
    packer = binding._HEAD_LOSS_BACKWARD
    args = dict(FIELDS["head_loss_backward"], size=packer.size)
    args.update(change)
    with pytest.raises(binding.CmoeError, match=msg):
        binding._check(lib.cmoe_head_loss_backward_scaled(packer.pack(*args.values()), factor, None), "cmoe_head_loss_backward_scaled")


def test_the_binding_refuses():
    x, w, ids, row = torch.zeros(4, 16), torch.zeros(24, 16), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    for scale, msg in ((torch.tensor(0.5), "HIP device"), (torch.tensor([0.5], dtype=torch.float64), "HIP device"), (torch.tensor(float("inf")), "finite")):
        with pytest.raises(binding.CmoeError, match=msg):
            binding.head_loss_backward(x, w, ids, row, dx=torch.zeros(4, 16), scale=scale)
