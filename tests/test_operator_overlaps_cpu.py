"""Which buffers of a call of the operators may be the same: refusals, none of which reaches a launch."""
import pytest

from paper_2502_04416_amd import binding
from test_operators_cpu import _adapter_args, _norm_args, _norm_backward_args, lib  # noqa: F401


def refused(entry, args, msg):
    with pytest.raises(binding.CmoeError, match=msg):
        binding._check(entry(args, None), entry.__name__)


@pytest.mark.parametrize("change,msg", [
    # of one size, but read by every row, or by others than who writes them
    (dict(rows=16, weight=3 << 20, mean=3 << 20), "mean overlaps weight"), (dict(rows=16, weight=3 << 20, rstd=3 << 20), "rstd overlaps weight"),
    (dict(rows=16, bias=3 << 20, mean=3 << 20), "mean overlaps bias"), (dict(rows=16, bias=3 << 20, rstd=3 << 20), "rstd overlaps bias"),
    (dict(rows=1, weight=3 << 20, sum_out=3 << 20), "sum_out overlaps weight"), (dict(rows=1, bias=3 << 20, sum_out=3 << 20), "sum_out overlaps bias"),
    (dict(rows=16, cols=1, rstd=1 << 20), "rstd overlaps x"),
])
def test_norm_forward_refuses_what_is_no_batch_in_place(lib, change, msg):  # noqa: F811
    refused(lib.cmoe_norm_forward, _norm_args(**change), msg)


@pytest.mark.parametrize("change,msg", [
    (dict(workspace=1 << 20), "workspace overlaps dy"), (dict(workspace=2 << 20), "workspace overlaps s"),
    (dict(workspace=8 << 20, dsum=8 << 20), "workspace overlaps dsum"), (dict(workspace=7 << 20, weight=7 << 20, rows=64), "workspace overlaps weight"),
    (dict(workspace=7 << 20, dweight=3 << 20, rows=16), "dweight overlaps mean"),
])
def test_norm_backward_refuses_what_is_no_batch_in_place(lib, change, msg):  # noqa: F811
    # (a workspace of a batch's very size)
    refused(lib.cmoe_norm_backward, _norm_backward_args(**{**dict(dweight=6 << 20, rows=64, workspace_bytes=64 * 16 * 4), **change}), msg)


@pytest.mark.parametrize("change,msg", [
    (dict(u=6 << 24), "u overlaps base"), (dict(u=(6 << 24) + 64), "u overlaps base"), (dict(u=6 << 24, rank=32, d_out=32), "u overlaps base"),
    (dict(y=6 << 24, x=6 << 24, d_in=64), "y overlaps x"),
])
def test_adapters_forward_refuses_outputs_over_the_base(lib, change, msg):  # noqa: F811
    refused(lib.cmoe_adapters_forward, _adapter_args(True, **change), msg)


@pytest.mark.parametrize("change,msg", [
    (dict(da=8 << 24), "da overlaps dx_base"), (dict(db=(8 << 24) + 128), "db overlaps dx_base"), (dict(workspace=8 << 24), "workspace overlaps dx_base"),
    (dict(workspace=(8 << 24) - (1 << 21)), "workspace overlaps dx_base"), (dict(dx=8 << 24, x=8 << 24), "dx overlaps x"),
])
def test_adapters_backward_refuses_outputs_over_the_base(lib, change, msg):  # noqa: F811
    refused(lib.cmoe_adapters_backward, _adapter_args(False, **change), msg)
