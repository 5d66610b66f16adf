"""The operators around the feed-forward layer without a GPU: the oracle's generator against published values, the argument
structs against the header's, and every refusal of the binding and of the C entry points (none of which reaches a launch)."""
import re
import os
import subprocess

import numpy as np
import pytest
import torch

import operator_oracle as O
from paper_2502_04416_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return binding.load()


@pytest.mark.parametrize("counter,key,words", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
])
def test_oracle_generator_gives_the_published_values(counter, key, words):
    assert tuple(int(w) for w in O.philox(counter, key)) == words


def test_oracle_mask_keeps_the_share_it_says():
    m = O.mask(300, 1003, binding.Dropout(0.3, 12345, 7))
    share = float((m == 0).double().mean())
    assert abs(share - 0.3) < 5 * (0.21 / m.numel()) ** 0.5 + 2.0 ** -17
    assert set(np.unique(m.numpy())) == {0.0, 65536 / (65536 - round(0.3 * 65536))}


def test_structs_have_the_sizes_of_the_header(lib, tmp_path):
    names = ("norm_forward", "norm_backward", "adapters_forward", "adapters_backward")
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "cmoe.h"\nint main(void) { printf("%s\\n", %s); return 0; }' % (
        " ".join(["%zu"] * 4), ", ".join("sizeof(cmoe_%s_args)" % n for n in names)))
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    sizes = [int(v) for v in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()]
    assert sizes == [getattr(binding, "_%s" % n.upper()).size for n in names]


def test_structs_have_the_order_of_the_header():
    """A 64-bit word per pointer, then counts and doubles, then 32-bit words: as the header declares them."""
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cmoe.h")).read(), flags=re.S)
    code = {"int64_t": "q", "uint64_t": "Q", "double": "d", "int32_t": "i", "float": "f"}
    for name in ("norm_forward", "norm_backward", "adapters_forward", "adapters_backward"):
        body = re.search(r"typedef struct \{([^}]*)\} cmoe_%s_args;" % name, header).group(1)
        fields = ""
        for line in filter(None, (l.strip() for l in body.split(";"))):
            kind, rest = re.match(r"(?:const )?(\w+)\s*(.*)", line, flags=re.S).groups()
            fields += "".join("Q" if "*" in part else code[kind] for part in rest.split(","))
        packed = re.sub(r"(\d+)(\w)", lambda m: m.group(2) * int(m.group(1)), getattr(binding, "_%s" % name.upper()).format[1:])
        assert fields == packed, name


def _norm_args(**kw):
    f = dict(x=1 << 20, residual=0, sum_out=0, y=2 << 20, weight=0, bias=0, mean=0, rstd=0, rows=4, p=0.0, seed=0, offset=0,
             size=binding._NORM_FORWARD.size, dtype=0, form=0, cols=16, eps=1e-5, reserved=0)
    f.update(kw)
    return binding._NORM_FORWARD.pack(*f.values())


@pytest.mark.parametrize("change,msg", [
    (dict(size=8), "version"), (dict(dtype=2), "dtype"), (dict(form=2), "form"), (dict(cols=0), "cols"), (dict(cols=32769), "cols"),
    (dict(rows=-1), "rows"), (dict(rows=1 << 40), "rows"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps"), (dict(p=-0.1), "rate"), (dict(p=1.01), "rate"), (dict(p=float("nan")), "rate"), (dict(x=0), "null"), (dict(y=0), "null"),
    (dict(x=(1 << 20) + 2), "aligned"), (dict(y=(1 << 20) + 64), "y overlaps x"), (dict(sum_out=2 << 20), "overlaps"),
    (dict(rstd=(2 << 20) + 4), "overlaps"), (dict(residual=(2 << 20) - 4), "overlaps"),
])
def test_norm_forward_refuses(lib, change, msg):
    with pytest.raises(binding.CmoeError, match=msg):
        binding._check(lib.cmoe_norm_forward(_norm_args(**change), None), "cmoe_norm_forward")


def test_norm_forward_of_no_rows_is_no_work(lib):
    assert lib.cmoe_norm_forward(_norm_args(rows=0, x=0, y=0), None) == 0
    assert lib.cmoe_norm_forward(None, None) < 0


def _norm_backward_args(**kw):
    f = dict(dy=1 << 20, s=2 << 20, dsum=0, weight=0, mean=3 << 20, rstd=4 << 20, dx=5 << 20, dresidual=0, dweight=0, dbias=0, workspace=0,
             workspace_bytes=0, rows=4, p=0.0, seed=0, offset=0, size=binding._NORM_BACKWARD.size, dtype=0, form=0, cols=16)
    f.update(kw)
    return binding._NORM_BACKWARD.pack(*f.values())


@pytest.mark.parametrize("change,msg", [
    (dict(size=8), "version"), (dict(dtype=3), "dtype"), (dict(form=-1), "form"), (dict(cols=40000), "cols"), (dict(rows=-3), "rows"), (dict(p=2.0), "rate"),
    (dict(dy=0), "null"), (dict(s=0), "null"), (dict(dx=0), "null"), (dict(rstd=0), "null"), (dict(mean=0), "null"),
    (dict(dbias=6 << 20), "dbias without"), (dict(dweight=6 << 20), "workspace"), (dict(dweight=6 << 20, workspace=7 << 20, workspace_bytes=8), "workspace"),
    (dict(dweight=6 << 20, workspace=(7 << 20) + 4, workspace_bytes=1 << 16), "aligned"), (dict(dresidual=5 << 20), "overlaps"),
    (dict(dweight=6 << 20, workspace=6 << 20, workspace_bytes=1 << 16), "overlaps"), (dict(dx=(2 << 20) + 64), "overlaps"),
])
def test_norm_backward_refuses(lib, change, msg):
    with pytest.raises(binding.CmoeError, match=msg):
        binding._check(lib.cmoe_norm_backward(_norm_backward_args(**change), None), "cmoe_norm_backward")


@pytest.mark.parametrize("change,msg", [
    (dict(x=0), "null"), (dict(y=0), "null"), (dict(rows=-1), "rows"), (dict(cols=0), "cols"), (dict(cols=1 << 31 - 1, rows=1 << 40), "cols|large"),
    (dict(rows=1 << 40), "large"), (dict(dtype=5), "dtype"), (dict(p=1.5), "rate"), (dict(x=(1 << 20) + 1), "aligned"), (dict(y=(1 << 20) + 4), "overlaps"),
    (dict(residual=(2 << 20) + 4), "overlaps"),
])
def test_dropout_refuses(lib, change, msg):
    f = dict(x=1 << 20, y=2 << 20, residual=0, rows=4, cols=16, dtype=0, p=0.5, seed=1, offset=2)
    f.update(change)
    with pytest.raises(binding.CmoeError, match=msg):
        binding._check(lib.cmoe_dropout(*f.values(), None), "cmoe_dropout")


def _adapter_args(forward, **kw):
    if forward:
        f = dict(x=1 << 24, a=2 << 24, b=3 << 24, scale=4 << 24, ids=5 << 24, base=6 << 24, y=7 << 24, u=8 << 24)
    else:
        f = dict(dy=1 << 24, x=2 << 24, u=3 << 24, a=4 << 24, b=5 << 24, scale=6 << 24, ids=7 << 24, dx_base=8 << 24, dx=9 << 24, da=10 << 24,
                 db=11 << 24, workspace=12 << 24, workspace_bytes=1 << 22)
    packer = binding._ADAPTERS_FORWARD if forward else binding._ADAPTERS_BACKWARD
    f.update(dict(tokens=4, p=0.0, seed=0, offset=0, size=packer.size, dtype=0, d_in=32, d_out=64, rank=8, n=2))
    f.update(kw)
    return packer.pack(*f.values())


SIZES = [
    (dict(size=8), "version"), (dict(dtype=2), "dtype"), (dict(tokens=-1), "tokens"), (dict(tokens=(1 << 20) + 1), "tokens"), (dict(d_in=0), "d_in"),
    (dict(d_out=0), "d_out"), (dict(rank=0), "rank"), (dict(rank=65), "rank"), (dict(n=0), "n_adapters"), (dict(n=70000), "n_adapters"), (dict(p=-1.0), "rate"),
    (dict(a=0), "null"), (dict(b=0), "null"), (dict(scale=0), "null"),
]


@pytest.mark.parametrize("change,msg", SIZES + [
    (dict(x=0), "null"), (dict(y=0), "null"), (dict(y=(6 << 24) + 4), "y overlaps base"), (dict(y=1 << 24), "overlaps"), (dict(u=7 << 24), "overlaps"),
    (dict(ids=(5 << 24) + 2), "aligned"),
])
def test_adapters_forward_refuses(lib, change, msg):
    with pytest.raises(binding.CmoeError, match=msg):
        binding._check(lib.cmoe_adapters_forward(_adapter_args(True, **change), None), "cmoe_adapters_forward")


@pytest.mark.parametrize("change,msg", SIZES + [
    (dict(dy=0), "null"), (dict(x=0), "da needs x"), (dict(u=0), "db needs u"), (dict(workspace=0), "workspace"), (dict(workspace_bytes=4), "workspace"),
    (dict(dx=(8 << 24) + 4), "dx overlaps dx_base"), (dict(dx=2 << 24), "overlaps"), (dict(da=11 << 24), "overlaps"),
])
def test_adapters_backward_refuses(lib, change, msg):
    with pytest.raises(binding.CmoeError, match=msg):
        binding._check(lib.cmoe_adapters_backward(_adapter_args(False, **change), None), "cmoe_adapters_backward")


def test_no_tokens_are_no_work(lib):
    assert lib.cmoe_adapters_forward(_adapter_args(True, tokens=0, x=0, y=0), None) == 0
    assert lib.cmoe_adapters_backward(_adapter_args(False, tokens=0, dy=0, da=0, db=0), None) == 0


def test_workspace_sizes(lib):
    """Sizes that are refused take no workspace; others take more with more tokens."""
    assert lib.cmoe_norm_backward_workspace_bytes(-1, 16) == 0 and lib.cmoe_norm_backward_workspace_bytes(4, 40000) == 0
    assert lib.cmoe_norm_backward_workspace_bytes(4, 16) > 0
    assert lib.cmoe_adapters_backward_workspace_bytes(4, 32, 64, 65, 2, 0) == 0 and lib.cmoe_adapters_backward_workspace_bytes(4, 32, 64, 8, 2, 9) == 0
    small, large = (lib.cmoe_adapters_backward_workspace_bytes(t, 4096, 4096, 8, 2, 1) for t in (1, 4096))
    assert 0 < small < large


def test_binding_refuses_what_does_not_fit():
    x, y = torch.zeros(4, 16), torch.zeros(4, 16)
    f32 = dict(dtype=torch.float32)
    drop = binding.Dropout(0.1, 1, 2)

    def refused(msg, fn, *args, **kw):
        with pytest.raises(binding.CmoeError, match=msg):
            fn(*args, **kw)

    refused("x must be bfloat16 or float32", binding.norm_forward, x.half(), y)
    refused("rows, cols", binding.norm_forward, x[0], y)
    refused("form", binding.norm_forward, x, y, form="batch")
    refused("HIP device", binding.norm_forward, x, y)
    refused("rows, cols", binding.dropout, x[0], y, drop)
    refused("HIP device", binding.dropout, x, y, drop)
    refused("p must be", binding.dropout, x, y, binding.Dropout(1.5, 1))
    refused("p must be", binding.dropout, x, y, binding.Dropout(float("nan"), 1))
    refused("seed", binding.dropout, x, y, binding.Dropout(0.5, -1))
    refused("seed", binding.dropout, x, y, binding.Dropout(0.5, 1, 1 << 64))
    a, b, scale = torch.zeros(2, 8, 16), torch.zeros(2, 32, 8), torch.ones(2)
    refused("rank", binding.adapters_forward, x, y, a, torch.zeros(2, 32, 4), scale)
    refused("tokens, width", binding.adapters_forward, x[0], y, a, b, scale)
    refused("n, rank, d_in", binding.adapters_forward, x, y, a[0], b, scale)
    refused("HIP device", binding.adapters_forward, x, torch.zeros(4, 32), a, b, scale)
    refused("bfloat16 or float32", binding.adapters_backward, torch.zeros(4, 32, dtype=torch.float64), x, None, a, b, scale)

    # shapes, types and strides are looked at before the device is
    m = torch.empty
    shape, dtype = torch.Size((4, 16)), torch.float32
    refused("shape", binding._operand, "y", m(4, 17, **f32), dtype, shape)
    refused("bfloat16", binding._operand, "y", m(4, 16, dtype=torch.bfloat16), dtype, shape)
    refused("strides", binding._operand, "y", m(16, 4, **f32).t(), dtype, shape)
    refused("strides", binding._operand, "y", m(4, 32, **f32)[:, :16], dtype, shape)
    assert binding._operand("y", None, dtype, shape) == 0
