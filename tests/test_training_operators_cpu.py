"""The operators of a training step without a GPU: the argument structs against the header's, every refusal of the binding and of the C entry
points (none of which reaches a launch), workspace sizes, and the 64-bit oracle against autograd."""
import os
import re
import subprocess

import pytest
import torch

import training_oracle as R
from paper_2502_04416_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("ffn_forward", "ffn_backward", "head_loss_forward", "head_loss_backward")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return binding.load()


def test_structs_have_the_sizes_and_order_of_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    structs = ["cmoe_%s_args" % n for n in NAMES] + ["cmoe_gradient"]
    src.write_text('#include <stdio.h>\n#include "cmoe.h"\nint main(void) { printf("%s\\n", %s); return 0; }' % (
        " ".join(["%zu"] * len(structs)), ", ".join("sizeof(%s)" % n for n in structs)))
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    sizes = [int(v) for v in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()]
    packers = [getattr(binding, "_%s" % n.upper()) for n in NAMES] + [binding._GRADIENT]
    assert sizes == [p.size for p in packers]
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cmoe.h")).read(), flags=re.S)
    code = {"int64_t": "q", "uint64_t": "Q", "int32_t": "i", "float": "f"}
    for name, packer in zip(structs, packers):
        fields = ""
        for line in filter(None, (l.strip() for l in re.search(r"typedef struct \{([^}]*)\} %s;" % name, header).group(1).split(";"))):
            kind, rest = re.match(r"(?:const )?(\w+)\s*(.*)", line, flags=re.S).groups()
            fields += "".join("Q" if "*" in part else code[kind] for part in rest.split(","))
        assert fields == re.sub(r"(\d+)(\w)", lambda m: m.group(2) * int(m.group(1)), packer.format[1:]), name


M = 1 << 24
FIELDS = {
    "ffn_forward": dict(x=M, w_gate=2 * M, w_up=3 * M, w_down=4 * M, base=5 * M, hidden=6 * M, gate=7 * M, up=8 * M, y=9 * M, workspace=20 * M, workspace_bytes=M,
                        tokens=4, size=0, dtype=0, d=32, d_ff=64),
    "ffn_backward": dict(dy=M, x=2 * M, gate=3 * M, up=4 * M, hidden=5 * M, w_gate=6 * M, w_up=7 * M, w_down=8 * M, dx_base=9 * M, dgate=10 * M, dup=11 * M, dx=12 * M,
                         dw_gate=13 * M, dw_up=14 * M, dw_down=15 * M, workspace=20 * M, workspace_bytes=M, tokens=4, size=0, dtype=0, d=32, d_ff=64),
    "head_loss_forward": dict(x=M, weight=2 * M, ids=3 * M, loss=4 * M, lse=5 * M, workspace=20 * M, workspace_bytes=M, tokens=4, size=0, dtype=0, d=32, vocab=64),
    "head_loss_backward": dict(x=M, weight=2 * M, ids=3 * M, lse=4 * M, dloss=5 * M, dx=6 * M, dweight=7 * M, workspace=20 * M, workspace_bytes=M, tokens=4, size=0,
                               dtype=0, d=32, vocab=64, scale=1.0, reserved=0),
}


def refuse(lib, name, change, msg):
    packer = getattr(binding, "_%s" % name.upper())
    args = dict(FIELDS[name], size=packer.size)
    args.update(change)
    with pytest.raises(binding.CmoeError, match=msg):
        binding._check(getattr(lib, "cmoe_" + name)(packer.pack(*args.values()), None), name)


BIG = 1 << 20
BAD = [(dict(size=8), "version"), (dict(dtype=2), "dtype"), (dict(tokens=-1), "tokens"), (dict(tokens=BIG + 1), "tokens"), (dict(d=0), "2.20"),
       (dict(d=BIG + 1), "2.20"), (dict(x=M + 2), "aligned")]


@pytest.mark.parametrize("change,msg", BAD + [
    (dict(d_ff=0), "widths"), (dict(d_ff=BIG + 1), "widths"), (dict(x=0), "null"), (dict(w_gate=0), "null"), (dict(w_up=0), "null"), (dict(w_down=0), "null"),
    (dict(hidden=0), "null"), (dict(y=0), "null"), (dict(gate=0), "together"), (dict(up=0), "together"), (dict(y=M), "y overlaps x"), (dict(y=5 * M + 4), "y overlaps base"),
    (dict(hidden=7 * M), "overlaps"), (dict(gate=8 * M + 64), "overlaps"), (dict(up=3 * M), "overlaps"), (dict(hidden=M), "hidden overlaps x"),
])
def test_ffn_forward_refuses(lib, change, msg):
    refuse(lib, "ffn_forward", change, msg)


@pytest.mark.parametrize("change,msg", BAD + [
    (dict(dy=0), "null"), (dict(gate=0), "null"), (dict(up=0), "null"), (dict(w_down=0), "null"), (dict(dgate=0), "null"), (dict(dup=0), "null"),
    (dict(w_gate=0), "dx needs"), (dict(w_up=0), "dx needs"), (dict(x=0), "need x"), (dict(hidden=0), "needs hidden"), (dict(dx=0), "without dx"),
    (dict(dgate=3 * M + 4), "dgate overlaps gate"), (dict(dup=10 * M), "overlaps"), (dict(dgate=5 * M), "dgate overlaps hidden"),
    (dict(dx=9 * M + 4), "dx overlaps dx_base"), (dict(dx=M), "dx overlaps dy"), (dict(dx=10 * M), "dx overlaps dgate"), (dict(dw_gate=14 * M), "overlaps"),
    (dict(dw_down=8 * M), "overlaps w_down"), (dict(dw_up=12 * M), "overlaps"),
    # of one size, dgate over dx_base would be gone before it is read
    (dict(d=64, dgate=9 * M), "dgate overlaps dx_base"), (dict(d=64, dx=3 * M), "dx overlaps gate"),
])
def test_ffn_backward_refuses(lib, change, msg):
    refuse(lib, "ffn_backward", change, msg)


@pytest.mark.parametrize("change,msg", BAD + [
    (dict(vocab=0), "vocab"), (dict(vocab=BIG + 1), "vocab"), (dict(x=0), "null"), (dict(weight=0), "null"), (dict(ids=0), "null"), (dict(loss=0, lse=0), "neither"),
    (dict(ids=3 * M + 2), "aligned"), (dict(loss=5 * M), "overlaps"), (dict(lse=3 * M), "lse overlaps ids"), (dict(workspace=0), "workspace"),
    (dict(workspace=20 * M + 8), "workspace"), (dict(workspace_bytes=16), "needs"), (dict(workspace=4 * M), "overlaps"),
])
def test_head_loss_forward_refuses(lib, change, msg):
    refuse(lib, "head_loss_forward", change, msg)


@pytest.mark.parametrize("change,msg", BAD + [
    (dict(vocab=0), "vocab"), (dict(x=0), "null"), (dict(weight=0), "null"), (dict(ids=0), "null"), (dict(lse=0), "null"), (dict(dx=0, dweight=0), "neither"),
    (dict(dx=M), "dx overlaps x"), (dict(dweight=2 * M), "dweight overlaps weight"), (dict(dx=7 * M), "overlaps"), (dict(workspace=0), "workspace"),
    (dict(workspace_bytes=16), "needs"), (dict(workspace=7 * M), "overlaps"), (dict(lse=4 * M + 1), "aligned"),
])
def test_head_loss_backward_refuses(lib, change, msg):
    refuse(lib, "head_loss_backward", change, msg)


def clip(lib, tensors, max_norm=1.0, eps=1e-6, norm=M, workspace=2 * M, workspace_bytes=1 << 20, count=None):
    packed = b"".join(binding._GRADIENT.pack(*t, 0) for t in tensors)
    binding._check(lib.cmoe_clip_gradients(packed, len(tensors) if count is None else count, max_norm, eps, norm, workspace, workspace_bytes, None), "cmoe_clip_gradients")


@pytest.mark.parametrize("tensors,kw,msg", [
    ([(4 * M, 4 * M, -1, 0)], {}, "size"), ([(4 * M, 4 * M, 1 << 41, 0)], {}, "size"), ([(4 * M, 4 * M, 8, 2)], {}, "dtype"), ([(0, 4 * M, 8, 0)], {}, "null"),
    ([(4 * M, 0, 8, 0)], {}, "null"), ([(4 * M + 2, 5 * M, 8, 0)], {}, "aligned"), ([(4 * M, 5 * M + 1, 8, 1)], {}, "aligned"), ([(4 * M, 4 * M, 8, 0)], dict(norm=0), "norm"),
    ([(4 * M, 4 * M, 8, 0)], dict(norm=M + 2), "norm"), ([(4 * M, 4 * M, 8, 0)], dict(workspace=0), "workspace"), ([(4 * M, 4 * M, 8, 0)], dict(workspace=2 * M + 4), "workspace"),
    ([(4 * M, 4 * M, 8, 0)], dict(workspace_bytes=4), "workspace"), ([(4 * M, 4 * M, 8, 0)], dict(max_norm=-1.0), "max_norm"), ([(4 * M, 4 * M, 8, 0)], dict(max_norm=float("nan")), "max_norm"),
    ([(4 * M, 4 * M, 8, 0)], dict(eps=-1.0), "eps"), ([(4 * M, 4 * M, 8, 0)], dict(eps=float("inf")), "eps"), ([(4 * M, 4 * M + 4, 8, 0)], {}, "overlaps"),
    ([(4 * M, 4 * M, 8, 0)] * 2, {}, "overlaps"), ([(4 * M, 4 * M, 8, 0), (5 * M, 4 * M + 28, 8, 0)], {}, "overlaps"), ([(4 * M, 5 * M, 8, 0), (5 * M, 6 * M, 8, 0)], {}, "overlaps"),
    ([(4 * M, 4 * M, 8, 0)], dict(norm=4 * M + 4), "overlaps"), ([(4 * M, 4 * M, 8, 0)], dict(workspace=4 * M), "overlaps"), ([], dict(count=-1), "list"), ([], dict(count=70000), "list"),
    # a long tensor before the short ones around an output
    ([(4 * M, 5 * M, 1 << 20, 0), (4 * M + 4096, 6 * M, 8, 0), (7 * M, 4 * M + 8192, 8, 0)], {}, "overlaps"),
])
def test_clip_refuses(lib, tensors, kw, msg):
    with pytest.raises(binding.CmoeError, match=msg):
        clip(lib, tensors, **kw)


def test_no_tokens_are_no_work(lib):
    for name in ("ffn_forward", "head_loss_forward"):
        packer = getattr(binding, "_%s" % name.upper())
        args = dict(FIELDS[name], size=packer.size, tokens=0, x=0)
        assert getattr(lib, "cmoe_" + name)(packer.pack(*args.values()), None) == 0
        assert getattr(lib, "cmoe_" + name)(None, None) < 0
    packer = binding._HEAD_LOSS_BACKWARD
    assert lib.cmoe_head_loss_backward(packer.pack(*dict(FIELDS["head_loss_backward"], size=packer.size, tokens=0, dweight=0).values()), None) == 0
    packer = binding._FFN_BACKWARD
    assert lib.cmoe_ffn_backward(packer.pack(*dict(FIELDS["ffn_backward"], size=packer.size, tokens=0, dw_gate=0, dw_up=0, dw_down=0).values()), None) == 0


def test_workspace_sizes(lib):
    """Sizes that are refused take none; the logits of a vocabulary are in none of them."""
    for name in NAMES:
        size = getattr(lib, "cmoe_%s_workspace_bytes" % name)
        assert size(-1, 64, 64, 1) == 0 and size(4, 0, 64, 1) == 0 and size(4, 64, BIG + 1, 1) == 0 and size(4, 64, 64, 7) == 0 and size(0, 64, 64, 0) >= 0
    for dtype, logits in ((0, 8192 * 131072 * 4), (1, 8192 * 131072 * 2)):
        assert 0 < lib.cmoe_head_loss_forward_workspace_bytes(8192, 4096, 131072, dtype) < logits // 2
        assert 0 < lib.cmoe_head_loss_backward_workspace_bytes(8192, 4096, 131072, dtype) < logits // 2
    assert lib.cmoe_clip_gradients_workspace_bytes(binding._GRADIENT.pack(0, 0, 5, 0, 0), 1) == 8
    assert lib.cmoe_clip_gradients_workspace_bytes(binding._GRADIENT.pack(0, 0, 0, 0, 0), 1) == 0
    assert lib.cmoe_clip_gradients_workspace_bytes(binding._GRADIENT.pack(0, 0, 1 << 30, 0, 0), 1) < 1 << 16


def test_binding_refuses_what_does_not_fit():
    def refused(msg, fn, *args, **kw):
        with pytest.raises(binding.CmoeError, match=msg):
            fn(*args, **kw)

    x, w, wd, h = torch.zeros(4, 16), torch.zeros(16, 24), torch.zeros(24, 16), torch.zeros(4, 24)
    refused("bfloat16 or float32", binding.ffn_forward, x.half(), x, w, w, wd, h)
    refused("tokens, d", binding.ffn_forward, x[0], x, w, w, wd, h)
    refused("tokens, d", binding.ffn_forward, x, x, w, w, torch.zeros(24, 17), h)
    refused("HIP device", binding.ffn_forward, x, x, w, w, wd, h)
    refused("bfloat16 or float32", binding.ffn_backward, x.double(), x, h, h, h, w, w, wd, h, h)
    refused("tokens, d", binding.ffn_backward, x, x, h, h, h, w, w, wd[0], h, h)
    refused("HIP device", binding.ffn_backward, x, x, h, h, h, w, w, wd, h, h)
    ids, row = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    refused("vocab, d", binding.head_loss_forward, x, w, ids, row)
    refused("HIP device", binding.head_loss_forward, x, wd, ids, row)
    refused("vocab, d", binding.head_loss_backward, x[0], wd, ids, row)
    refused("scale", binding.head_loss_backward, x, wd, ids, row, scale=float("inf"))
    refused("scale", binding.head_loss_backward, x, wd, ids, row, scale=float("nan"))
    refused("HIP device", binding.head_loss_backward, x, wd, ids, row)
    refused("HIP device", binding.clip_gradients, [x], torch.zeros(1), 1.0)
    refused("max_norm", binding.clip_gradients, [x], torch.zeros(1), -1.0)
    refused("max_norm", binding.clip_gradients, [x], torch.zeros(1), float("nan"))
    refused("max_norm", binding.clip_gradients, [x], torch.zeros(1), 1.0, eps=float("inf"))
    refused("out must have", binding.clip_gradients, [x], torch.zeros(1), 1.0, out=[])


def test_clip_refuses_lists_of_other_things(monkeypatch):
    """A list with the gradient of a parameter that has none."""
    monkeypatch.setattr(binding, "_place", lambda name, t: (-1, 0))
    for grads, kw in (([torch.zeros(3), None], {}), ([torch.zeros(3)], dict(out=[None])), ([1.0], {})):
        with pytest.raises(binding.CmoeError, match="tensors"):
            binding.clip_gradients(grads, torch.zeros(1), 1.0, **kw)


def test_oracle_against_autograd():
    g = torch.Generator().manual_seed(0)
    n = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).requires_grad_()  # noqa: E731
    x, wg, wu, wd, w = n(7, 6), n(6, 9), n(6, 9), n(9, 6), n(11, 6)
    gate, up = x @ wg, x @ wu
    gate.retain_grad(), up.retain_grad()
    h = torch.nn.functional.silu(gate) * up
    y = h @ wd
    fwd = R.ffn_forward(x.detach(), wg.detach(), wu.detach())
    assert torch.allclose(fwd["hidden"][0], h, rtol=1e-12)
    dy = torch.randn(7, 6, generator=g, dtype=torch.float64)
    y.backward(dy)
    got = R.ffn_gates(dy, wd.detach(), gate.detach(), up.detach())
    assert torch.allclose(got["dgate"][0], gate.grad, rtol=1e-10) and torch.allclose(got["dup"][0], up.grad, rtol=1e-10)
    x.grad = None
    ids = torch.tensor([3, -100, 0, 10, 10, 11, 5])
    weight = torch.rand(7, generator=g, dtype=torch.float64)
    kept = torch.where((ids >= 0) & (ids < 11), ids, -100)
    each = torch.nn.functional.cross_entropy(x @ w.t(), kept, ignore_index=-100, reduction="none")
    want = R.head_loss(x.detach(), w.detach(), ids)
    assert torch.allclose(want["loss"][0], each)
    (0.3 * (weight * each).sum()).backward()
    got = R.head_gradients(x.detach(), w.detach(), ids, want["lse"][0], weight, 0.3)
    assert torch.allclose(got["dx"][0], x.grad, rtol=1e-10, atol=1e-14) and torch.allclose(got["dw"][0], w.grad, rtol=1e-10, atol=1e-14)
