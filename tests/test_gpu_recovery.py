"""The operators together, as the recovery block uses them, on the GPU."""
import numpy as np
import pytest
import torch

import operator_oracle as O
from paper_2502_04416_amd import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2502_04416_amd import binding as b
    b.load()
    return b


@pytest.mark.parametrize("form", ["rms", "layer"])
def test_gradients_of_the_block(B, form):
    """Against autograd in 64 bits on the same masks, with the layer's own outputs; fp32, sums of at most 300 terms in a row: 1e-5 of the norm."""
    from paper_2502_04416_amd.recovery import Block
    cfg = synth.scaled(synth.CONFIGS[0], d_model=96, d_ff=256, n_experts=4, n_shared=1, top_k=1)
    part = synth.trivial_partition(cfg)
    layer = B.Layer.from_partition(cfg, *synth.make_weights(cfg), part["neuron_order"], part["rep_neuron"])
    block = Block(layer, n_adapters=3, rank=5, p=0.2, form=form, seed=3)
    block.steps = 7
    rng = torch.Generator().manual_seed(1)
    block.params["b"].copy_(torch.randn(block.params["b"].shape, generator=rng) * 0.3)
    block._cast()
    x, residual, target = (torch.randn(70, 96, generator=rng).cuda() for _ in range(3))
    ids = torch.randint(-1, 3, (70,), generator=rng).to(torch.int32).cuda()
    loss, grads = block.gradients(x, residual, target, ids)

    f = torch.empty_like(x)
    layer.forward_device(x, f)
    before, after = (O.mask(70, 96, B.Dropout(0.2, 3, 14 + i), "cuda") for i in (0, 1))
    leaves = {k: v.double().requires_grad_() for k, v in block.params.items()}
    pick = ids.long().clamp(min=0)
    has = (ids >= 0).double()[:, None]
    u = torch.bmm(leaves["a"][pick], (x.double() * before)[:, :, None])[:, :, 0]
    z = f.double() + has * block.scale.double()[pick][:, None] * torch.bmm(leaves["b"][pick], u[:, :, None])[:, :, 0]
    s = z * after + residual.double()
    if form == "layer":
        s = s - s.mean(1, keepdim=True)
    out = s / (s.square().mean(1, keepdim=True) + block.eps).sqrt() * leaves["weight"]
    want = (out - target.double()).square().mean()
    want.backward()
    want = want.detach()
    assert abs(float(loss) - float(want)) <= 1e-5 * float(want)
    for k, g in grads.items():
        assert float((g.double() - leaves[k].grad).norm()) <= 1e-5 * float(leaves[k].grad.norm()), k
    layer.close()


def test_adapters_recover_part_of_the_loss(B, capsys):
    """A few steps bring the block closer to the dense layer on tokens that it was not trained on."""
    from paper_2502_04416_amd import recovery
    first, last = recovery.main(steps=60, tokens=512)
    assert np.isfinite(last) and last < first
    assert "before" in capsys.readouterr().out


def test_served_tokens_have_their_own_adapters(B):
    """A batch of requests gives each token what it gets alone with its adapter (bf16: the norm's sum of a token does not see the others)."""
    from paper_2502_04416_amd.recovery import Block
    cfg = synth.scaled(synth.CONFIGS[1], d_model=256, d_ff=1024, n_experts=8, n_shared=1, top_k=2, n_centres=8)
    part = synth.trivial_partition(cfg)
    layer = B.Layer.from_partition(cfg, *synth.make_weights(cfg), part["neuron_order"], part["rep_neuron"])
    block = Block(layer, n_adapters=3, rank=8)
    rng = torch.Generator().manual_seed(2)
    block.params["b"].copy_(torch.randn(block.params["b"].shape, generator=rng) * 0.1)
    block._cast()
    x, residual = (torch.randn(12, 256, generator=rng).to("cuda", torch.bfloat16) for _ in range(2))
    ids = torch.tensor([0, 1, 2, -1] * 3, dtype=torch.int32, device="cuda")
    out, stream = block.serve(x, residual, ids)
    f = torch.empty_like(x)
    layer.forward_device(x, f)
    want, tol = O.adapters(x, None, block.a, block.b, block.scale, ids.tolist(), f, None, torch.ones(12, 256, dtype=torch.float64, device="cuda"))
    # the adapters' output is rounded once before the residual is added: half a step of it, and of the sum
    half = O.half_step(torch.bfloat16)
    total = want["y"] + residual.double()
    O.check(stream, total, tol["y"] + half * (total.abs() + tol["y"]), "stream")
    y, bound = O.norm_forward(stream, block.weight, None, "rms", block.eps, torch.bfloat16)
    O.check(out, y["y"], bound["y"], "out")
    layer.close()
