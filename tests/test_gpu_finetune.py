"""The operators of a training step together, as the dense block and the recovery on tokens use them, on the GPU."""
import numpy as np
import pytest
import torch

import operator_oracle as O
from paper_2502_04416_amd import binding, finetune, recovery, synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    binding.load()


def made(dtype, d, f, v, seed=1):
    g = torch.Generator().manual_seed(seed)
    head = finetune.Head(torch.randn(v, d, generator=g) * d ** -0.5, dtype)
    dense = finetune.Dense(*(torch.randn(*s, generator=g) * s[0] ** -0.5 for s in ((d, f), (d, f), (f, d))), head)
    return g, dense


@pytest.mark.parametrize("d,f,v", [(64, 136, 300), (65, 131, 257)])
def test_gradients_of_the_dense_block(d, f, v):
    """Against autograd in 64 bits; fp32, sums of at most 300 terms in a row, four products deep: 4e-5 of the norm."""
    g, dense = made(torch.float32, d, f, v)
    x = torch.randn(90, d, generator=g).cuda()
    targets = torch.randint(-20, v, (90,), generator=g).to(torch.int32).cuda()
    dx = torch.empty_like(x)
    loss, grads = dense.gradients(x, x, targets, dx=dx)
    leaves = {k: p.double().requires_grad_() for k, p in dense.params.items()}
    xl = x.double().requires_grad_()
    a = xl @ leaves["gate"]
    s = xl + (a * torch.sigmoid(a) * (xl @ leaves["up"])) @ leaves["down"]
    out = s / (s.square().mean(1, keepdim=True) + dense.eps).sqrt() * leaves["weight"]
    t = targets.long()
    want = torch.nn.functional.cross_entropy(out @ leaves["head"].t(), torch.where(t < 0, -100, t), ignore_index=-100)
    want.backward()
    assert abs(float(loss) - want.item()) <= 4e-5 * want.item()
    for k, got in list(grads.items()) + [("x", dx)]:
        ref = xl.grad if k == "x" else leaves[k].grad
        assert float((got.double() - ref).norm()) <= 4e-5 * float(ref.norm()), k


def test_a_step_clips_all_gradients_together():
    """A step of Adam moves every parameter as its clipped gradient says."""
    g, dense = made(torch.float32, 32, 40, 90)
    x, residual = torch.randn(50, 32, generator=g).cuda(), torch.randn(50, 32, generator=g).cuda()
    targets = torch.randint(0, 90, (50,), generator=g).to(torch.int32).cuda()
    before = {k: p.clone() for k, p in dense.params.items()}
    _, grads = dense.gradients(x, residual, targets)
    total = sum(float(v.double().square().sum()) for v in grads.values()) ** 0.5
    loss, norm = dense.step(x, residual, targets, lr=1e-2, max_norm=total / 3)
    assert abs(float(norm) - total) <= 1e-6 * total
    for k, p in dense.params.items():
        m, v = dense.moments[k]
        want = grads[k].double() / 3
        # (the first moment is a tenth of the clipped gradient: three roundings and the norm's)
        assert float((m.double() - 0.1 * want).abs().max()) <= 1e-6 * float(want.abs().max()), k
        moved = before[k] - p
        assert float(moved.abs().max()) <= 1.01e-2 and bool(torch.isfinite(p).all())
        assert torch.equal(moved > 0, (grads[k] > 0) & (moved != 0)), k


def test_token_gradients_of_the_recovery_block():
    """Against autograd in 64 bits, with the layer's own outputs; fp32, sums of at most 300 terms in a row: 2e-5 of the norm."""
    cfg = synth.scaled(synth.CONFIGS[0], d_model=96, d_ff=256, n_experts=4, n_shared=1, top_k=1)
    part = synth.trivial_partition(cfg)
    layer = binding.Layer.from_partition(cfg, *synth.make_weights(cfg), part["neuron_order"], part["rep_neuron"])
    block = recovery.Block(layer, n_adapters=1, rank=5, p=0.2, seed=3)
    block.steps = 4
    g = torch.Generator().manual_seed(2)
    block.params["b"].copy_(torch.randn(block.params["b"].shape, generator=g) * 0.3)
    block._cast()
    head = finetune.Head(torch.randn(200, 96, generator=g) * 0.1, torch.float32)
    x, residual = (torch.randn(70, 96, generator=g).cuda() for _ in range(2))
    targets = torch.randint(-30, 200, (70,), generator=g).to(torch.int32).cuda()
    loss, grads = block.token_gradients(x, residual, targets, head)
    f = torch.empty_like(x)
    layer.forward_device(x, f)
    before, after = (O.mask(70, 96, binding.Dropout(0.2, 3, 8 + i), "cuda") for i in (0, 1))
    leaves = {k: p.double().requires_grad_() for k, p in block.params.items()}
    z = f.double() + block.scale.double()[0] * ((x.double() * before) @ leaves["a"][0].t()) @ leaves["b"][0].t()
    s = z * after + residual.double()
    out = s / (s.square().mean(1, keepdim=True) + block.eps).sqrt() * leaves["weight"]
    t = targets.long()
    want = torch.nn.functional.cross_entropy(out @ head.params["head"].double().t(), torch.where(t < 0, -100, t), ignore_index=-100)
    want.backward()
    assert abs(float(loss) - want.item()) <= 2e-5 * want.item()
    for k, got in grads.items():
        assert float((got.double() - leaves[k].grad).norm()) <= 2e-5 * float(leaves[k].grad.norm()), k
    layer.close()


def test_the_whole_way(capsys):
    """Trained, restructured and recovered, the example runs through and says what it measured."""
    losses = finetune.main(steps=5, tokens=256)
    assert len(losses) == 4 and np.isfinite(losses).all()
    assert "recovered" in capsys.readouterr().out
