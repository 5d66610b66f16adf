"""What the dense block and the head that are trained do with tensors of the caller's, on the GPU."""
import pytest
import torch

from paper_2502_04416_amd import binding, finetune, recovery, synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    binding.load()


def tensors(d, f, v):
    g = torch.Generator().manual_seed(d)
    return [torch.randn(*s, generator=g).cuda() * s[0] ** -0.5 for s in ((v, d), (d, f), (d, f), (f, d))]


def step(dense, d, v, n=50):
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, d, generator=g).cuda().to(dense.head.dtype)
    return dense.step(x, torch.zeros_like(x), torch.randint(0, v, (n,), generator=g).to(torch.int32).cuda(), lr=1e-2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("parameters", [False, True])
def test_training_leaves_what_it_began_with(dtype, parameters):
    """fp32 tensors on the device, a module's parameters among them, are copied like all others: a step changes none of them, and none of their graph."""
    d, f, v = 64, 136, 300
    given = tensors(d, f, v)
    if parameters:
        given = [torch.nn.Parameter(t) for t in given]
    before = [t.detach().clone() for t in given]
    dense = finetune.Dense(*given[1:], finetune.Head(given[0], dtype))
    for _ in range(2):
        step(dense, d, v)
    for t, b in zip(given, before):
        assert torch.equal(t, b)
    for k, p in dense.params.items():
        assert p.grad_fn is None and not p.requires_grad, k
    assert not torch.equal(dense.params["gate"], before[1]) and not torch.equal(dense.params["head"], before[0])


def test_matrices_with_strides():
    """Transposed views are taken as what they hold."""
    d, f, v = 32, 40, 90
    w = tensors(d, f, v)
    one = finetune.Dense(*w[1:], finetune.Head(w[0], torch.float32))
    other = finetune.Dense(*(t.t().contiguous().t() for t in w[1:]), finetune.Head(w[0].t().contiguous().t(), torch.float32))
    step(one, d, v), step(other, d, v)
    for k, p in one.params.items():
        assert p.is_contiguous() and other.params[k].is_contiguous() and torch.equal(p, other.params[k]), k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_torch_default_type_is_not_asked(dtype):
    """A program whose torch makes bf16 tensors by default trains the same block to the same bits."""
    d, f, v = 64, 136, 300
    w, made, g = tensors(d, f, v), [], torch.Generator().manual_seed(5)
    x, targets = torch.randn(50, d, generator=g).cuda().to(dtype), torch.randint(0, v, (50,), generator=g).to(torch.int32).cuda()
    for default in (torch.float32, torch.bfloat16):
        torch.set_default_dtype(default)
        try:
            dense = finetune.Dense(*w[1:], finetune.Head(w[0], dtype))
            made.append((dense, *dense.step(x, torch.zeros_like(x), targets)))
        finally:
            torch.set_default_dtype(torch.float32)
    (one, loss, norm), (other, its_loss, its_norm) = made
    assert torch.equal(loss, its_loss) and torch.equal(norm, its_norm)
    for k, p in one.params.items():
        assert other.params[k].dtype is torch.float32 and torch.equal(p, other.params[k]), k


def test_recovery_blocks_do_not_ask_for_torch_default_type():
    cfg = synth.scaled(synth.CONFIGS[0], d_model=96, d_ff=256, n_experts=4, n_shared=1, top_k=1)
    part = synth.trivial_partition(cfg)
    layer = binding.Layer.from_partition(cfg, *synth.make_weights(cfg), part["neuron_order"], part["rep_neuron"])
    g = torch.Generator().manual_seed(6)
    head = finetune.Head(torch.randn(200, 96, generator=g) * 0.1, torch.float32)
    x, targets, made = torch.randn(40, 96, generator=g).cuda(), torch.randint(0, 200, (40,), generator=g).to(torch.int32).cuda(), []
    for default in (torch.float32, torch.bfloat16):
        torch.set_default_dtype(default)
        try:
            block = recovery.Block(layer, rank=5, p=0.2, seed=3)
            made.append((block, block.step_tokens(x, torch.zeros_like(x), targets, head)))
        finally:
            torch.set_default_dtype(torch.float32)
    (one, loss), (other, its_loss) = made
    assert torch.equal(loss, its_loss)
    for k, p in one.params.items():
        assert other.params[k].dtype is torch.float32 and torch.equal(p, other.params[k]), k
    layer.close()
