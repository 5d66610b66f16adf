"""What training a block on tokens rounds, and how often, on the GPU."""
import pytest
import torch

import operator_oracle as O
from paper_2502_04416_amd import binding, finetune
from test_gpu_operators import Arena, TYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    binding.load()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t,d,v", [(70, 64, 300), (5, 33, 70), (300, 40, 1003)])
def test_gradients_of_the_mean_loss_are_rounded_once(dtype, t, d, v):
    """They have the bits of the entry point's with the mean's factor, which is applied to sums in fp32."""
    g = torch.Generator().manual_seed(t)
    head = finetune.Head(torch.randn(v, d, generator=g) * d ** -0.5, TYPES[dtype])
    out = torch.randn(t, d, generator=g).cuda().to(TYPES[dtype])
    targets = torch.randint(0, v, (t,), generator=g).to(torch.int32)
    targets[::4] = -100
    count = int((targets >= 0).sum())
    assert count & (count - 1)                               # (a power of two rounds nothing)
    targets = targets.cuda()
    loss, dout, dweight = head.loss(out, targets)
    each, lse = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
    binding.head_loss_forward(out, head.weight, targets, each, lse)
    dx, dw = torch.empty_like(out), torch.empty_like(head.weight)
    binding.head_loss_backward(out, head.weight, targets, lse, dx=dx, dweight=dw, scale=float(torch.tensor(1.0 / count)))
    assert torch.equal(dout, dx) and torch.equal(dweight, dw)
    assert abs(float(loss) - float(each.double().sum()) / count) <= 4 * t * O.U32 * float(each.double().sum()) / count


def gradients(m, dt, t, d, v, scale):
    g = torch.Generator().manual_seed(t + v)
    x, w = m.put(torch.randn(t, d, generator=g).to(dt)), m.put((torch.randn(v, d, generator=g) * d ** -0.5).to(dt))
    ids = torch.randint(-v // 4, v, (t,), generator=g).to(torch.int32).cuda()
    lse, dx, dw = m.out(t), m.out(t, d, dtype=dt), m.out(v, d, dtype=dt)
    binding.head_loss_forward(x, w, ids, lse=lse)
    binding.head_loss_backward(x, w, ids, lse, dx=dx, dweight=dw, scale=scale)
    m.intact()
    return dx, dw


ON_TILES = [(dtype, shift, 130, 67 + 197 * (dtype == "bf16" and shift == 0), 520, tile, split) for dtype, shift in (("bf16", 0), ("bf16", 1), ("fp32", 1))
            for tile, split in ((-1, -1), (0, 1), (1, 4), (2, 2), (3, 4), (4, 1))]


@pytest.mark.parametrize("dtype,shift,t,d,v,tile,split", ON_TILES + [("bf16", 0, 65600, 8, 2051, -1, -1), ("fp32", 0, 65600, 8, 2051, -1, -1), ("fp32", 0, 3, 1, 1, -1, -1)])
def test_a_factor_on_the_device_is_the_number(dtype, shift, t, d, v, tile, split):
    """The same bits, on every tile, where K is split and where the vocabulary is taken in pieces."""
    binding.cmoe_set_tuning("CMOE_MAT_TILE", tile)
    binding.cmoe_set_tuning("CMOE_MAT_SPLIT", split)
    try:
        dt, number = TYPES[dtype], torch.tensor(0.37)
        want = gradients(Arena(1, shift=shift), dt, t, d, v, float(number))
        for factor in (number.cuda(), number.cuda()[None], number):
            for got, one in zip(gradients(Arena(1, shift=shift), dt, t, d, v, factor), want):
                assert torch.equal(got, one)
    finally:
        binding.cmoe_set_tuning("CMOE_MAT_TILE", -1)
        binding.cmoe_set_tuning("CMOE_MAT_SPLIT", -1)


def test_a_factor_is_read_when_the_kernels_run():
    """From a captured graph: the factor of every replay; a NaN is passed on; without tokens the gradient is zeros whatever it is."""
    m = Arena(2, shift=0)
    t, d, v, dt = 40, 64, 300, torch.bfloat16
    x, w, ids = m.normal(t, d, dtype=dt), m.normal(v, d, dtype=dt, std=0.1), torch.randint(0, v, (t,), generator=m.rng).to(torch.int32).cuda()
    lse, dx, dw, factor = m.out(t), m.out(t, d, dtype=dt), m.out(v, d, dtype=dt), torch.ones((), device="cuda")
    binding.head_loss_forward(x, w, ids, lse=lse)
    call = lambda scale: binding.head_loss_backward(x, w, ids, lse, dx=dx, dweight=dw, scale=scale)  # noqa: E731
    call(factor)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(factor)
    for value in (0.3, 2.0, -0.7):
        call(float(torch.tensor(value)))
        want = dx.clone(), dw.clone()
        dx.fill_(float("nan")), dw.fill_(float("nan"))
        factor.fill_(value)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
    factor.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert bool(torch.isnan(dx).all()) and bool(torch.isnan(dw).all())
    none = torch.empty(0, d, dtype=dt, device="cuda")
    binding.head_loss_backward(none, w, ids[:0], lse[:0], dx=none.clone(), dweight=dw, scale=factor)
    assert bool((dw == 0).all())
    m.intact()
