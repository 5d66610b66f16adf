"""How exact the operators of a training step are where a sum's bound over many roundings would not show it: single products of fp32 matrices
on the matrix cores, logits that both passes of the head have to share, factors of the head's gradients, joins of its ranges."""
import pytest
import torch

import operator_oracle as O
from test_gpu_operators import Arena, TYPES
from test_gpu_training_operators import run_head

pytestmark = pytest.mark.gpu

RINGS = {"ring 128": 1, "ring 64": 2}


@pytest.fixture(scope="module")
def B():
    from paper_2502_04416_amd import binding as b
    b.load()
    return b


@pytest.fixture
def forced(B):
    def force(tile=None):
        B.cmoe_set_tuning("CMOE_MAT_TILE", RINGS.get(tile, -1))
    yield force
    force()


# ---- products of fp32 matrices from planes of bf16 --------------------------------------------------------------------


def outer_as_gradient(B, h, d):
    """The gradient of w_down of a single token: h[i] d[j], a product over one K."""
    f, n = len(h), len(d)
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    out = torch.empty(f, n, device="cuda")
    B.ffn_backward(d[None], z(1, n), z(1, f), z(1, f), h[None], z(n, f), z(n, f), z(f, n), z(1, f), z(1, f), dw_down=out)
    return out


def outer_as_output(B, h, d):
    """y of a hidden state that is one wide, h[i] d[j]: hidden = gate / (1 + exp(-gate)) * up with a gate that is its own silu."""
    t, n = len(h), len(d)
    hidden, y = torch.empty(t, 1, device="cuda"), torch.empty(t, n, device="cuda")
    x = torch.zeros(t, n, device="cuda")
    x[:, 0], x[:, 1] = 128.0, h                              # exp(-128) is below half a step of 1
    wg, wu = torch.zeros(n, 1, device="cuda"), torch.zeros(n, 1, device="cuda")
    wg[0], wu[1] = 1.0, 2.0 ** -7
    B.ffn_forward(x, y, wg, wu, d[None], hidden)
    assert torch.equal(hidden[:, 0], h)
    return y


def spread(n, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    sign = torch.where(torch.rand(n, generator=g) < 0.5, -1.0, 1.0)
    return (sign * (1 + torch.rand(n, generator=g)) * scale).cuda()


# Three planes of eight bits, each rounded to nearest: the second is at most 2^-8 of the value's power of two, the third 2^-17.  The pairs that
# are left out, second times third twice and third times third, come to less than 2^-24 (1 + 2^-9) of the product; the small pairs' sum is 2^-7 of it at most and
# rounded five times, the last sum once: 2^-24 (1 + 10 * 2^-7).
ONE_PRODUCT = 2.15 * O.U32


def check_products(out, h, d):
    want = h.double()[:, None] * d.double()[None]
    off = (out.double() - want) / want.abs()
    assert float(off.abs().max()) <= ONE_PRODUCT, float(off.abs().max()) / O.U32
    return off * want.sign()


@pytest.mark.parametrize("tile,outer", [("ring 128", outer_as_gradient), ("ring 128", outer_as_output), ("ring 64", outer_as_output)])
def test_products_of_fp32_have_24_bits_and_no_side(B, forced, tile, outer):
    forced(tile)
    h, d = spread(1024, 1), spread(1000, 2)
    h[:4] = torch.tensor([0x3f80ffff, 0x3fffffff, 0x3f800001, 0x3f7f7fff], dtype=torch.int32).view(torch.float32).cuda()
    d[:4] = h[:4]
    short = check_products(outer(B, h, d), h, d)
    # errors of either sign: independent from row to row, each at most the bound, so that their mean is within 5 deviations of 2.15 / sqrt(1000)
    assert abs(float(short.mean())) <= 5 * ONE_PRODUCT / 1000 ** 0.5, float(short.mean()) / O.U32


@pytest.mark.parametrize("power", [-110, -100, -60, 60, 127])
def test_products_of_fp32_over_the_range(B, forced, power):
    """From 2^-110, whose last bit is bf16's smallest number, to the largest, which no plane may round to infinity."""
    forced("ring 128")
    h, d = spread(128, 3, 2.0 ** power), spread(128, 4, 2.0 ** (-power // 2 - 2))
    most = torch.finfo(torch.float32).max
    if power == 127:
        h[0], h[1] = most, -most
        h[2:5] = torch.tensor([0x7f7f7fff, 0x7f7f8000, 0x7f7f8001], dtype=torch.int32).view(torch.float32).cuda()
    check_products(outer_as_gradient(B, h, d), h, d)


# ---- the logits of both passes -----------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,shift,t,d,v", [
    (torch.float32, 0, 65600, 8, 2051), (torch.float32, 0, 65600, 5, 2051), (torch.float32, 1, 2048, 14, 131075), (torch.bfloat16, 1, 65600, 8, 2051),
    (torch.bfloat16, 1, 65600, 7, 2051), (torch.bfloat16, 0, 65600, 8, 2051), (torch.float32, 0, 300, 3, 7), (torch.float32, 0, 40, 1, 2051),
])
def test_a_certain_target_has_no_gradient(B, dtype, shift, t, d, v):
    """A target that has all of the softmax, in a last piece of the vocabulary that is a few entries wide: every other logit lies more than 104 below
    (exp is 0 in fp32), so lse is the target's logit, loss 0, and its entry exp(z - lse) - 1 is 0 as long as both passes have the same bits of z."""
    m = Arena(t + d, shift=shift)
    # positive factors of many sizes, so that the order of a sum shows in its last bits
    size = lambda n: torch.exp2(-9 * torch.rand(n, d, generator=m.rng)) * torch.tensor([16.0] + [4.0] * (d - 1))  # noqa: E731
    x, w = size(t), -size(v)
    x[:, 0] = 16 + torch.rand(t, generator=m.rng)
    w[v - 1] = size(1)[0]
    w[:, 0] = -16 - torch.rand(v, generator=m.rng)
    w[v - 1, 0] *= -1
    x, w = m.put(x.to(dtype)), m.put(w.to(dtype))
    ids = torch.full((t,), v - 1, dtype=torch.int32, device="cuda")
    loss, lse, dx, dw = m.out(t), m.out(t), m.out(t, d, dtype=dtype), m.out(v, d, dtype=dtype)
    B.head_loss_forward(x, w, ids, loss, lse)
    assert bool((loss == 0).all())
    B.head_loss_backward(x, w, ids, lse, dx=dx, dweight=dw)
    assert int((dx != 0).sum()) == 0 and int((dw != 0).sum()) == 0
    m.intact()


# ---- the join of the ranges --------------------------------------------------------------------------------------------


def test_ranges_are_joined_with_fp32_exponentials(B):
    """One logit of 0 behind 2^20 - 1 equal ones of -12.2 to -13.8, where an exponential as 2^(x log2 e) is off by up to 14 roundings.  Every range
    but the last sums to a whole number, exactly; what is left to be rounded lies where the last range meets the others."""
    t, v = 64, 1 << 20
    m = Arena(3, shift=0)
    x, w = torch.zeros(t, 8), torch.zeros(v, 8)
    x[:, 0], w[:v - 1, 0] = 12.2 + 1.6 * torch.rand(t, generator=m.rng), -1.0
    x, w, ids = m.put(x), m.put(w), torch.full((t,), v - 1, dtype=torch.int32, device="cuda")
    loss, lse = m.out(t), m.out(t)
    B.head_loss_forward(x, w, ids, loss, lse)
    want = torch.log1p((v - 1) * torch.exp(-x[:, 0].double()))
    # Roundings of 2^-24, spread evenly over what each may be off by (a third of its square is the variance).  The sum S = 1 + (2 to 6.3) has twelve
    # additions below 2 and two beyond: (12 + 2 * 4) / 3 / S^2, at S = 2.06 1.57; the others' exponential within one unit of the last place, two roundings:
    # 4/3, and its product 1/3, of at most (1 - 1 / S)^2 = 0.71; the logarithm within one unit of its last place, two roundings from 1 on: 4/3.
    # Of 64 tokens' mean square five standard deviations, each sqrt(2 / 64), more.
    variance = 1.57 + (4 / 3 + 1 / 3) * 0.71 + 4 / 3
    for got in (loss, lse):
        off = (got.double() - want) / O.U32
        assert float(off.square().mean()) <= variance * (1 + 5 * (2 / t) ** 0.5), float(off.square().mean()) ** 0.5
    m.intact()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t,d,v", [(1, 8, 1), (1, 9, 1), (3, 8, 2), (1, 15, 7), (2, 7, 1), (5, 14, 9), (1, 4, 2)])
def test_heads_of_a_few_values(B, dtype, t, d, v):
    """Operands that have just the 16 bytes that a load takes, and fewer."""
    run_head(B, Arena(t + d + v, shift=1), TYPES[dtype], t, d, v, weighted=v == 1)
