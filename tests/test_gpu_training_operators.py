"""The feed-forward block, the head's loss and the clipping on the GPU against their definitions in 64 bits (training_oracle.py).

Tensors lie in larger buffers of NaN: at addresses of an element's alignment, where the kernels that take any operand run, or of 16 bytes,
where widths of multiples of 8 run on the ring, with every tile and K split forced in turn.
"""
import pytest
import torch

import operator_oracle as O
import training_oracle as R
from test_gpu_operators import Arena, TYPES

pytestmark = pytest.mark.gpu

RING = {"ring 256": 0, "ring 128": 1, "ring 64": 2}
ANY = {"any 64": 3, "any 32": 4}
TILES = {None: -1, **RING, **ANY}


@pytest.fixture(scope="module")
def B():
    from paper_2502_04416_amd import binding as b
    b.load()
    return b


@pytest.fixture
def forced(B):
    def force(tile=None, split=-1):
        B.cmoe_set_tuning("CMOE_MAT_TILE", TILES[tile])
        B.cmoe_set_tuning("CMOE_MAT_SPLIT", split)
    yield force
    force()


def close(got, want, dtype, name):
    value, bound = want
    O.check(got, value, R.stored(value, bound, dtype), name)


def run_ffn(B, m, dt, t, d, f, base=False, train=True, in_place=False):
    x, dy = m.normal(t, d, dtype=dt), m.normal(t, d, dtype=dt, std=0.5)
    wg, wu, wd = (m.normal(*s, dtype=dt, std=s[0] ** -0.5) for s in ((d, f), (d, f), (f, d)))
    y, hidden = m.out(t, d, dtype=dt), m.out(t, f, dtype=dt)
    b = m.normal(t, d, dtype=dt) if base else None
    gate, up = (m.out(t, f, dtype=dt) for _ in range(2)) if train else (None, None)
    if in_place and base:
        y.copy_(b)
    B.ffn_forward(x, y, wg, wu, wd, hidden, gate=gate, up=up, base=y if in_place and base else b)
    want = R.ffn_forward(x, wg, wu)
    if train:
        close(gate, want["gate"], dt, "gate")
        close(up, want["up"], dt, "up")
    close(hidden, want["hidden"], dt, "hidden")
    value, bound = R.product(hidden, wd)
    if base:
        value, bound = value + b.double(), bound + 2 * O.U32 * (value.abs() + b.double().abs())
    close(y, (value, bound), dt, "y")
    if not train:
        m.intact()
        return
    want = R.ffn_gates(dy, wd, gate, up)
    dgate, dup = (gate, up) if in_place else (m.out(t, f, dtype=dt), m.out(t, f, dtype=dt))
    dx, dx_base = m.out(t, d, dtype=dt), m.normal(t, d, dtype=dt) if base else None
    if in_place and base:
        dx.copy_(dx_base)
    dwg, dwu, dwd = m.out(d, f, dtype=dt), m.out(d, f, dtype=dt), m.out(f, d, dtype=dt)
    B.ffn_backward(dy, x, gate, up, hidden, wg, wu, wd, dgate, dup, dx=dx, dx_base=dx if in_place and base else dx_base, dw_gate=dwg, dw_up=dwu, dw_down=dwd)
    close(dgate, want["dgate"], dt, "dgate")
    close(dup, want["dup"], dt, "dup")
    (v1, b1), (v2, b2) = R.product(dgate, wg.double().t()), R.product(dup, wu.double().t())
    bound = 2 * (2 * f + 32) * O.U32 * (dgate.double().abs() @ wg.double().t().abs() + dup.double().abs() @ wu.double().t().abs())
    value = v1 + v2
    if base:
        value, bound = value + dx_base.double(), bound + 2 * O.U32 * (value.abs() + dx_base.double().abs())
    close(dx, (value, bound), dt, "dx")
    close(dwg, R.product(x.t(), dgate), dt, "dw_gate")
    close(dwu, R.product(x.t(), dup), dt, "dw_up")
    close(dwd, R.product(hidden.t(), dy), dt, "dw_down")
    m.intact()


ODD = [(1, 1, 1), (1, 8, 8), (3, 5, 7), (17, 64, 128), (33, 72, 136), (31, 33, 65), (70, 129, 260), (130, 131, 383), (257, 40, 129), (5, 1027, 264), (300, 260, 1001)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t,d,f", ODD)
def test_ffn_of_any_size_and_address(B, dtype, t, d, f):
    run_ffn(B, Arena(t * 7 + d, shift=1), TYPES[dtype], t, d, f, base=t % 2 == 1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tile", list(ANY))
@pytest.mark.parametrize("split", [1, 2, 16])
def test_ffn_on_the_tiles_for_any_operand(B, forced, dtype, tile, split):
    forced(tile, split)
    run_ffn(B, Arena(split, shift=3), TYPES[dtype], 135, 139, 270, base=True)


@pytest.mark.parametrize("dtype,shift", [("bf16", 1), ("fp32", 0), ("fp32", 1)])
@pytest.mark.parametrize("tile", list(RING))
@pytest.mark.parametrize("split", [1, 4])
@pytest.mark.parametrize("t,d,f", [(1, 1, 1), (3, 33, 70), (130, 67, 131), (300, 515, 264)])
def test_ffn_on_the_ring_from_copies(B, forced, dtype, shift, tile, split, t, d, f):
    forced(tile, split)
    run_ffn(B, Arena(t + split, shift=shift), TYPES[dtype], t, d, f, base=split == 1)


@pytest.mark.parametrize("tile", list(RING))
@pytest.mark.parametrize("split", [1, 2, 8])
@pytest.mark.parametrize("t,d,f", [(1, 8, 8), (64, 64, 64), (130, 200, 328), (300, 264, 520), (600, 520, 264), (77, 1032, 136), (1030, 72, 776)])
def test_ffn_on_the_ring(B, forced, tile, split, t, d, f):
    forced(tile, split)
    run_ffn(B, Arena(t + split, shift=0), TYPES["bf16"], t, d, f, base=split == 2)


@pytest.mark.parametrize("t,d,f", [(1, 4096, 1032), (24, 1032, 4096), (2048, 512, 768), (4100, 128, 264)])
def test_ffn_as_chosen(B, t, d, f):
    run_ffn(B, Arena(t, shift=0), TYPES["bf16"], t, d, f)


@pytest.mark.parametrize("dtype,shift", [("bf16", 0), ("fp32", 1)])
def test_ffn_in_place_and_without_gradients(B, dtype, shift):
    run_ffn(B, Arena(5, shift=shift), TYPES[dtype], 40, 64, 96, base=True, in_place=True)
    run_ffn(B, Arena(6, shift=shift), TYPES[dtype], 40, 64, 96, base=True, in_place=True, train=False)


def test_ffn_parts_of_the_gradient(B):
    """Each gradient alone has the bits that it has among the others."""
    m = Arena(8, shift=0)
    t, d, f, dt = 70, 64, 136, torch.bfloat16
    x, dy, gate, up, hidden = m.normal(t, d, dtype=dt), m.normal(t, d, dtype=dt), *(m.normal(t, f, dtype=dt) for _ in range(3))
    w = [m.normal(d, f, dtype=dt), m.normal(d, f, dtype=dt), m.normal(f, d, dtype=dt)]
    dgate, dup = m.out(t, f, dtype=dt), m.out(t, f, dtype=dt)
    full = dict(dx=m.out(t, d, dtype=dt), dw_gate=m.out(d, f, dtype=dt), dw_up=m.out(d, f, dtype=dt), dw_down=m.out(f, d, dtype=dt))
    B.ffn_backward(dy, x, gate, up, hidden, *w, dgate, dup, **full)
    for name, whole in full.items():
        one = torch.empty_like(whole)
        B.ffn_backward(dy, x if "dw_" in name else None, gate, up, hidden if name == "dw_down" else None, w[0], w[1], w[2], dgate, dup, **{name: one})
        assert torch.equal(one, whole), name
    m.intact()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_tokens(B, dtype):
    dt = TYPES[dtype]
    m = Arena(1, shift=0)
    e = lambda *s: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    wg, wu, wd = m.normal(16, 24, dtype=dt), m.normal(16, 24, dtype=dt), m.normal(24, 16, dtype=dt)
    B.ffn_forward(e(0, 16), e(0, 16), wg, wu, wd, e(0, 24), gate=e(0, 24), up=e(0, 24))
    out = [m.out(16, 24, dtype=dt), m.out(16, 24, dtype=dt), m.out(24, 16, dtype=dt)]
    B.ffn_backward(e(0, 16), e(0, 16), e(0, 24), e(0, 24), e(0, 24), wg, wu, wd, e(0, 24), e(0, 24), dx=e(0, 16), dw_gate=out[0], dw_up=out[1], dw_down=out[2])
    dw = m.out(40, 16, dtype=dt)
    i32, f32 = (torch.empty(0, dtype=k, device="cuda") for k in (torch.int32, torch.float32))
    w = m.normal(40, 16, dtype=dt)
    B.head_loss_forward(e(0, 16), w, i32, f32, f32.clone())
    B.head_loss_backward(e(0, 16), w, i32, f32, dx=e(0, 16), dweight=dw)
    for g in out + [dw]:
        assert bool((g == 0).all())
    m.intact()


def test_ffn_of_large_and_infinite_gates(B):
    """Gates far out on both sides, where 1 + exp(-gate) overflows or is 1: the definition's values, and no NaN of finite inputs' making."""
    for dt, shift in ((torch.bfloat16, 0), (torch.float32, 1)):
        m = Arena(4, shift=shift)
        x = m.put(torch.tensor([[-300.0], [-90.0], [-1.0], [0.0], [1.0], [90.0], [300.0]]).repeat(1, 8).to(dt))
        wg, wu, wd = (m.put(torch.eye(8).to(dt)) for _ in range(3))
        y, hidden, gate, up = (m.out(7, 8, dtype=dt) for _ in range(4))
        B.ffn_forward(x, y, wg, wu, wd, hidden, gate=gate, up=up)
        a, slope = R.silu(x.double())
        O.check(hidden, a * x.double(), O.half_step(dt) * (a * x.double()).abs() + 2000 * O.U32 * (a * x.double()).abs() + 1e-30, "hidden")
        dgate, dup, dx = (m.out(7, 8, dtype=dt) for _ in range(3))
        B.ffn_backward(x, x, gate, up, hidden, wg, wu, wd, dgate, dup, dx=dx)
        want = x.double() ** 2 * slope
        O.check(dgate, want, O.half_step(dt) * want.abs() + 2000 * O.U32 * (want.abs() + x.double().abs() ** 2 * a.abs()) + 1e-30, "dgate")
        assert bool(torch.isfinite(dx).all())
        m.intact()


# ---- the head's loss -------------------------------------------------------------------------------------------------


def run_head(B, m, dt, t, d, v, weighted=False, scale=0.25, ids=None):
    x, w = m.normal(t, d, dtype=dt), m.normal(v, d, dtype=dt, std=2 * d ** -0.5)
    if ids is None:
        ids = torch.randint(0, v, (t,), generator=m.rng)
        none = torch.tensor([-100, -1, v, 2 ** 31 - 1, -2 ** 31])
        ids = torch.where(torch.rand(t, generator=m.rng) < 0.3, none[torch.randint(0, 5, (t,), generator=m.rng)], ids)
        if t > 3:
            ids[1], ids[2] = 0, v - 1
    ids = ids.to(torch.int32).cuda()
    loss, lse = m.out(t), m.out(t)
    B.head_loss_forward(x, w, ids, loss, lse)
    want = R.head_loss(x, w, ids)
    for got, name in ((loss, "loss"), (lse, "lse")):
        O.check(got, want[name][0], want[name][1], name)
    has = (ids >= 0) & (ids < v)
    assert bool((loss[~has] == 0).all())
    dloss = m.put(torch.rand(t, generator=m.rng) * 2 - 0.5) if weighted else None
    dx, dw = m.out(t, d, dtype=dt), m.out(v, d, dtype=dt)
    B.head_loss_backward(x, w, ids, lse, dx=dx, dweight=dw, dloss=dloss, scale=scale)
    want = R.head_gradients(x, w, ids, lse, dloss, scale)
    close(dx, want["dx"], dt, "dx")
    close(dw, want["dw"], dt, "dw")
    assert bool((dx[~has] == 0).all())
    one, other = torch.empty_like(dx), torch.empty_like(dw)
    B.head_loss_backward(x, w, ids, lse, dx=one, dloss=dloss, scale=scale)
    B.head_loss_backward(x, w, ids, lse, dweight=other, dloss=dloss, scale=scale)
    assert torch.equal(one, dx) and torch.equal(other, dw)
    m.intact()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t,d,v", [(1, 1, 1), (1, 8, 3), (2, 5, 2), (7, 33, 31), (33, 64, 128), (65, 40, 257), (130, 129, 1000), (300, 67, 130), (3, 515, 5003), (513, 9, 70)])
def test_head_of_any_size_and_address(B, dtype, t, d, v):
    run_head(B, Arena(t + v, shift=1), TYPES[dtype], t, d, v, weighted=t % 2 == 1)


@pytest.mark.parametrize("tile", list(RING))
@pytest.mark.parametrize("t,d,v", [(1, 64, 40), (70, 136, 257), (300, 64, 1003), (257, 520, 130), (64, 32, 2050)])
def test_head_on_the_ring(B, forced, tile, t, d, v):
    forced(tile)
    run_head(B, Arena(t + v, shift=0), TYPES["bf16"], t, d, v, weighted=t % 2 == 1)


@pytest.mark.parametrize("dtype,shift", [("bf16", 1), ("fp32", 0), ("fp32", 1)])
@pytest.mark.parametrize("tile", list(RING))
@pytest.mark.parametrize("t,d,v", [(1, 9, 3), (70, 67, 257), (300, 64, 1003)])
def test_head_on_the_ring_from_copies(B, forced, dtype, shift, tile, t, d, v):
    forced(tile)
    run_head(B, Arena(t + v, shift=shift), TYPES[dtype], t, d, v, weighted=t % 2 == 1)


def test_head_forward_in_pieces(B, forced):
    """Rows so wide that the forward pass takes the vocabulary in pieces too, from copies and in place."""
    run_head(B, Arena(8, shift=0), torch.bfloat16, 5, 40000, 4100)
    forced("ring 128")
    run_head(B, Arena(8, shift=1), torch.float32, 3, 32771, 4097)


@pytest.mark.parametrize("tile", list(RING) + list(ANY))
@pytest.mark.parametrize("split", [2, 16])
def test_head_with_k_splits(B, forced, tile, split):
    forced(tile, split)
    run_head(B, Arena(split, shift=0), TYPES["bf16"], 140, 72, 1050)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_head_in_pieces(B, dtype):
    """A batch so long that the vocabulary is taken in three pieces, the last one narrow and odd."""
    run_head(B, Arena(11, shift=0), TYPES[dtype], 65600, 8, 2051, scale=1.0 / 64)


def test_head_as_chosen(B):
    run_head(B, Arena(2, shift=0), torch.bfloat16, 2048, 256, 4096)
    run_head(B, Arena(3, shift=0), torch.bfloat16, 1, 4096, 3000)


def test_head_without_any_target(B):
    m = Arena(7, shift=0)
    run_head(B, m, torch.bfloat16, 40, 64, 300, ids=torch.full((40,), -100))


def test_head_ignores_what_a_token_without_a_target_holds(B):
    """NaN and infinities in rows without a target reach their own lse alone."""
    for dt, shift in ((torch.bfloat16, 0), (torch.float32, 1)):
        m = Arena(9, shift=shift)
        x, w = m.normal(40, 64, dtype=dt), m.normal(300, 64, dtype=dt, std=0.1)
        ids = torch.randint(0, 300, (40,), generator=m.rng).to(torch.int32).cuda()
        ids[::4] = -100
        loss, lse = m.out(40), m.out(40)
        x[0, 3], x[4, :] = float("nan"), float("inf")
        B.head_loss_forward(x, w, ids, loss, lse)
        assert bool((loss[::4] == 0).all()) and bool(torch.isfinite(loss).all())
        assert bool(torch.isnan(lse[0])) and bool(torch.isfinite(lse[8:]).all())
        dx, dw = m.out(40, 64, dtype=dt), m.out(300, 64, dtype=dt)
        B.head_loss_backward(x, w, ids, lse, dx=dx, dweight=dw)
        assert bool((dx[::4] == 0).all()) and bool(torch.isfinite(dx).all())
        clean, other, also = x.clone(), torch.empty_like(lse), torch.empty_like(dw)
        clean[::4] = 0
        B.head_loss_forward(clean, w, ids, lse=other)
        B.head_loss_backward(clean, w, ids, other, dweight=also)
        assert torch.equal(dw, also)
        # and with a target the NaN is seen
        ids[0] = 5
        B.head_loss_forward(x, w, ids, loss, lse)
        assert bool(torch.isnan(loss[0])) and bool(torch.isfinite(loss[1:]).all())
        m.intact()


def test_head_of_large_logits(B):
    """Logits of hundreds: the largest is taken out before the exponential, over every range of columns and in what joins them."""
    for dt, shift in ((torch.bfloat16, 0), (torch.float32, 1)):
        m = Arena(12, shift=shift)
        x, w = m.normal(33, 16, dtype=dt, std=30.0), m.normal(700, 16, dtype=dt, std=3.0)
        ids = torch.randint(0, 700, (33,), generator=m.rng).to(torch.int32).cuda()
        loss, lse = m.out(33), m.out(33)
        B.head_loss_forward(x, w, ids, loss, lse)
        want = R.head_loss(x, w, ids)
        for got, name in ((loss, "loss"), (lse, "lse")):
            O.check(got, want[name][0], want[name][1], name)
        m.intact()


@pytest.mark.parametrize("dtype,shift", [("bf16", 0), ("bf16", 1), ("fp32", 0), ("fp32", 1)])
@pytest.mark.parametrize("t,d,v", [(1, 512, 900), (50, 256, 3000), (300, 136, 5003), (1100, 64, 2500)])
def test_head_gradients_of_nearly_certain_targets(B, dtype, shift, t, d, v):
    """1 - p of a target that has nearly all of it is small: both passes have to have the same logits, and the loss is not lse - z."""
    dt = TYPES[dtype]
    m = Arena(t + v, shift=shift)
    w = m.normal(v, d, dtype=dt, std=d ** -0.5)
    ids = torch.randint(0, v, (t,), generator=m.rng).cuda()
    lean = torch.linspace(14, 24, t)[:, None].cuda()          # the target's logit above the others', whose log of the sum is 7 to 9
    x = m.put((torch.randn(t, d, generator=m.rng).cuda() + lean * w[ids].float() / w[ids].float().square().sum(1, keepdim=True)).to(dt))
    ids = ids.to(torch.int32)
    loss, lse = m.out(t), m.out(t)
    B.head_loss_forward(x, w, ids, loss, lse)
    z, e = R.head_logits(x, w)
    certain = torch.logsumexp(z, 1)
    want = certain - z[torch.arange(t), ids.long()]
    p = torch.exp(-want)
    # the loss moves by (1 - p) times the errors of the logits; its logarithm and difference are of numbers near it, the ranges' sums of ones near 1
    O.check(loss, want, 3 * (1 - p) * e.amax(1) + (40 + 4 * want) * O.U32, "loss")
    assert float(want.min()) < (1e-2 if t == 1 else 1e-4)    # (a property of the inputs)
    dx, dw = m.out(t, d, dtype=dt), m.out(v, d, dtype=dt)
    B.head_loss_backward(x, w, ids, lse, dx=dx, dweight=dw)
    want = R.head_gradients_of_one_pass(x, w, ids, None, 1.0)
    close(dx, want["dx"], dt, "dx")
    close(dw, want["dw"], dt, "dw")
    m.intact()


@pytest.mark.parametrize("split", [1, 3])
@pytest.mark.parametrize("dtype,shift,tiles", [("bf16", 0, [*RING]), ("bf16", 1, [*RING]), ("bf16", 1, [*ANY]), ("fp32", 0, ["ring 128", "ring 64"]), ("fp32", 0, [*ANY])])
def test_logits_have_the_same_bits_on_every_tile(B, forced, dtype, shift, tiles, split):
    """One column of ranges and one token: lse and dweight are functions of the logits alone."""
    dt = TYPES[dtype]
    m = Arena(6, shift=shift)
    x, w, ids = m.normal(1, 1496, dtype=dt), m.normal(20, 1496, dtype=dt, std=0.1), torch.tensor([7], dtype=torch.int32, device="cuda")
    seen = []
    for tile in tiles:
        forced(tile, split)
        lse, dw = m.out(1), m.out(20, 1496, dtype=dt)
        B.head_loss_forward(x, w, ids, lse=lse)
        B.head_loss_backward(x, w, ids, lse, dweight=dw)
        seen.append((lse, dw))
    for tile, (lse, dw) in zip(tiles[1:], seen[1:]):
        assert torch.equal(lse, seen[0][0]), tile
        # (a gradient of weights has no tile of 64 rows: in fp32 its own sums are then those of another kernel)
        assert torch.equal(dw, seen[0][1]) or (dtype == "fp32" and tile == "ring 64"), tile


def test_head_gradients_against_differences(B):
    """Along a direction the loss changes as the gradients say, in fp32 with the differences in 64 bits of the oracle's logits."""
    m = Arena(13, shift=0)
    t, d, v = 20, 24, 50
    x, w, ids = m.normal(t, d), m.normal(v, d, std=0.4), torch.randint(-2, v, (t,), generator=m.rng).to(torch.int32).cuda()
    lse, loss, dx, dw = m.out(t), m.out(t), m.out(t, d), m.out(v, d)
    B.head_loss_forward(x, w, ids, loss, lse)
    B.head_loss_backward(x, w, ids, lse, dx=dx, dweight=dw)
    px, pw = torch.randn(t, d, generator=m.rng).double().cuda(), torch.randn(v, d, generator=m.rng).double().cuda()
    h = 1e-4
    f = lambda s: float(R.head_loss(x.double() + s * h * px, w.double() + s * h * pw, ids)["loss"][0].sum())  # noqa: E731
    slope = (f(1) - f(-1)) / (2 * h)
    said = float((dx.double() * px).sum() + (dw.double() * pw).sum())
    # the third derivative of a log-sum-exp along a direction is below 4 (largest |dz|)^3: of z's change here
    dz = (px @ w.double().t() + x.double() @ pw.t()).abs().amax(1)
    second = 2 * (px @ pw.t()).abs().amax(1)
    curve = float((4 * (dz + second) ** 3 + 6 * (dz + second) * second).sum())
    want = R.head_gradients(x, w, ids, lse, None, 1.0)
    off = float((want["dx"][1] * px.abs()).sum() + (want["dw"][1] * pw.abs()).sum())
    assert abs(slope - said) <= curve * h * h + 1e-9 / h + off + 2 * O.U32 * abs(said) + float((dx.abs().double() * px.abs()).sum() + (dw.abs().double() * pw.abs()).sum()) * O.U32


def test_ffn_gradients_against_differences(B):
    m = Arena(14, shift=0)
    t, d, f = 9, 16, 24
    x, dy, wg, wu, wd = m.normal(t, d), m.normal(t, d), m.normal(d, f, std=0.3), m.normal(d, f, std=0.3), m.normal(f, d, std=0.3)
    y, hidden, gate, up, dgate, dup, dx = m.out(t, d), *(m.out(t, f) for _ in range(5)), m.out(t, d)
    dws = [m.out(d, f), m.out(d, f), m.out(f, d)]
    B.ffn_forward(x, y, wg, wu, wd, hidden, gate=gate, up=up)
    B.ffn_backward(dy, x, gate, up, hidden, wg, wu, wd, dgate, dup, dx=dx, dw_gate=dws[0], dw_up=dws[1], dw_down=dws[2])
    held = [x, wg, wu, wd]
    ways = [torch.randn(v.shape, generator=m.rng).double().cuda() for v in held]

    def value(s):
        a, b, c, e = (v.double() + s * w for v, w in zip(held, ways))
        return float(((R.silu(a @ b)[0] * (a @ c)) @ e * dy.double()).sum())
    # Richardson's: the differences at h and h / 2 leave an error of the fourth order, seen in how they differ
    h = 1e-3
    d1, d2 = (value(h) - value(-h)) / (2 * h), (value(h / 2) - value(-h / 2)) / h
    slope = (4 * d2 - d1) / 3
    said = sum(float((g.double() * w).sum()) for g, w in zip([dx] + dws, ways))
    size = sum(float((g.double().abs() * w.abs()).sum()) for g, w in zip([dx] + dws, ways))
    # fp32 chains of at most 2 (d + f) products, three deep
    assert abs(slope - said) <= abs(d1 - d2) + 1e-8 + 12 * (d + f) * O.U32 * size * 4


# ---- clipping --------------------------------------------------------------------------------------------------------


def check_clip(B, m, grads, max_norm, eps=1e-6, in_place=False):
    norm = m.out(1)
    before = [g.clone() for g in grads]
    out = grads if in_place else [m.out(*g.shape, dtype=g.dtype) for g in grads]
    B.clip_gradients(grads, norm, max_norm, eps=eps, out=None if in_place else out)
    want, c = R.clip(before, max_norm, eps)
    assert abs(float(norm) - want) <= 2 * O.U32 * want
    for o, b in zip(out, before):
        O.check(o, b.double() * c, O.half_step(o.dtype) * (b.double() * c).abs() + 4 * O.U32 * (b.double() * c).abs() + 1e-45, "out")
        if c == 1.0:
            assert torch.equal(o, b)
    if not in_place:
        for g, b in zip(grads, before):
            assert torch.equal(g, b)
    m.intact()
    return norm


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("sizes", [[1], [7], [8], [2047], [16384], [16385, 1, 8191], [3] * 121, list(range(1, 300)), [40000, 5, 70001], [9] * 500])
def test_clip(B, sizes, in_place):
    for shift in (0, 1):
        m = Arena(len(sizes) + sizes[0], shift=shift)
        grads = [m.normal(n, dtype=(torch.bfloat16, torch.float32)[i % 2]) for i, n in enumerate(sizes)]
        check_clip(B, m, grads, 0.5, in_place=in_place)
    check_clip(B, m, grads, 1e6, in_place=in_place)


def test_clip_of_a_large_list(B):
    m = Arena(4, shift=0)
    check_clip(B, m, [m.normal(3000, 4001, dtype=torch.bfloat16), m.normal(7, 3), m.normal(2000, 5003), m.normal(12345, dtype=torch.bfloat16)], 1.0)


def test_clip_of_nothing(B):
    norm = torch.full((1,), float("nan"), device="cuda")
    B.clip_gradients([], norm, 1.0)
    assert float(norm) == 0
    norm.fill_(float("nan"))
    empty = torch.empty(0, 5, device="cuda")
    B.clip_gradients([empty, empty], norm, 1.0)
    assert float(norm) == 0
    m = Arena(1)
    check_clip(B, m, [m.normal(5), empty, m.normal(3, dtype=torch.bfloat16)], 0.1)
    check_clip(B, m, [m.put(torch.zeros(40))], 1.0, eps=0.0)
    check_clip(B, m, [m.normal(40)], 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("std", [1e30, 1e-30, 1e-38])
def test_clip_at_the_ends_of_the_range(B, dtype, std):
    """Squares beyond fp32 on either side."""
    m = Arena(3)
    grads = [m.normal(5000, dtype=TYPES[dtype], std=std), m.normal(70, 9, std=std)]
    check_clip(B, m, grads, 1.0, eps=0.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("std,max_norm", [(1e30, 1e-12), (1e37, 1e-8), (1e36, 1e-38), (1e20, 1e-30)])
def test_clip_by_a_factor_below_normal_numbers(B, dtype, std, max_norm):
    """The factor alone would be a subnormal number of a few bits; what it scales to is an ordinary one, or nothing."""
    m = Arena(5)
    grads, norm = [m.normal(5000, dtype=TYPES[dtype], std=std), m.normal(70, 9, std=std)], m.out(1)
    out = [m.out(*g.shape, dtype=g.dtype) for g in grads]
    B.clip_gradients(grads, norm, max_norm, eps=0.0, out=out)
    want, c = R.clip(grads, max_norm, 0.0)
    # 5630 normal numbers of 1e37: their norm is 7.4e38, beyond the largest fp32 of 3.4e38, and the factor is none the less 1e-8 of its inverse
    if want > torch.finfo(torch.float32).max:
        assert float(norm) == float("inf")
    else:
        assert abs(float(norm) - want) <= 2 * O.U32 * want
    for o, g in zip(out, grads):
        # half a step of the type, of the factor and of the product, and half of the smallest numbers' step (1.4e-45, in bf16 9.2e-41)
        size = (g.double() * c).abs()
        O.check(o, g.double() * c, O.half_step(o.dtype) * size + 4 * O.U32 * size + (5e-41 if o.dtype == torch.bfloat16 else 1e-45), "out")
    m.intact()


def test_clip_of_infinities_and_nan(B):
    inf = float("inf")
    m = Arena(6)
    g, h = m.normal(300), m.normal(1000, dtype=torch.bfloat16)
    norm = m.out(1)
    h[7] = inf
    out = [torch.empty_like(g), torch.empty_like(h)]
    B.clip_gradients([g, h], norm, 1.0, out=out)
    assert float(norm) == inf and bool((out[0] == 0).all()) and bool(torch.isnan(out[1][7])) and int(torch.isnan(out[1]).sum()) == 1
    B.clip_gradients([g, h], norm, inf, out=out)
    assert float(norm) == inf and torch.equal(out[0], g) and torch.equal(out[1], h)
    g[0] = float("nan")
    B.clip_gradients([g, h], norm, 1.0, out=out)
    assert bool(torch.isnan(norm).all()) and bool(torch.isnan(out[0]).all()) and bool(torch.isnan(out[1]).all())
    B.clip_gradients([g, h], norm, inf)
    assert bool(torch.isnan(norm).all()) and int(torch.isnan(g).sum()) == 1 and float(h[7]) == inf


def test_clip_of_a_tensor_listed_twice(B):
    m = Arena(2)
    g = m.normal(100)
    check_clip(B, m, [g, g], 0.5)
    with pytest.raises(B.CmoeError, match="overlaps"):
        B.clip_gradients([g, g], m.out(1), 0.5)


# ---- streams and graphs ----------------------------------------------------------------------------------------------


def step_of(B, dt, t, d, f, v, m):
    """A run of all operators, as a training step makes it: its outputs' buffers and the call."""
    s = {k: m.normal(*shape, dtype=dt, std=std) for k, shape, std in (
        ("x", (t, d), 1.0), ("wg", (d, f), d ** -0.5), ("wu", (d, f), d ** -0.5), ("wd", (f, d), f ** -0.5), ("w", (v, d), d ** -0.5))}
    s["ids"] = torch.randint(-5, v, (t,), generator=m.rng).to(torch.int32).cuda()
    o = {k: torch.empty(*shape, dtype=kind, device="cuda") for k, shape, kind in (
        ("y", (t, d), dt), ("hidden", (t, f), dt), ("gate", (t, f), dt), ("up", (t, f), dt), ("dgate", (t, f), dt), ("dup", (t, f), dt), ("dx", (t, d), dt),
        ("dy", (t, d), dt), ("dwg", (d, f), dt), ("dwu", (d, f), dt), ("dwd", (f, d), dt), ("dw", (v, d), dt), ("loss", (t,), torch.float32),
        ("lse", (t,), torch.float32), ("norm", (1,), torch.float32))}

    def call():
        B.ffn_forward(s["x"], o["y"], s["wg"], s["wu"], s["wd"], o["hidden"], gate=o["gate"], up=o["up"], base=s["x"])
        B.head_loss_forward(o["y"], s["w"], s["ids"], o["loss"], o["lse"])
        B.head_loss_backward(o["y"], s["w"], s["ids"], o["lse"], dx=o["dy"], dweight=o["dw"], scale=1.0 / t)
        B.ffn_backward(o["dy"], s["x"], o["gate"], o["up"], o["hidden"], s["wg"], s["wu"], s["wd"], o["dgate"], o["dup"], dx=o["dx"], dx_base=o["dy"],
                       dw_gate=o["dwg"], dw_up=o["dwu"], dw_down=o["dwd"])
        B.clip_gradients([o[k] for k in ("dwg", "dwu", "dwd", "dw")], o["norm"], 0.01)
    return s, o, call


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_step_against_autograd(B, dtype):
    """Block, loss, gradients and clipping together against torch's autograd in 64 bits: forward rounding of every stored tensor moves the
    gradients by a few roundings of the type relative to their norm."""
    dt = TYPES[dtype]
    t, d, f, v = 150, 64, 136, 500
    s, o, call = step_of(B, dt, t, d, f, v, Arena(21, shift=0))
    call()
    held = {k: s[k].double().requires_grad_() for k in ("x", "wg", "wu", "wd", "w")}
    g = held["x"] @ held["wg"]
    y = held["x"] + (g * torch.sigmoid(g) * (held["x"] @ held["wu"])) @ held["wd"]
    z = y @ held["w"].t()
    ids = s["ids"].long()
    loss = torch.nn.functional.cross_entropy(z, torch.where(ids < 0, -100, ids), ignore_index=-100, reduction="sum") / t
    loss.backward()
    norm = sum(float(held[k].grad.square().sum()) for k in ("wg", "wu", "wd", "w")) ** 0.5
    c = min(1.0, 0.01 / norm)
    # seven tensors are stored on the way to the last gradient; each rounding is at most half a step of its value, and what they do
    # to logits of order one goes through a softmax, whose slope is at most one
    tol = 16 * O.half_step(dt) if dt is torch.bfloat16 else 400 * O.U32
    assert abs(float(o["norm"]) - norm) <= tol * norm
    for k, got in (("x", o["dx"]), ("wg", o["dwg"]), ("wu", o["dwu"]), ("wd", o["dwd"]), ("w", o["dw"])):
        want = held[k].grad * (1.0 if k == "x" else c)
        assert float((got.double() - want).norm()) <= tol * float(want.norm()), k


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_step_on_other_streams_and_in_graphs(B, dtype):
    """The same bits on a stream of one's own, from two graphs that share a pool of memory, replayed among eager work, and from run to run."""
    dt = TYPES[dtype]
    runs = [step_of(B, dt, t, 72, 264, 1003, Arena(t, shift=0)) for t in (40, 333)]
    want = []
    for _, o, call in runs:
        call()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in o.items()})

    def same(i):
        torch.cuda.synchronize()
        for k, v in runs[i][1].items():
            assert torch.equal(v, want[i][k]), k

    def blank(i):
        for v in runs[i][1].values():
            v.fill_(float("nan"))
        torch.cuda.synchronize()

    stream = torch.cuda.Stream()
    for i in range(2):
        blank(i)
        with torch.cuda.stream(stream):
            runs[i][2]()
        same(i)
    graphs, pool = [], torch.cuda.graph_pool_handle()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            runs[i][2]()
        graphs.append(g)
    for turn in range(3):
        for i in ((0, 1), (1, 0), (0, 1))[turn]:
            blank(i)
            graphs[i].replay()
            same(i)
        runs[turn % 2][2]()
        same(turn % 2)
