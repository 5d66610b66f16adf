"""The norm, dropout and adapters on the GPU against their definitions in 64 bits (operator_oracle.py holds both and the bounds).

Every tensor lies inside a larger buffer of NaN at an address with only an element's alignment, so that what a kernel reads past a
row shows in its results and what it writes past one shows in the buffer."""
import numpy as np
import pytest
import torch

import operator_oracle as O

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
PAD = 24


@pytest.fixture(scope="module")
def B():
    from paper_2502_04416_amd import binding as b
    b.load()
    return b


class Arena:
    """Tensors with NaN around them."""

    def __init__(self, seed, shift=1):
        self.rng = torch.Generator().manual_seed(seed)
        self.shift = shift
        self.held = []

    def put(self, value):
        n = value.numel()
        if value.dtype == torch.int32:
            return value.cuda()
        buf = torch.full((n + 2 * PAD,), float("nan"), dtype=value.dtype, device="cuda")
        t = buf[PAD - self.shift:PAD - self.shift + n].view(value.shape)
        t.copy_(value)
        self.held.append((buf, PAD - self.shift, n))
        return t

    def normal(self, *shape, dtype=torch.float32, std=1.0, mean=0.0):
        return self.put((torch.randn(*shape, generator=self.rng) * std + mean).to(dtype))

    def out(self, *shape, dtype=torch.float32):
        return self.put(torch.full(shape, float("nan"), dtype=dtype))

    def intact(self):
        for buf, at, n in self.held:
            assert bool(torch.isnan(buf[:at]).all()) and bool(torch.isnan(buf[at + n:]).all()), "written outside of a tensor"


# ---- dropout ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols,p,residual", [
    (1, 1, 0.5, False), (1, 7, 0.3, True), (3, 8, 0.1, False), (5, 9, 0.25, True), (64, 256, 0.1, False), (37, 1027, 0.02, True), (2, 70001, 0.6, False),
    (1025, 40, 0.9, True), (70001, 3, 0.4, False), (4, 64, 0.0, True), (4, 65, 1.0, True), (4, 64, 1.0, False), (3, 24, 1e-6, False), (3, 24, 1 - 1e-9, False),
])
def test_dropout(B, dtype, rows, cols, p, residual):
    dt = TYPES[dtype]
    m = Arena(rows * 7 + cols)
    x, y = m.normal(rows, cols, dtype=dt), m.out(rows, cols, dtype=dt)
    res = m.normal(rows, cols, dtype=dt) if residual else None
    drop = B.Dropout(p, (cols << 40) + 17 * rows, (1 << 35) + rows)
    mk = O.mask(rows, cols, drop, "cuda")
    x[mk == 0] = float("nan")                               # a dropped element is 0 whatever it was
    B.dropout(x, y, drop, residual=res)
    want, tol = O.norm_sum(x, res, mk)
    O.check(y, want, tol, "y")
    if not residual:
        assert torch.equal(y == 0, (mk == 0) | (x == 0))
    m.intact()


def test_dropout_in_place_and_backward(B):
    m = Arena(3)
    x, res = m.normal(33, 100), m.normal(33, 100)
    drop = B.Dropout(0.4, 99, 5)
    y, z, g, dx = m.out(33, 100), res.clone(), m.normal(33, 100), m.out(33, 100)
    B.dropout(x, y, drop, residual=res)
    B.dropout(x, z, drop, residual=z)
    assert torch.equal(y, z)
    B.dropout(g, dx, drop)
    # y is linear in x: the difference along a direction is the gradient's product with it
    way = m.normal(33, 100)
    y2 = m.out(33, 100)
    B.dropout((x + way).contiguous(), y2, drop, residual=res)
    lhs, rhs = ((y2 - y).double() * g.double()).sum(), (dx.double() * way.double()).sum()
    size = ((y2.abs() + y.abs() + x.abs() + way.abs()).double() * g.double().abs()).sum() * drop_scale(0.4)
    assert abs(float(lhs - rhs)) <= 4 * O.U32 * float(size)
    B.dropout(x, x, drop)
    assert torch.equal(x != 0, O.mask(33, 100, drop, "cuda") != 0)
    m.intact()


def drop_scale(p):
    return 65536 / (65536 - round(p * 65536))


# ---- norm ------------------------------------------------------------------------------------------------------------

NORM_CASES = [
    # rows, cols, form, residual, p, weight, bias: every number of threads per row and chunks per thread, full and ragged
    (1, 1, "layer", False, 0.0, True, True), (3, 5, "rms", True, 0.0, True, False), (17, 8, "layer", False, 0.3, False, True),
    (33, 128, "rms", True, 0.1, True, True), (5, 129, "layer", True, 0.2, True, False), (7, 512, "rms", False, 0.0, False, False),
    (9, 515, "layer", True, 0.1, True, True), (6, 1024, "rms", True, 0.0, True, False), (333, 1027, "layer", False, 0.0, True, True),
    (2, 2048, "layer", True, 0.1, True, True), (1, 2055, "rms", True, 0.0, True, False), (4, 4096, "layer", True, 0.1, True, True),
    (1200, 1001, "rms", False, 0.0, True, True), (3, 4103, "rms", False, 0.5, True, False), (2, 8192, "layer", True, 0.0, True, True),
    (3, 8200, "layer", False, 0.1, True, True), (2, 16384, "rms", True, 0.1, True, False), (2, 16390, "layer", True, 0.0, True, True),
    (1, 32768, "rms", False, 0.0, True, False), (2, 32761, "layer", True, 0.3, True, True), (5000, 72, "layer", True, 0.1, True, True),
    (1027, 4096, "rms", True, 0.1, True, False),
]


def run_norm(B, m, dt, rows, cols, form, residual, p, weight, bias, mean_of_x=0.5):
    drop = B.Dropout(p, 1234567890123, (1 << 33) + cols) if p > 0 else None
    mk = O.mask(rows, cols, drop, "cuda")
    x = m.normal(rows, cols, dtype=dt, mean=mean_of_x)
    res = m.normal(rows, cols, dtype=dt, std=2.0) if residual else None
    w, b = (m.normal(cols, dtype=dt, std=0.2, mean=1.0) if weight else None), (m.normal(cols, dtype=dt) if bias else None)
    y, mean, rstd = m.out(rows, cols, dtype=dt), m.out(rows), m.out(rows)
    stored = m.out(rows, cols, dtype=dt) if residual or p > 0 else None
    B.norm_forward(x, y, w, b, form=form, eps=1e-5, residual=res, dropout=drop, sum_out=stored, mean=mean, rstd=rstd)
    if stored is not None:
        want, tol = O.norm_sum(x, res, mk)
        O.check(stored, want, tol, "sum")
    s = x if stored is None else stored
    want, tol = O.norm_forward(s, w, b, form, 1e-5, dt)
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd)):
        O.check(got, want[name], tol[name], name)
    return x, res, w, b, s, y, mean, rstd, drop, mk


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", NORM_CASES, ids=lambda c: "-".join(map(str, c)))
def test_norm(B, dtype, case):
    rows, cols, form, residual, p, weight, bias = case
    dt = TYPES[dtype]
    m = Arena(rows + cols)
    x, res, w, b, s, y, mean, rstd, drop, mk = run_norm(B, m, dt, *case)
    dy, dsum = m.normal(rows, cols, dtype=dt), m.normal(rows, cols, dtype=dt) if residual else None
    dx, dres = m.out(rows, cols, dtype=dt), m.out(rows, cols, dtype=dt) if residual else None
    dw, db = m.out(cols), m.out(cols) if bias else None
    B.norm_backward(dy, s, dx, mean, rstd, w, form=form, dsum=dsum, dropout=drop, dresidual=dres, dweight=dw, dbias=db)
    want, tol = O.norm_backward(dy, s, mean, rstd, w, form, dsum, mk)
    for name, got in (("dx", dx), ("dresidual", dres), ("dweight", dw), ("dbias", db)):
        if got is not None:
            O.check(got, want[name], tol[name], name)
    again = m.out(cols)
    B.norm_backward(dy, s, dx, mean, rstd, w, form=form, dsum=dsum, dropout=drop, dresidual=dres, dweight=again)
    assert torch.equal(again, dw)                           # (a fixed order of sums)
    O.check(dx, want["dx"], tol["dx"], "dx without dbias")
    m.intact()


def test_norm_of_rows_that_differ_by_much(B):
    """A row of equal values, rows of 0, far from 0, tiny and large; infinities and NaN stay in their rows."""
    m = Arena(1)
    x = m.normal(8, 640)
    x[0], x[1], x[2], x[3] = 0.0, 7.0, x[2] + 1000.0, x[3] * 1e-12
    x[4] *= 1e15
    x[5, 3], x[6, 639] = float("inf"), float("nan")
    for form in ("layer", "rms"):
        y, mean, rstd = m.out(8, 640), m.out(8), m.out(8)
        B.norm_forward(x, y, form=form, mean=mean, rstd=rstd)
        keep = [0, 1, 2, 3, 4, 7]
        want, tol = O.norm_forward(x[keep], None, None, form, 1e-5, torch.float32)
        O.check(y[keep], want["y"], tol["y"] + 1e-30, form)
        assert bool((y[0] == 0).all()) and not bool(torch.isfinite(y[6]).any()) and bool(torch.isnan(rstd[6]))
        assert not bool(torch.isfinite(rstd[5])) or float(rstd[5]) == 0.0
    m.intact()


def test_norm_in_place(B):
    m = Arena(5, shift=0)
    x, res, w = m.normal(9, 384, dtype=torch.bfloat16), m.normal(9, 384, dtype=torch.bfloat16), m.normal(384, dtype=torch.bfloat16)
    drop = B.Dropout(0.2, 5, 6)
    y, s = m.out(9, 384, dtype=torch.bfloat16), m.out(9, 384, dtype=torch.bfloat16)
    B.norm_forward(x, y, w, residual=res, dropout=drop, sum_out=s)
    stream, out = res.clone(), x.clone()
    B.norm_forward(out, out, w, residual=stream, dropout=drop, sum_out=stream)
    assert torch.equal(out, y) and torch.equal(stream, s)
    mean, rstd, dx, dres = m.out(9), m.out(9), m.out(9, 384, dtype=torch.bfloat16), m.out(9, 384, dtype=torch.bfloat16)
    B.norm_forward(x, y, w, residual=res, dropout=drop, sum_out=s, mean=mean, rstd=rstd)
    dy = m.normal(9, 384, dtype=torch.bfloat16)
    B.norm_backward(dy, s, dx, mean, rstd, w, dsum=res, dropout=drop, dresidual=dres)
    g, ds = dy.clone(), res.clone()
    B.norm_backward(g, s, g, mean, rstd, w, dsum=ds, dropout=drop, dresidual=ds)
    assert torch.equal(g, dx) and torch.equal(ds, dres)


def test_norm_without_rows(B):
    z = torch.empty(0, 40, device="cuda")
    st, dw, db = torch.empty(0, device="cuda"), torch.full((40,), 7.0, device="cuda"), torch.full((40,), 7.0, device="cuda")
    B.norm_forward(z, z.clone(), mean=st, rstd=st.clone())
    B.norm_backward(z, z.clone(), z.clone(), st, st.clone(), dweight=dw, dbias=db)
    assert not dw.any() and not db.any()
    B.dropout(z, z.clone(), B.Dropout(0.5, 1))


@pytest.mark.parametrize("form", ["layer", "rms"])
def test_norm_gradients_are_differences(B, form):
    """d(sum of y * g) along a direction, by central differences of the forward pass.

    With |s| ~ 1, 96 columns and a step of h = 2^-6 along a unit-size direction the third-order term is below 4 h^2 of the
    gradient's size, and the roundings of two sums of n terms of size 1 are below 2^-24 * 8 * sqrt(n) / h."""
    m = Arena(8)
    rows, cols, h = 6, 96, 2.0 ** -6
    x, res, w, b = m.normal(rows, cols), m.normal(rows, cols), m.normal(cols, mean=1.0, std=0.2), m.normal(cols)
    g, drop = m.normal(rows, cols), B.Dropout(0.25, 31, 1)
    y, s, mean, rstd = m.out(rows, cols), m.out(rows, cols), m.out(rows), m.out(rows)

    def value(x, res, w, b):
        B.norm_forward(x, y, w, b, form=form, residual=res, dropout=drop, sum_out=s, mean=mean, rstd=rstd)
        return float((y.double() * g.double()).sum())

    value(x, res, w, b)
    dx, dres, dw, db = m.out(rows, cols), m.out(rows, cols), m.out(cols), m.out(cols)
    B.norm_backward(g, s.clone(), dx, mean.clone(), rstd.clone(), w, form=form, dropout=drop, dresidual=dres, dweight=dw, dbias=db)
    base = [x, res, w, b]
    for i, grad in enumerate((dx, dres, dw, db)):
        way = m.normal(*grad.shape)
        lo, hi = list(base), list(base)
        lo[i], hi[i] = (base[i] - h * way).contiguous(), (base[i] + h * way).contiguous()
        slope = (value(*hi) - value(*lo)) / (2 * h)
        want = float((grad.double() * way.double()).sum())
        size = float((grad.double() * way.double()).abs().sum())
        assert abs(slope - want) <= 4 * h * h * size + O.U32 * 8 * (rows * cols) ** 0.5 * 8 / h, (i, slope, want)


# ---- adapters --------------------------------------------------------------------------------------------------------

def make_ids(kind, t, n, rng):
    if kind == "runs":
        cuts = np.sort(rng.integers(0, t + 1, 4))
        return np.repeat(rng.integers(-1, n, 5), np.diff(np.concatenate([[0], cuts, [t]])))
    if kind == "mixed":
        return rng.integers(-1, n, t)
    if kind == "odd":                                        # ids that name no adapter
        return rng.choice([0, n - 1, n, n + 7, -1, -5, 2 ** 31 - 1, -2 ** 31], t)
    if kind == "none":
        return np.full(t, -1)
    return np.full(t, n - 1)                                 # "one"


ADAPTER_CASES = [
    # tokens, d_in, d_out, rank, bank, ids, p, base
    (1, 64, 64, 8, 1, "one", 0.0, True), (1, 1, 1, 1, 1, "one", 0.0, True), (1, 4096, 512, 8, 8, "one", 0.1, True), (2, 7, 9, 3, 2, "mixed", 0.3, False),
    (5, 33, 130, 4, 3, "mixed", 0.0, True), (16, 256, 128, 16, 4, "mixed", 0.1, True), (17, 250, 96, 12, 40, "mixed", 0.2, True),
    (31, 515, 257, 17, 3, "odd", 0.1, True), (33, 128, 1001, 24, 2, "one", 0.0, False), (64, 1000, 777, 33, 48, "mixed", 0.05, True),
    (100, 96, 2000, 64, 2, "runs", 0.1, True), (40, 64, 64, 8, 3, "none", 0.1, True), (130, 2056, 64, 1, 2, "runs", 0.0, True),
    (300, 320, 192, 8, 1, "one", 0.05, True), (513, 200, 136, 8, 5, "runs", 0.1, True), (700, 131, 67, 12, 3, "runs", 0.1, True),
    (777, 264, 300, 40, 64, "mixed", 0.1, True), (1100, 192, 520, 64, 2, "runs", 0.1, False), (1500, 512, 384, 16, 2, "odd", 0.0, True),
    (2100, 136, 264, 32, 7, "runs", 0.1, True), (4100, 72, 40, 8, 9, "mixed", 0.0, True), (520, 1500, 1030, 48, 4, "runs", 0.3, True),
]


def adapter_inputs(B, m, dt, case, shuffle=0):
    t, d_in, d_out, rank, bank, kind, p, with_base = case
    rng = np.random.default_rng(t * 31 + d_in)
    ids = [int(v) for v in make_ids(kind, t, bank, rng)]
    x, a = m.normal(t, d_in, dtype=dt), m.normal(bank, rank, d_in, dtype=dt, std=d_in ** -0.5)
    b, scale = m.normal(bank, d_out, rank, dtype=dt, std=0.3), m.normal(bank, mean=2.0)
    base = m.normal(t, d_out, dtype=dt) if with_base else None
    drop = B.Dropout(p, 777 + t, (1 << 34) + rank) if p > 0 else None
    mk = O.mask(t, d_in, drop, "cuda")
    # what must not be looked at: adapters that no token has, dropped elements
    for k in set(range(bank)) - set(ids):
        a[k], b[k], scale[k] = float("nan"), float("nan"), float("nan")
    x[mk == 0] = float("nan")
    return x, a, b, scale, torch.tensor(ids, dtype=torch.int32, device="cuda"), ids, base, drop, mk


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", ADAPTER_CASES, ids=lambda c: "-".join(map(str, c)))
def test_adapters(B, dtype, case):
    dt = TYPES[dtype]
    t, d_in, d_out, rank, bank, kind, p, with_base = case
    m = Arena(sum(case[:5]))
    x, a, b, scale, ids, id_list, base, drop, mk = adapter_inputs(B, m, dt, case)
    dy = m.normal(t, d_out, dtype=dt)
    dx_base = m.normal(t, d_in, dtype=dt) if with_base else None
    # what has no adapter takes no part, whatever it holds
    idle = [i for i, k in enumerate(id_list) if not 0 <= k < bank]
    x[idle] = float("nan")
    dy[idle] = float("nan")
    y, u = m.out(t, d_out, dtype=dt), m.out(t, rank)
    B.adapters_forward(x, y, a, b, scale, ids=ids, base=base, dropout=drop, u=u)
    dx, da, db = m.out(t, d_in, dtype=dt), m.out(bank, rank, d_in), m.out(bank, d_out, rank)
    B.adapters_backward(dy, x, u, a, b, scale, ids=ids, dx=dx, dx_base=dx_base, dropout=drop, da=da, db=db)
    want, tol = O.adapters(x, dy, a, b, scale, id_list, base, dx_base, mk)
    for name, got in (("u", u), ("y", y), ("dx", dx), ("da", da), ("db", db)):
        O.check(got, want[name], tol[name], name)
    for name, got, n in (("da", da, t), ("db", db, t)):      # all of it together: roundings of random sign, and 16 bits of the factors at least
        err, size = float((got.double() - want[name]).norm()), float(want[name].norm())
        assert err <= (8 * (n + max(d_in, d_out)) ** 0.5 * O.U32) * size * 4, name
    # without u, and each gradient by itself
    y2 = m.out(t, d_out, dtype=dt)
    B.adapters_forward(x, y2, a, b, scale, ids=ids, base=base, dropout=drop)
    O.check(y2, want["y"], tol["y"], "y without u")
    again = {"dx": m.out(t, d_in, dtype=dt), "da": m.out(bank, rank, d_in), "db": m.out(bank, d_out, rank)}
    B.adapters_backward(dy, None, None, a, b, scale, ids=ids, dx=again["dx"], dx_base=dx_base, dropout=drop)
    B.adapters_backward(dy, x, None, a, b, scale, ids=ids, dropout=drop, da=again["da"])
    B.adapters_backward(dy, None, u, a, b, scale, ids=ids, dropout=drop, db=again["db"])
    for name, got in again.items():
        O.check(got, want[name], tol[name], name + " alone")
    m.intact()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", [
    # tiles of 32 tokens; banks whose counts leave the ordering two waves and one, and sums a launch of their own
    (8200, 136, 72, 40, 3, "runs", 0.1, True), (8225, 70, 104, 64, 5, "mixed", 0.0, True), (8193, 64, 33, 33, 2, "odd", 0.2, False),
    (600, 16, 24, 2, 3000, "mixed", 0.1, True), (530, 24, 40, 3, 8191, "mixed", 0.0, True),
], ids=lambda c: "-".join(map(str, c)))
def test_adapters_of_large_batches_and_banks(B, dtype, case):
    test_adapters(B, dtype, case)


@pytest.mark.parametrize("t", [3, 200, 900])
def test_adapters_without_ids_and_in_place(B, t):
    m = Arena(t, shift=0)
    case = (t, 264, 136, 8, 1, "one", 0.1, True)
    x, a, b, scale, ids, id_list, base, drop, mk = adapter_inputs(B, m, torch.bfloat16, case)
    y, y2 = m.out(t, 136, dtype=torch.bfloat16), base.clone()
    u = m.out(t, 8)
    B.adapters_forward(x, y, a, b, scale, ids=ids, base=base, dropout=drop, u=u)
    B.adapters_forward(x, y2, a, b, scale, base=y2, dropout=drop)
    assert torch.equal(y, y2)
    dy, dxb = m.normal(t, 136, dtype=torch.bfloat16), m.normal(t, 264, dtype=torch.bfloat16)
    dx, dx2 = m.out(t, 264, dtype=torch.bfloat16), dxb.clone()
    grads = [m.out(1, 8, 264) for _ in range(2)] + [m.out(1, 136, 8) for _ in range(2)]
    B.adapters_backward(dy, x, u, a, b, scale, ids=ids, dx=dx, dx_base=dxb, dropout=drop, da=grads[0], db=grads[2])
    B.adapters_backward(dy, x, u, a, b, scale, dx=dx2, dx_base=dx2, dropout=drop, da=grads[1], db=grads[3])
    assert torch.equal(dx, dx2) and torch.equal(grads[0], grads[1]) and torch.equal(grads[2], grads[3])


@pytest.mark.parametrize("t", [24, 640])
def test_an_adapter_that_has_diverged_stays_with_its_tokens(B, t):
    """Tokens of three adapters in turn, one of which holds NaN and infinities."""
    m = Arena(t)
    x, a, b, scale = m.normal(t, 96), m.normal(3, 8, 96), m.normal(3, 72, 8), m.normal(3)
    a[1, 2, 5], b[1] = float("inf"), float("nan")
    ids = torch.arange(t, dtype=torch.int32, device="cuda") % 3
    base, dy = m.normal(t, 72), m.normal(t, 72)
    y, u, dx, da, db = m.out(t, 72), m.out(t, 8), m.out(t, 96), m.out(3, 8, 96), m.out(3, 72, 8)
    B.adapters_forward(x, y, a, b, scale, ids=ids, base=base, u=u)
    B.adapters_backward(dy, x, u, a, b, scale, ids=ids, dx=dx, da=da, db=db)
    for name, got in (("y", y), ("u", u), ("dx", dx)):
        assert bool(torch.isfinite(got[ids != 1]).all()) and not bool(torch.isfinite(got[ids == 1]).all()), name
    for name, got in (("da", da), ("db", db)):
        assert bool(torch.isfinite(got[[0, 2]]).all()) and not bool(torch.isfinite(got[1]).all()), name


def test_adapters_without_tokens(B):
    z = dict(device="cuda")
    a, b, scale = torch.ones(2, 4, 16, **z), torch.ones(2, 24, 4, **z), torch.ones(2, **z)
    da, db = torch.full_like(a, 3.0), torch.full_like(b, 3.0)
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    B.adapters_forward(torch.empty(0, 16, **z), torch.empty(0, 24, **z), a, b, scale, ids=ids)
    B.adapters_backward(torch.empty(0, 24, **z), torch.empty(0, 16, **z), torch.empty(0, 4, **z), a, b, scale, ids=ids, dx=torch.empty(0, 16, **z), da=da, db=db)
    assert not da.any() and not db.any()


def test_adapter_gradients_are_differences(B):
    """y is linear in x, in a and in b: a whole step along a direction has the gradient's slope but for roundings."""
    m = Arena(12)
    case = (70, 130, 90, 6, 3, "mixed", 0.2, True)
    x, a, b, scale, ids, id_list, base, drop, mk = adapter_inputs(B, m, torch.float32, case)
    x = torch.nan_to_num(x)
    g = m.normal(70, 90)
    y, u = m.out(70, 90), m.out(70, 6)

    def outputs(x, a, b):
        B.adapters_forward(x, y, a, b, scale, ids=ids, base=base, dropout=drop, u=u)
        return y.double().clone()

    y0, u0 = outputs(x, a, b), u.clone()
    dx, da, db = m.out(70, 130), m.out(3, 6, 130), m.out(3, 90, 6)
    B.adapters_backward(g, x, u0, a, b, scale, ids=ids, dx=dx, dropout=drop, da=da, db=db)
    for i, grad in enumerate((dx, da, db)):
        way = m.normal(*grad.shape, std=0.1)
        moved = [x, a, b]
        moved[i] = (moved[i] + way).contiguous()
        y1 = outputs(*moved)
        slope, want = float(((y1 - y0) * g.double()).sum()), float((grad.double() * way.double()).sum())
        size = float(((y1.abs() + y0.abs()) * g.double().abs()).sum()) + float((grad.double() * way.double()).abs().sum())
        assert abs(slope - want) <= 300 * O.U32 * size, (i, slope, want)


# ---- streams and graphs ----------------------------------------------------------------------------------------------

def all_calls(B, m, dt, t):
    """One pass through every operator; returns (run, outputs)."""
    case = (t, 200, 136, 8, 3, "runs", 0.1, True)
    x, a, b, scale, ids, _, base, drop, _ = adapter_inputs(B, m, dt, case)
    x = torch.nan_to_num(x)
    w, bias, res = m.normal(200, dtype=dt), m.normal(200, dtype=dt), m.normal(t, 200, dtype=dt)
    s, h, mean, rstd = m.out(t, 200, dtype=dt), m.out(t, 200, dtype=dt), m.out(t), m.out(t)
    y, u, z = m.out(t, 136, dtype=dt), m.out(t, 8), m.out(t, 136, dtype=dt)
    dy, dh, dx, dres = m.normal(t, 136, dtype=dt), m.out(t, 200, dtype=dt), m.out(t, 200, dtype=dt), m.out(t, 200, dtype=dt)
    da, db, dw, dbias = m.out(3, 8, 200), m.out(3, 136, 8), m.out(200), m.out(200)

    def run():
        B.norm_forward(x, h, w, bias, residual=res, dropout=drop, sum_out=s, mean=mean, rstd=rstd)
        B.adapters_forward(h, y, a, b, scale, ids=ids, base=base, dropout=drop, u=u)
        B.dropout(y, z, drop)
        B.adapters_backward(z, h, u, a, b, scale, ids=ids, dx=dh, dropout=drop, da=da, db=db)
        B.norm_backward(dh, s, dx, mean, rstd, w, dropout=drop, dresidual=dres, dweight=dw, dbias=dbias)

    return run, [s, h, mean, rstd, y, u, z, dh, dx, dres, da, db, dw, dbias], x


@pytest.mark.parametrize("t", [20, 600])
def test_on_another_stream(B, t):
    m = Arena(t)
    run, outs, x = all_calls(B, m, torch.bfloat16, t)
    run()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    for _ in range(3):
        for o in outs:
            o.fill_(float("nan"))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    m.intact()


@pytest.mark.parametrize("dtype,t", [("bf16", 20), ("bf16", 600), ("fp32", 333)])
def test_captured_into_a_graph(B, dtype, t):
    m = Arena(t)
    run, outs, x = all_calls(B, m, TYPES[dtype], t)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        x.copy_(m.normal(*x.shape, dtype=x.dtype))
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for o in outs:
            o.fill_(float("nan"))
        run()                                                # eager work between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(o, g) for o, g in zip(outs, got)), i
    m.intact()
