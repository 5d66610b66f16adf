"""The norm, dropout and adapters in 64 bits, from their definitions, and how far fp32 arithmetic may be off.

A bound counts roundings: half a step of the output's type relative to the value, and 2^-24 per fp32 operation relative to the sum
of the magnitudes that went into it.
"""
import numpy as np
import torch

U32 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def philox(counter, key):
    """Philox-4x32-10 of arrays of four counter words and two key words (numpy uint64 below 2^32)."""
    c, k = [np.asarray(v, dtype=np.uint64) for v in counter], [int(v) for v in key]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def mask(rows, cols, drop, device="cpu"):
    """[rows, cols] in fp64: what each element is multiplied by."""
    if drop is None or drop.p == 0:
        return torch.ones(rows, cols, dtype=torch.float64, device=device)
    limit, per_row = int(np.rint(drop.p * 65536)), -(-cols // 8)
    n = np.arange(rows * per_row, dtype=np.uint64)
    full = np.ones_like(n)
    words = philox([n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), full * np.uint64(drop.offset % 2 ** 32), full * np.uint64(drop.offset >> 32)],
                   [drop.seed % 2 ** 32, drop.seed >> 32])
    bits = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1).astype(np.int64)
    kept = torch.from_numpy(bits.reshape(rows, per_row * 8)[:, :cols] >= limit).to(device)
    return kept.double() * (65536 / (65536 - limit) if limit < 65536 else 0.0)


def dropped(v, m):
    """Dropped elements are 0 whatever they were."""
    return torch.where(m > 0, v.double() * m, torch.zeros((), dtype=torch.float64, device=v.device))


def norm_sum(x, residual, m):
    """(s, bound) with the bound of a sum stored in x's type."""
    s = dropped(x, m)
    size = s.abs()
    if residual is not None:
        s = s + residual.double()
        size = size + residual.double().abs()
    return s, half_step(x.dtype) * s.abs() + 4 * U32 * size


def norm_forward(s, w, bias, form, eps, out_dtype):
    """({name: value}, {name: bound}) from s as stored.  Statistics: chains of at most 100 roundings."""
    s = s.double()
    mean = s.mean(1, keepdim=True) if form == "layer" else torch.zeros_like(s[:, :1])
    d_mean = 100 * U32 * s.abs().mean(1, keepdim=True) if form == "layer" else torch.zeros_like(mean)
    rstd = 1 / torch.sqrt(((s - mean) ** 2).mean(1, keepdim=True) + eps)
    d_h = (d_mean + 2 * U32 * (s.abs() + mean.abs())) * rstd
    # d rstd / rstd = rstd^2 * mean((s - mean) d(s - mean)) + the roundings of the sum and the root
    h = (s - mean) * rstd
    d_rstd = (h.abs() * d_h).mean(1, keepdim=True) + 110 * U32
    d_h = d_h + h.abs() * d_rstd
    scale = torch.ones_like(h[0]) if w is None else w.double()
    y = h * scale
    d_y = d_h * scale.abs() + 4 * U32 * y.abs()
    if bias is not None:
        y = y + bias.double()
        d_y = d_y + 2 * U32 * y.abs()
    return ({"y": y, "mean": mean[:, 0], "rstd": rstd[:, 0]},
            {"y": d_y * 1.01 + half_step(out_dtype) * y.abs(), "mean": d_mean[:, 0] + U32 * mean[:, 0].abs(), "rstd": rstd[:, 0] * d_rstd[:, 0] * 1.01})


def norm_backward(dy, s, mean, rstd, w, form, dsum, m):
    """The statistics are inputs.  Chains: 100 roundings along a row, rows + 100 across rows."""
    dtype = dy.dtype
    dy, s = dy.double(), s.double()
    mean = mean.double()[:, None] if form == "layer" else torch.zeros_like(s[:, :1])
    rstd = rstd.double()[:, None]
    h = (s - mean) * rstd
    size_h = (s.abs() + mean.abs()) * rstd
    g = dy if w is None else dy * w.double()
    mgh, size_mgh = (g * h).mean(1, keepdim=True), (g.abs() * size_h).mean(1, keepdim=True)
    ds = g - h * mgh
    size = g.abs() + size_h * mgh.abs() + h.abs() * size_mgh
    if form == "layer":
        ds = ds - g.mean(1, keepdim=True)
        size = size + g.abs().mean(1, keepdim=True)
    ds, d_ds = ds * rstd, 110 * U32 * size * rstd
    if dsum is not None:
        ds = ds + dsum.double()
        d_ds = d_ds + 2 * U32 * ds.abs()
    n = dy.shape[0] + 100
    return ({"dresidual": ds, "dx": torch.where(m > 0, ds * m, 0.0), "dweight": (dy * h).sum(0), "dbias": dy.sum(0)},
            {"dresidual": d_ds + half_step(dtype) * ds.abs(), "dx": (d_ds + (half_step(dtype) + 2 * U32) * ds.abs()) * m,
             "dweight": n * U32 * (dy.abs() * size_h).sum(0), "dbias": n * U32 * dy.abs().sum(0)})


SPLIT = 2.0 ** -16      # fp32 intermediates go into bf16 products as two terms: 16 of their 24 bits at least


def adapters(x, dy, a, b, scale, ids, base, dx_base, m):
    """Forward and backward: ({name: value}, {name: bound}).  ids: a list; dy None: forward alone."""
    dtype = x.dtype
    t, (n, rank, d_in), d_out = x.shape[0], a.shape, b.shape[1]
    f64 = dict(dtype=torch.float64, device=x.device)
    xm = dropped(x, m)
    want = {"u": torch.zeros(t, rank, **f64), "y": torch.zeros(t, d_out, **f64) if base is None else base.double()}
    tol = {"u": torch.zeros(t, rank, **f64), "y": half_step(dtype) * want["y"].abs()}
    if dy is not None:
        want |= {"dx": torch.zeros(t, d_in, **f64) if dx_base is None else dx_base.double(), "da": torch.zeros(n, rank, d_in, **f64),
                 "db": torch.zeros(n, d_out, rank, **f64)}
        tol |= {"dx": half_step(dtype) * want["dx"].abs(), "da": torch.zeros(n, rank, d_in, **f64), "db": torch.zeros(n, d_out, rank, **f64)}
    split = SPLIT if dtype == torch.bfloat16 else 0.0
    for k in sorted(set(i for i in ids if 0 <= i < n)):
        rows = torch.tensor([i for i, v in enumerate(ids) if v == k], device=x.device)
        ak, bk, sc = a[k].double(), b[k].double(), float(scale[k])
        xk = xm[rows]
        u, size_u = xk @ ak.T, xk.abs() @ ak.abs().T
        d_u = (d_in + 8) * U32 * size_u
        want["u"][rows], tol["u"][rows] = u, d_u
        y = want["y"][rows] + sc * (u @ bk.T)
        d_y = abs(sc) * ((d_u + (split + (rank + 8) * U32) * u.abs()) @ bk.abs().T) + 2 * U32 * y.abs()
        want["y"][rows], tol["y"][rows] = y, d_y + half_step(dtype) * y.abs()
        if dy is None:
            continue
        g = dy[rows].double()
        v, size_v = sc * (g @ bk), abs(sc) * (g.abs() @ bk.abs())
        d_v = (d_out + 8) * U32 * size_v
        mk = m[rows]
        dx = want["dx"][rows] + mk * (v @ ak)
        d_dx = mk * ((d_v + (split + (rank + 8) * U32) * v.abs()) @ ak.abs()) + 2 * U32 * dx.abs()
        want["dx"][rows], tol["dx"][rows] = dx, d_dx + half_step(dtype) * dx.abs()
        want["da"][k], want["db"][k] = v.T @ xk, sc * (g.T @ u)
        many = (len(rows) + 8) * U32
        tol["da"][k] = (d_v + many * v.abs()).T @ xk.abs()
        tol["db"][k] = abs(sc) * (g.abs().T @ (d_u + many * u.abs()))
    return want, tol


def check(got, want, tol, what):
    got = got.double()
    assert got.shape == want.shape, what
    assert bool(torch.isfinite(got).all()), "%s: not finite" % what
    over = (got - want).abs() - tol
    worst = int(over.argmax()) if over.numel() else 0
    assert over.numel() == 0 or float(over.max()) <= 1e-30, "%s: %g instead of %g, off by more than %g, at %d of %s" % (
        what, float(got.flatten()[worst]), float(want.flatten()[worst]), float(tol.flatten()[worst]), worst, tuple(want.shape))
