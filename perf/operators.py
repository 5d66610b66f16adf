"""The operators around the feed-forward layer, as cases a timing program can run.

Three operators, alone and together: the norm (layer norm and its root-mean-square form) with the residual addition and
the dropout in front of it, forward and backward; dropout from a counter-based generator whose mask is never stored; and
low-rank adapters of many requests beside a shared projection, forward and backward.  `run` computes them in their plain
form from elementary torch operations, or, where `own` is true, through the package's entry points on the same tensors.
"""
import math
from functools import reduce

import numpy as np
import torch

own = False  # set by the program that times the cases

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}


def _norm(name, dtype, form, rows, cols, residual=False, p=0.0, bias=False, train=False):
    case = {"op": "norm", "dtype": dtype, "form": form, "rows": rows, "cols": cols, "residual": residual, "p": p, "bias": bias, "train": train}
    return dict(case, name=name) if name else case


def _dropout(name, dtype, rows, cols, p, residual=False):
    case = {"op": "dropout", "dtype": dtype, "rows": rows, "cols": cols, "p": p, "residual": residual}
    return dict(case, name=name) if name else case


def _adapters(name, dtype, tokens, d_in, d_out, rank, bank, requests, p=0.0, train=False):
    """`requests` runs of tokens, each with an adapter of the `bank` or with none; as many requests as tokens: a decode batch."""
    case = {"op": "adapters", "dtype": dtype, "tokens": tokens, "d_in": d_in, "d_out": d_out, "rank": rank, "bank": bank, "requests": requests,
            "p": p, "train": train}
    return dict(case, name=name) if name else case


def listed():
    return [
        # the residual and the norm of one token of one stream being generated: all latency
        _norm("rms-decode-1", "bf16", "rms", 1, 4096, residual=True),
        # a small fp32 study with an odd width, forward only
        _norm("layer-odd-333", "fp32", "layer", 333, 1027, bias=True),
        # several prompts in front of a layer: residual added, normalised
        _norm("rms-prefill-8192", "bf16", "rms", 8192, 4096, residual=True),
        # a training step over the end of a block: dropout, residual, layer norm, and their gradients
        _norm("layer-train-4096", "bf16", "layer", 4096, 4096, residual=True, p=0.1, bias=True, train=True),
        # the same of a small fp32 model with a ragged batch and an odd width
        _norm("layer-train-odd-517", "fp32", "layer", 517, 1001, bias=True, train=True),
        # dropout of a small activation: all latency
        _dropout("dropout-64", "fp32", 64, 256, 0.1),
        # dropout of a large training batch on its way into the residual stream
        _dropout("dropout-add-16384", "bf16", 16384, 4096, 0.1, residual=True),
        # one token with its customer's adapter: the call every decode step makes
        _adapters("adapters-decode-1", "bf16", 1, 4096, 4096, 8, 8, 1),
        # a server's decode batch, each stream with one of many adapters or with none
        _adapters("adapters-decode-64", "bf16", 64, 4096, 11008, 16, 48, 64),
        # prompts of eleven customers in one batch
        _adapters("adapters-prefill-2048", "bf16", 2048, 4096, 4096, 32, 16, 11),
        # fine-tuning of one layer with the study's adapters (rank 8), dropout on their input
        _adapters("adapters-train-4096", "bf16", 4096, 4096, 4096, 8, 1, 1, p=0.05, train=True),
        # several adapters trained in one fp32 batch, nothing a multiple of anything
        _adapters("adapters-train-odd-700", "fp32", 700, 1001, 515, 12, 3, 5, p=0.1, train=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.3 else max(8, w // 64 * 64 if w >= 128 else w // 8 * 8)


LARGEST = 300e6  # bytes of the largest drawn case; the largest listed one has 403 MB


def draw(rng):
    while True:
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        op = rng.choice(["norm", "norm", "dropout", "adapters", "adapters", "adapters"])
        if op == "norm":
            case = _norm("", dtype, rng.choice(["layer", "rms"]), _log_int(rng, 1, 16384), _width(rng, 64, 16384), rng.random() < 0.6,
                         rng.choice([0.0, 0.0, 0.1, 0.3]), rng.random() < 0.5, rng.random() < 0.5)
        elif op == "dropout":
            case = _dropout("", dtype, _log_int(rng, 1, 16384), _width(rng, 64, 16384), round(rng.uniform(0.02, 0.6), 3), rng.random() < 0.5)
        else:
            tokens, train = _log_int(rng, 1, 8192), rng.random() < 0.4
            rank, bank = rng.choice([4, 8, 8, 16, 16, 24, 32, 64, rng.randint(1, 64)]), _log_int(rng, 1, 64)
            requests = tokens if not train and rng.random() < 0.5 and tokens <= 512 else min(tokens, rng.randint(1, 24))
            case = _adapters("", dtype, tokens, _width(rng, 256, 12288), _width(rng, 256, 12288), rank, bank, requests,
                             rng.choice([0.0, 0.1]) if train else 0.0, train)
            if rank * bank > 1024:
                continue
        if work(case)["bytes"] <= LARGEST:
            return case


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "adapters":
        t, i, o, r, n = (case[k] for k in ("tokens", "d_in", "d_out", "rank", "bank"))
        used = n * (1 - (1 - 1 / n) ** (case["requests"] * (1 if case["train"] else 0.9)))  # adapters that a batch can be expected to name
        b = t * (i + 2 * o) * e + used * r * (i + o) * e + 4 * t
        f = 2 * t * r * (i + o)
        if case["train"]:  # forward and backward: dy, dx_base and x again read, dx and the weights' gradients written, u in between
            b += t * (3 * i + o) * e + n * r * (i + o) * 4 + used * r * (i + o) * e + t * r * 4
            f *= 3
        return {"bytes": b, "flops": f}
    n = case["rows"] * case["cols"]
    if case["op"] == "dropout":
        return {"bytes": n * e * (3 if case["residual"] else 2), "flops": 2 * n}
    summed = case["residual"] or case["p"] > 0
    b = n * e * (2 + (1 if case["residual"] else 0) + (1 if summed else 0)) + case["cols"] * e * (2 if case["bias"] else 1)
    f = 8 * n
    if case["train"]:  # dy, the sum and, with a residual stream, its gradient read; one or two gradients written; the weights' gradients
        b += n * e * (3 + (1 if case["residual"] else 0) + (1 if case["residual"] and case["p"] > 0 else 0)) + case["cols"] * 4 * (2 if case["bias"] else 1)
        f += 14 * n
    return {"bytes": b, "flops": f}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dt)

    s = {"case": case, "seed": seed * 2654435761 % (1 << 62), "offset": seed % 1000 + (1 << 33)}
    if case["op"] == "adapters":
        t, i, o, r, n = (case[k] for k in ("tokens", "d_in", "d_out", "rank", "bank"))
        host = np.random.RandomState(seed % (1 << 32))
        # runs of random lengths, one at least each; in a served batch every tenth request has no adapter
        cuts = np.sort(host.choice(t - 1, case["requests"] - 1, replace=False)) + 1 if case["requests"] > 1 else np.zeros(0, dtype=np.int64)
        runs = np.diff(np.concatenate([[0], cuts, [t]]))
        of_run = host.randint(0, n, case["requests"])
        if not case["train"] and case["requests"] > 1:
            of_run = np.where(host.rand(case["requests"]) < 0.1, -1, of_run)
        s["ids"] = torch.from_numpy(np.repeat(of_run, runs).astype(np.int32)).cuda()
        s["x"], s["base"] = normal(t, i), normal(t, o)
        s["a"], s["b"] = normal(n, r, i, std=i ** -0.5), normal(n, o, r, std=0.02)
        s["scale"] = torch.rand(n, generator=g, device="cuda") * 4 + 1  # alpha / rank
        s["y"] = torch.empty(t, o, dtype=dt, device="cuda")
        if case["train"]:
            s["dy"], s["dx_base"], s["dx"] = normal(t, o, std=0.1), normal(t, i, std=0.1), torch.empty(t, i, dtype=dt, device="cuda")
            s["u"] = torch.empty(t, r, device="cuda")
            s["da"], s["db"] = torch.empty(n, r, i, device="cuda"), torch.empty(n, o, r, device="cuda")
        return s
    r, c = case["rows"], case["cols"]
    s["x"], s["y"] = normal(r, c), torch.empty(r, c, dtype=dt, device="cuda")
    s["res"] = normal(r, c, std=2.0, mean=0.5) if case["residual"] else None
    if case["op"] == "norm":
        s["w"] = normal(c, std=0.2, mean=1.0)
        s["bias"] = normal(c, std=0.2) if case["bias"] else None
        s["sum"] = torch.empty(r, c, dtype=dt, device="cuda") if case["residual"] or case["p"] > 0 else None
        if case["train"]:
            s["mean"], s["rstd"] = torch.empty(r, device="cuda"), torch.empty(r, device="cuda")
            s["dy"], s["dx"] = normal(r, c, std=0.1), torch.empty(r, c, dtype=dt, device="cuda")
            s["dsum"] = normal(r, c, std=0.1) if case["residual"] else None  # what reaches the residual stream past the norm
            s["dres"] = torch.empty(r, c, dtype=dt, device="cuda") if case["residual"] and case["p"] > 0 else None
            s["dw"], s["db"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda") if case["bias"] else None
    return s


EPS = 1e-5

# ---- plain form ---------------------------------------------------------------------------------------------------


def _philox_round(state, _):
    """One round of Philox-4x32 (Salmon, Moraes, Dror, Shaw, SC 2011) on four counter words and two key words in int64."""
    c0, c1, c2, c3, k0, k1 = state
    p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # 64-bit products: the sign is cut off with the mask below
    low = 0xFFFFFFFF
    return (p1 >> 32 & low) ^ c1 ^ k0, p1 & low, (p0 >> 32 & low) ^ c3 ^ k1, p0 & low, (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low


def _keep(rows, cols, p, seed, offset):
    """Which elements dropout keeps, and what it multiplies them by: eight elements of a row share one counter."""
    limit = round(p * 65536)
    blocks = -(-cols // 8)
    n = torch.arange(rows * blocks, device="cuda")
    zero = torch.zeros_like(n)
    start = (n & 0xFFFFFFFF, n >> 32, zero + (offset & 0xFFFFFFFF), zero + (offset >> 32), seed & 0xFFFFFFFF, seed >> 32)
    words = torch.stack(reduce(_philox_round, range(10), start)[:4], -1)
    halves = torch.stack([words & 0xFFFF, words >> 16], -1).reshape(rows, blocks * 8)[:, :cols]
    return halves >= limit, 65536 / (65536 - limit)


def _dropped(v, mask):
    if mask is None:
        return v
    keep, scale = mask
    return torch.where(keep, v * scale, 0.0)


def _mask(s, rows, cols):
    return _keep(rows, cols, s["case"]["p"], s["seed"], s["offset"]) if s["case"]["p"] > 0 else None


def _plain_norm(s):
    case = s["case"]
    dt = TYPES[case["dtype"]]
    mask = _mask(s, case["rows"], case["cols"])
    v = _dropped(s["x"].float(), mask)
    if s["res"] is not None:
        v = v + s["res"].float()
    v = v.to(dt)
    out = {"sum": v} if s["sum"] is not None else {}
    v = v.float()
    mean = v.mean(-1, keepdim=True) if case["form"] == "layer" else torch.zeros_like(v[:, :1])
    v = v - mean
    rstd = 1 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    h = v * rstd
    w = s["w"].float()
    out["y"] = (h * w + s["bias"].float() if case["bias"] else h * w).to(dt)
    if not case["train"]:
        return out
    if case["form"] == "layer":
        out["mean"] = mean[:, 0]
    out["rstd"] = rstd[:, 0]
    dy = s["dy"].float()
    gw = dy * w
    ds = gw - h * (gw * h).mean(-1, keepdim=True)
    if case["form"] == "layer":
        ds = ds - gw.mean(-1, keepdim=True)
    ds = ds * rstd
    if s["dsum"] is not None:
        ds = ds + s["dsum"].float()
    if s["dres"] is not None:
        out["dres"] = ds.to(dt)
    out["dx"] = _dropped(ds, mask).to(dt)
    out["dw"] = (dy * h).sum(0)
    if case["bias"]:
        out["db"] = dy.sum(0)
    return out


def _plain_dropout(s):
    case = s["case"]
    v = _dropped(s["x"].float(), _mask(s, case["rows"], case["cols"]))
    return (v + s["res"].float() if s["res"] is not None else v).to(TYPES[case["dtype"]])


def _plain_adapters(s):
    """Every token against every adapter of the bank, all but its own taken out in between."""
    case = s["case"]
    dt, t, r, n = TYPES[case["dtype"]], case["tokens"], case["rank"], case["bank"]
    mask = _mask(s, t, case["d_in"])
    x = _dropped(s["x"].float(), mask)
    a = s["a"].float().reshape(n * r, -1)
    b = s["b"].float().permute(0, 2, 1).reshape(n * r, -1)
    mine = (s["ids"][:, None] == torch.arange(n, device="cuda")).repeat_interleave(r, 1)
    scale = s["scale"].repeat_interleave(r)
    u = torch.where(mine, x @ a.t(), 0.0)
    y = (s["base"].float() + (u * scale) @ b).to(dt)
    if not case["train"]:
        return {"y": y}
    dy = s["dy"].float()
    v = torch.where(mine, dy @ b.t(), 0.0) * scale
    dx = (s["dx_base"].float() + _dropped(v @ a, mask)).to(dt)
    return {"y": y, "dx": dx, "da": (v.t() @ x).reshape(n, r, -1), "db": ((u * scale).t() @ dy).reshape(n, r, -1).permute(0, 2, 1).contiguous()}


# ---- the package's entry points -----------------------------------------------------------------------------------

_lib = []


def _binding():
    if not _lib:
        from paper_2502_04416_amd import binding
        _lib.append(binding)
    return _lib[0]


def _own_norm(s):
    case, lib = s["case"], _binding()
    drop = lib.Dropout(case["p"], s["seed"], s["offset"]) if case["p"] > 0 else None
    mean, rstd = s.get("mean"), s.get("rstd")
    lib.norm_forward(s["x"], s["y"], s["w"], s["bias"], form=case["form"], eps=EPS, residual=s["res"], dropout=drop, sum_out=s["sum"], mean=mean, rstd=rstd)
    out = {"y": s["y"]}
    if s["sum"] is not None:
        out["sum"] = s["sum"]
    if not case["train"]:
        return out
    lib.norm_backward(s["dy"], s["x"] if s["sum"] is None else s["sum"], s["dx"], mean, rstd, s["w"], form=case["form"], dsum=s["dsum"], dropout=drop,
                      dresidual=s["dres"], dweight=s["dw"], dbias=s["db"])
    out |= {"rstd": rstd, "dx": s["dx"], "dw": s["dw"]}
    if case["form"] == "layer":
        out["mean"] = mean
    if s["dres"] is not None:
        out["dres"] = s["dres"]
    if s["db"] is not None:
        out["db"] = s["db"]
    return out


def _own_dropout(s):
    lib = _binding()
    lib.dropout(s["x"], s["y"], lib.Dropout(s["case"]["p"], s["seed"], s["offset"]), residual=s["res"])
    return s["y"]


def _own_adapters(s):
    case, lib = s["case"], _binding()
    drop = lib.Dropout(case["p"], s["seed"], s["offset"]) if case["p"] > 0 else None
    lib.adapters_forward(s["x"], s["y"], s["a"], s["b"], s["scale"], ids=s["ids"], base=s["base"], dropout=drop, u=s.get("u"))
    if not case["train"]:
        return {"y": s["y"]}
    lib.adapters_backward(s["dy"], s["x"], s["u"], s["a"], s["b"], s["scale"], ids=s["ids"], dx=s["dx"], dx_base=s["dx_base"], dropout=drop, da=s["da"], db=s["db"])
    return {"y": s["y"], "dx": s["dx"], "da": s["da"], "db": s["db"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return (_own_norm if op == "norm" else _own_dropout if op == "dropout" else _own_adapters)(state)
    return (_plain_norm if op == "norm" else _plain_dropout if op == "dropout" else _plain_adapters)(state)


# ---- 64 bits ------------------------------------------------------------------------------------------------------


def _exact_mask(rows, cols, p, seed, offset):
    """[rows, cols] in fp64: 0 where dropped, 65536 / (65536 - limit) where kept."""
    if p == 0:
        return torch.ones(rows, cols, dtype=torch.float64, device="cuda")
    mask32, limit, per_row = np.uint64(0xFFFFFFFF), int(np.rint(p * 65536)), (cols + 7) // 8
    block = np.arange(rows * per_row, dtype=np.uint64)
    half = np.uint64(32)
    ctr = [block & mask32, block >> half, np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, offset >> 32)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for k in range(10):
        a, b = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ctr = [(b >> half) ^ ctr[1] ^ np.uint64((key[0] + k * 0x9E3779B9) % (1 << 32)), b & mask32,
               (a >> half) ^ ctr[3] ^ np.uint64((key[1] + k * 0xBB67AE85) % (1 << 32)), a & mask32]
    bits = np.empty((rows * per_row, 8), dtype=np.int32)
    for w in range(4):
        bits[:, 2 * w], bits[:, 2 * w + 1] = ctr[w] & np.uint64(0xFFFF), ctr[w] >> np.uint64(16)
    kept = torch.from_numpy(bits.reshape(rows, per_row * 8)[:, :cols] >= limit).cuda()
    return kept.double() * (65536.0 / (65536 - limit))


def _exact_norm(s):
    case = s["case"]
    m = _exact_mask(case["rows"], case["cols"], case["p"], s["seed"], s["offset"])
    total = s["x"].double() * m
    if s["res"] is not None:
        total += s["res"].double()
    out = {}
    if s["sum"] is not None:
        out["sum"] = total
        total = total.to(TYPES[case["dtype"]]).double()  # the norm is that of the sum as it is stored
    width = case["cols"]
    mu = total.sum(1) / width if case["form"] == "layer" else torch.zeros(case["rows"], dtype=torch.float64, device="cuda")
    centred = total - mu[:, None]
    r = ((centred ** 2).sum(1) / width + EPS) ** -0.5
    unit = centred * r[:, None]
    w = s["w"].double()
    out["y"] = unit * w
    if case["bias"]:
        out["y"] = out["y"] + s["bias"].double()
    if not case["train"]:
        return out
    if case["form"] == "layer":
        out["mean"] = mu
    out["rstd"] = r
    dy = s["dy"].double()
    # d y_j / d s_i = w_j r (delta_ij - [layer] 1 / C - unit_i unit_j / C)
    back = dy * w
    ds = r[:, None] * (back - unit * ((back * unit).sum(1) / width)[:, None])
    if case["form"] == "layer":
        ds -= r[:, None] * (back.sum(1) / width)[:, None]
    if s["dsum"] is not None:
        ds += s["dsum"].double()
    if s["dres"] is not None:
        out["dres"] = ds
    out["dx"] = ds * m
    out["dw"] = torch.einsum("rc,rc->c", dy, unit)
    if case["bias"]:
        out["db"] = dy.sum(0)
    return out


def _exact_adapters(s):
    case = s["case"]
    m = _exact_mask(case["tokens"], case["d_in"], case["p"], s["seed"], s["offset"])
    x = s["x"].double() * m
    y = s["base"].double()
    train = case["train"]
    if train:
        dx, da, db = s["dx_base"].double(), torch.zeros(s["a"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["b"].shape, dtype=torch.float64, device="cuda")
    for k in sorted(set(s["ids"].tolist()) - {-1}):
        rows = (s["ids"] == k).nonzero()[:, 0]
        a, b, sc = s["a"][k].double(), s["b"][k].double(), float(s["scale"][k])
        u = x[rows] @ a.T
        y[rows] += sc * (u @ b.T)
        if train:
            g = s["dy"][rows].double()
            v = sc * (g @ b)
            dx[rows] += m[rows] * (v @ a)
            da[k], db[k] = v.T @ x[rows], sc * (g.T @ u)
    return {"y": y, "dx": dx, "da": da, "db": db} if train else {"y": y}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    if case["op"] == "adapters":
        return _exact_adapters(s)
    y = s["x"].double() * _exact_mask(case["rows"], case["cols"], case["p"], s["seed"], s["offset"])
    return y + s["res"].double() if s["res"] is not None else y
