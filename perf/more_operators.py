"""What training a feed-forward block towards a language model's loss takes, as cases a timing program can run.

Three operators, alone: the gated feed-forward block on weights that are trained (plain matrices, nothing packed), forward and
backward; the softmax cross entropy of a head over a vocabulary whose logits are never kept, with its gradients; and the norm of
all gradients of a step with the clipping by it.  `run` computes them in their plain form from elementary torch operations, or, where
`own` is true, through the package's entry points on the same tensors.
"""
import math

import torch

own = False  # set by the program that times the cases

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}


def _ffn(name, dtype, tokens, d, d_ff, train=False):
    case = {"op": "ffn", "dtype": dtype, "tokens": tokens, "d": d, "d_ff": d_ff, "train": train}
    return dict(case, name=name) if name else case


def _head(name, dtype, tokens, d, vocab, ignored=0.0, weighted=False, train=False):
    """`ignored`: the share of tokens without a target, `weighted`: tokens count differently, as answers and prompts do."""
    case = {"op": "head", "dtype": dtype, "tokens": tokens, "d": d, "vocab": vocab, "ignored": ignored, "weighted": weighted, "train": train}
    return dict(case, name=name) if name else case


def _clip(name, dtype, kind, layers, d, width, std=1e-2):
    """Gradients of `layers` blocks: "adapters" (pairs of rank `width` and the norm's weight) or "dense" (the three matrices of a gated
    block of that width and the norm's weight, which stays in fp32)."""
    case = {"op": "clip", "dtype": dtype, "kind": kind, "layers": layers, "d": d, "width": width, "std": std}
    return dict(case, name=name) if name else case


def listed():
    return [
        # one token of one stream through a block that is still being trained: its weights once
        _ffn("ffn-decode-1", "bf16", 1, 4096, 11008),
        # a small batch of streams sampled from the model in training
        _ffn("ffn-decode-24", "bf16", 24, 4096, 11008),
        # a training step of a block, its batch of ordinary length
        _ffn("ffn-train-2048", "bf16", 2048, 4096, 11008, train=True),
        # the same with a wider block and a longer batch: the most work
        _ffn("ffn-train-4096", "bf16", 4096, 4096, 14336, train=True),
        # a small fp32 study, nothing a multiple of anything
        _ffn("ffn-train-odd-517", "fp32", 517, 515, 1379, train=True),
        # the log-probability of one token of a sequence being scored
        _head("head-score-1", "bf16", 1, 4096, 32768),
        # a training step's loss: prompts without a target, both gradients
        _head("head-train-2048", "bf16", 2048, 4096, 32768, ignored=0.25, train=True),
        # a long batch over a large vocabulary, whose logits would take 2 GB
        _head("head-train-8192", "bf16", 8192, 4096, 131072, ignored=0.1, train=True),
        # a small fp32 study with an odd vocabulary, tokens weighted
        _head("head-train-odd-301", "fp32", 301, 515, 10007, ignored=0.2, weighted=True, train=True),
        # the trained tensors of one recovery block: all latency
        _clip("clip-adapters-1", "fp32", "adapters", 1, 4096, 8),
        # adapters of a whole model, odd sizes, each tensor wherever the one before it ends
        _clip("clip-adapters-odd-40", "bf16", "adapters", 40, 1027, 12, std=1e-4),
        # eight dense blocks
        _clip("clip-dense-8", "bf16", "dense", 8, 4096, 11008),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.3 else max(8, w // 64 * 64 if w >= 128 else w // 8 * 8)


# of the largest drawn cases; the listed ones have 26 TFLOP and 4.3 GB
FLOPS = {"bf16": 3e12, "fp32": 3e11}
BYTES = 2e9


def draw(rng):
    while True:
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        op = rng.choice(["ffn", "ffn", "head", "head", "clip"])
        if op == "ffn":
            case = _ffn("", dtype, _log_int(rng, 1, 8192), _width(rng, 128, 8192), _width(rng, 256, 16384), rng.random() < 0.7)
        elif op == "head":
            case = _head("", dtype, _log_int(rng, 1, 8192), _width(rng, 128, 8192), _log_int(rng, 500, 160000), rng.choice([0.0, 0.1, 0.5, 0.9]),
                         rng.random() < 0.3, rng.random() < 0.7)
        else:
            kind = rng.choice(["adapters", "dense"])
            case = _clip("", dtype, kind, _log_int(rng, 1, 64), _width(rng, 64, 8192), rng.choice([4, 8, 16, 31, 64]) if kind == "adapters" else _width(rng, 128, 16384),
                         rng.choice([1e-2, 1e-4, 1e-7]))
        w = work(case)
        if w["flops"] <= FLOPS[dtype] and w["bytes"] <= BYTES:
            return case


def _shapes(case):
    """The shapes of the case's gradients of its type, and of those in fp32."""
    n, d, w = case["layers"], case["d"], case["width"]
    if case["kind"] == "adapters":
        return [(w, d), (d, w)] * n, [(d,)] * n
    return [(d, w), (d, w), (w, d)] * n, [(d,)] * n


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "clip":
        main, rest = (sum(math.prod(s) for s in group) for group in _shapes(case))
        return {"bytes": 2 * (main * e + rest * 4) + 4, "flops": 3 * (main + rest)}
    t, d = case["tokens"], case["d"]
    if case["op"] == "ffn":
        f = case["d_ff"]
        b, flops = (2 * t * d + t * f + 3 * d * f) * e, 6 * t * d * f
        if case["train"]:  # gate and up written; then dy, x, gate, up, hidden and the weights read, dgate, dup, dx and the weights' gradients written
            b += (2 * t * f + 3 * t * d + 5 * t * f + 6 * d * f) * e
            flops *= 3
        return {"bytes": b, "flops": flops}
    v = case["vocab"]
    b, flops = (t * d + v * d) * e + 12 * t, 2 * t * d * v
    if case["train"]:
        b += (2 * t * d + 2 * v * d) * e + 8 * t
        flops *= 3
    return {"bytes": b, "flops": flops}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).to(dtype)

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    s = {"case": case}
    if case["op"] == "clip":
        s["max_norm"], s["norm"] = 1.0, empty(1, dtype=torch.float32)
        s["grads"], s["out"], s["flat"] = [], [], {}
        for key, kind, shapes in zip(("main", "rest"), (dt, torch.float32), _shapes(case)):  # a bucket of each: what a reducer of gradients keeps
            sizes = [math.prod(x) for x in shapes]
            bucket = normal(sum(sizes), std=case["std"], dtype=kind)
            s["flat"][key] = torch.empty_like(bucket)
            s["grads"] += [p.view(x) for p, x in zip(bucket.split(sizes), shapes)]
            s["out"] += [p.view(x) for p, x in zip(s["flat"][key].split(sizes), shapes)]
        return s
    t, d = case["tokens"], case["d"]
    if case["op"] == "ffn":
        f = case["d_ff"]
        s["x"], s["y"] = normal(t, d), empty(t, d)
        s["wg"], s["wu"], s["wd"] = normal(d, f, std=d ** -0.5), normal(d, f, std=d ** -0.5), normal(f, d, std=f ** -0.5)
        s["hidden"] = empty(t, f)
        if case["train"]:
            s["gate"], s["up"], s["dgate"], s["dup"] = (empty(t, f) for _ in range(4))
            s["dy"], s["dx"] = normal(t, d, std=0.1), empty(t, d)
            s["dwg"], s["dwu"], s["dwd"] = empty(d, f), empty(d, f), empty(f, d)
        return s
    v = case["vocab"]
    s["w"] = normal(v, d, std=0.02)
    ids = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    # a normalised stream that leans towards the target's row by what a model has learnt: nothing here, nearly all there
    lean = torch.rand(t, 1, generator=g, device="cuda") * (16 / (0.02 * d ** 0.5) / (0.02 * d ** 0.5))
    s["x"] = (torch.randn(t, d, generator=g, device="cuda") + lean * s["w"][ids.long()].float()).to(dt)
    s["ids"] = torch.where(torch.rand(t, generator=g, device="cuda") < case["ignored"], -100, ids).to(torch.int32)
    s["loss"], s["lse"] = empty(t, dtype=torch.float32), empty(t, dtype=torch.float32)
    if case["train"]:
        s["dloss"] = torch.rand(t, generator=g, device="cuda") * 1.5 + 0.5 if case["weighted"] else None
        s["scale"] = 1.0 / max(1, int((s["ids"] >= 0).sum()))
        s["dx"], s["dw"] = empty(t, d), empty(v, d)
    return s


EPS = 1e-6

# ---- plain form ---------------------------------------------------------------------------------------------------


def _plain_ffn(s):
    dt = s["x"].dtype
    x, wg, wu, wd = (s[k].float() for k in ("x", "wg", "wu", "wd"))
    gate, up = x @ wg, x @ wu
    hidden = (gate / (1 + torch.exp(-gate)) * up).to(dt)
    out = {"y": (hidden.float() @ wd).to(dt), "hidden": hidden}
    if not s["case"]["train"]:
        return out
    out["gate"], out["up"] = gate.to(dt), up.to(dt)  # what a backward pass finds is what was stored
    gate, up, dy = out["gate"].float(), out["up"].float(), s["dy"].float()
    share = 1 / (1 + torch.exp(-gate))
    dh = dy @ wd.t()
    out["dgate"] = (dh * up * share * (1 + gate * (1 - share))).to(dt)
    out["dup"] = (dh * gate * share).to(dt)
    dgate, dup = out["dgate"].float(), out["dup"].float()
    out["dx"] = (dgate @ wg.t() + dup @ wu.t()).to(dt)
    out["dwg"], out["dwu"] = (x.t() @ dgate).to(dt), (x.t() @ dup).to(dt)
    out["dwd"] = (hidden.float().t() @ dy).to(dt)
    return out


def _plain_head(s):
    x, w, ids = s["x"].float(), s["w"].float(), s["ids"].long()
    logits = x @ w.t()
    has = (ids >= 0) & (ids < w.shape[0])
    at = torch.where(has, ids, 0)[:, None]
    top = logits.amax(1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(logits - top).sum(1))
    out = {"loss": torch.where(has, lse - logits.gather(1, at)[:, 0], 0.0), "lse": lse}
    if not s["case"]["train"]:
        return out
    share = has * s["scale"] if s["dloss"] is None else has * s["scale"] * s["dloss"]
    g = torch.exp(logits - lse[:, None])
    del logits
    g.scatter_add_(1, at, torch.full_like(g[:, :1], -1.0))
    g *= share[:, None]
    out["dx"], out["dw"] = (g @ w).to(s["x"].dtype), (g.t() @ x).to(s["x"].dtype)
    return out


def _plain_clip(s):
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    c = torch.clamp(s["max_norm"] / (norm + EPS), max=1.0)
    [out.copy_(g.double() * c) for out, g in zip(s["out"], s["grads"])]
    return {"norm": norm.float().reshape(1), **s["flat"]}


# ---- the package's entry points -----------------------------------------------------------------------------------

_lib = []


def _binding():
    if not _lib:
        from paper_2502_04416_amd import binding
        _lib.append(binding)
    return _lib[0]


def _own_ffn(s):
    lib = _binding()
    lib.ffn_forward(s["x"], s["y"], s["wg"], s["wu"], s["wd"], s["hidden"], gate=s.get("gate"), up=s.get("up"))
    if not s["case"]["train"]:
        return {"y": s["y"], "hidden": s["hidden"]}
    lib.ffn_backward(s["dy"], s["x"], s["gate"], s["up"], s["hidden"], s["wg"], s["wu"], s["wd"], s["dgate"], s["dup"], dx=s["dx"],
                     dw_gate=s["dwg"], dw_up=s["dwu"], dw_down=s["dwd"])
    return {k: s[k] for k in ("y", "hidden", "gate", "up", "dgate", "dup", "dx", "dwg", "dwu", "dwd")}


def _own_head(s):
    lib = _binding()
    lib.head_loss_forward(s["x"], s["w"], s["ids"], s["loss"], s["lse"])
    if not s["case"]["train"]:
        return {"loss": s["loss"], "lse": s["lse"]}
    lib.head_loss_backward(s["x"], s["w"], s["ids"], s["lse"], dx=s["dx"], dweight=s["dw"], dloss=s["dloss"], scale=s["scale"])
    return {"loss": s["loss"], "lse": s["lse"], "dx": s["dx"], "dw": s["dw"]}


def _own_clip(s):
    _binding().clip_gradients(s["grads"], s["norm"], s["max_norm"], out=s["out"], eps=EPS)
    return {"norm": s["norm"], **s["flat"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return (_own_ffn if op == "ffn" else _own_head if op == "head" else _own_clip)(state)
    return (_plain_ffn if op == "ffn" else _plain_head if op == "head" else _plain_clip)(state)


# ---- 64 bits ------------------------------------------------------------------------------------------------------


def _exact_ffn(s):
    dt, train = s["x"].dtype, s["case"]["train"]
    x, wg, wu, wd = (s[k].double() for k in ("x", "wg", "wu", "wd"))
    a, b = torch.mm(x, wg), torch.mm(x, wu)
    hidden = a * b * torch.sigmoid(a)
    kept = hidden.to(dt).double()  # the product behind it is that of the hidden state as it is stored
    out = {"hidden": hidden, "y": torch.mm(kept, wd)}
    if not train:
        return out
    out["gate"], out["up"] = a, b
    a, b = a.to(dt).double(), b.to(dt).double()
    # d/da [a b / (1 + e^-a)] = b (1 + e^-a + a e^-a) / (1 + e^-a)^2
    e = torch.exp(-a.abs())
    slope = torch.where(a >= 0, (1 + e + a * e) / (1 + e) ** 2, (e * e + e + a * e) / (1 + e) ** 2)
    dy = s["dy"].double()
    dh = torch.mm(dy, wd.T.contiguous())
    out["dgate"], out["dup"] = dh * b * slope, dh * (a * torch.sigmoid(a))
    da, db = (out[k].to(dt).double() for k in ("dgate", "dup"))
    xt = x.T.contiguous()
    out["dwg"], out["dwu"], out["dwd"] = torch.mm(xt, da), torch.mm(xt, db), torch.mm(kept.T.contiguous(), dy)
    out["dx"] = torch.mm(da, wg.T.contiguous()).add_(torch.mm(db, wu.T.contiguous()))
    return out


def _exact_head(s):
    """In blocks of tokens: the logits of all of them would be large in 64 bits."""
    t, v = s["x"].shape[0], s["w"].shape[0]
    w, train = s["w"].double(), s["case"]["train"]
    wt = w.T.contiguous()
    loss, lse = (torch.zeros(t, dtype=torch.float64, device="cuda") for _ in range(2))
    if train:
        dx, dw = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda"), torch.zeros_like(w)
        each = torch.full((t,), float(s["scale"]), dtype=torch.float64, device="cuda")
        if s["dloss"] is not None:
            each = each * s["dloss"].double()
    step = max(1, (1 << 28) // v)
    for i in range(0, t, step):
        x, ids = s["x"][i:i + step].double(), s["ids"][i:i + step].long()
        z = torch.mm(x, wt)
        lse[i:i + step] = torch.logsumexp(z, 1)
        rows = ((ids >= 0) & (ids < v)).nonzero()[:, 0]
        loss[i + rows] = lse[i + rows] - z[rows, ids[rows]]
        if train:
            z = torch.softmax(z, 1)
            z[rows, ids[rows]] -= 1
            keep = torch.zeros(len(ids), dtype=torch.float64, device="cuda")
            keep[rows] = each[i + rows]
            z *= keep[:, None]
            dx[i:i + step] = torch.mm(z, w)
            dw += torch.mm(z.T.contiguous(), x)
    return {"loss": loss, "lse": lse, "dx": dx, "dw": dw} if train else {"loss": loss, "lse": lse}


def _exact_clip(s):
    squares = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in s["grads"]:
        squares += torch.linalg.vector_norm(g.double()) ** 2
    norm = float(squares) ** 0.5
    c = min(1.0, s["max_norm"] / (norm + EPS))
    case_rest, out = s["case"]["layers"], {}
    for group, key in zip((s["grads"][:-case_rest], s["grads"][-case_rest:]), ("main", "rest")):
        out[key] = torch.cat([g.reshape(-1).double() for g in group]) * c
    return {"norm": torch.tensor([norm], dtype=torch.float64, device="cuda"), **out}


def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_ffn if case["op"] == "ffn" else _exact_head if case["op"] == "head" else _exact_clip)(s)
