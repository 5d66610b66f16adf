"""A dense block trained on tokens before it is restructured, and its recovery on the same tokens after.

    out = norm(residual + ffn(x)) * weight,    loss = softmax cross entropy of head(out) against the next token

`Dense.step` trains the three matrices, the norm's weight and the head by the package's own operators: the gated block's forward and
backward pass, the head's loss without its logits, all gradients clipped together.  `Dense.restructured` hands the matrices to
cmoe_build; recovery.Block then trains adapters beside the restructured layer on the same loss.

    python -m paper_2502_04416_amd.finetune        # on an MI355X: a small block, its loss trained, restructured and recovered
"""
from __future__ import annotations

from . import binding, recovery, synth


def _trained(v):
    """A copy of a tensor or array, in fp32 on the device: what is trained is not the caller's."""
    import torch
    return torch.as_tensor(v).detach().to(device="cuda", dtype=torch.float32, copy=True, memory_format=torch.contiguous_format)


class Head:
    """Rows of a vocabulary, [vocab, d] in fp32 as trained, a copy of those given; the operators read them in `dtype`."""

    def __init__(self, weight, dtype):
        self.params, self.dtype = {"head": _trained(weight)}, dtype
        self.cast()

    def cast(self):
        self.weight = self.params["head"].to(self.dtype)

    def loss(self, out, targets, train: bool = True):
        """(mean loss of the targets in the vocabulary, gradient of out, gradient of the rows or None)."""
        import torch
        loss, lse = (torch.empty(len(out), dtype=torch.float32, device="cuda") for _ in range(2))
        dout = torch.empty_like(out)
        dweight = torch.empty_like(self.weight) if train else None
        binding.head_loss_forward(out, self.weight, targets, loss, lse)
        # the mean's factor, on the device and in fp32: the gradients' sums are scaled by it before they are rounded
        each = ((targets >= 0) & (targets < len(self.weight))).sum().clamp(min=1).float().reciprocal()
        binding.head_loss_backward(out, self.weight, targets, lse, dx=dout, dweight=dweight, scale=each)
        return loss.sum() * each, dout, dweight


class Dense:
    """The trained dense block.  Matrices in the paper's orientation: w_gate, w_up [d, d_ff], w_down [d_ff, d]; copies of them are trained."""

    def __init__(self, w_gate, w_up, w_down, head: Head, form: str = "rms", eps: float = 1e-5):
        import torch
        self.head, self.form, self.eps, self.steps = head, form, eps, 0
        self.params = {k: _trained(v) for k, v in (("gate", w_gate), ("up", w_up), ("down", w_down))}
        self.params["weight"] = torch.ones(self.params["gate"].shape[0], dtype=torch.float32, device="cuda")
        self.params.update(head.params)
        self.moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in self.params.items()}
        self._cast()

    def _cast(self):
        self.gate, self.up, self.down, self.weight = (self.params[k].to(self.head.dtype) for k in ("gate", "up", "down", "weight"))
        self.head.cast()

    def forward(self, x, residual, train: bool = False):
        """(out, what the backward pass needs): [tokens, d] of the head's type."""
        import torch
        f32 = dict(dtype=torch.float32, device="cuda")
        s, out = torch.empty_like(x), torch.empty_like(x)
        hidden, gate, up = (torch.empty(len(x), self.gate.shape[1], dtype=x.dtype, device="cuda") if i == 0 or train else None for i in range(3))
        mean, rstd = torch.empty(len(x), **f32), torch.empty(len(x), **f32)
        binding.ffn_forward(x, s, self.gate, self.up, self.down, hidden, gate=gate, up=up, base=residual)
        binding.norm_forward(s, out, self.weight, form=self.form, eps=self.eps, mean=mean, rstd=rstd)
        return out, (s, hidden, gate, up, mean, rstd)

    def gradients(self, x, residual, targets, dx=None):
        """(mean loss, {name: gradient}); dx receives the gradient of x, and with it that of the residual where x is the residual itself."""
        import torch
        out, (s, hidden, gate, up, mean, rstd) = self.forward(x, residual, train=True)
        loss, dout, dhead = self.head.loss(out, targets)
        grads = {"gate": torch.empty_like(self.gate), "up": torch.empty_like(self.up), "down": torch.empty_like(self.down),
                 "weight": torch.empty_like(self.params["weight"]), "head": dhead}
        ds = torch.empty_like(x)
        binding.norm_backward(dout, s, ds, mean, rstd, self.weight, form=self.form, dweight=grads["weight"])
        binding.ffn_backward(ds, x, gate, up, hidden, self.gate, self.up, self.down, gate, up, dx=dx, dx_base=ds if dx is not None and x is residual else None,
                             dw_gate=grads["gate"], dw_up=grads["up"], dw_down=grads["down"])
        return loss, grads

    def step(self, x, residual, targets, lr: float = 1e-3, betas=(0.9, 0.95), max_norm: float = 1.0):
        """One step of Adam on gradients clipped together; (loss, their norm) before it, on the device."""
        import torch
        loss, grads = self.gradients(x, residual, targets)
        norm = torch.empty(1, dtype=torch.float32, device="cuda")
        binding.clip_gradients(list(grads.values()), norm, max_norm)
        self.steps += 1
        for k, g in grads.items():
            g = g.float()
            m, v = self.moments[k]
            m.lerp_(g, 1 - betas[0])
            v.lerp_(g * g, 1 - betas[1])
            self.params[k] -= lr * (m / (1 - betas[0] ** self.steps)) / ((v / (1 - betas[1] ** self.steps)).sqrt() + 1e-12)
        self._cast()
        return loss, norm

    def restructured(self, cfg, calibration) -> binding.Layer:
        """The block's matrices as shared and routed experts (cmoe_build), uploaded."""
        return binding.Layer.build(cfg, *(self.params[k].cpu().numpy() for k in ("gate", "up", "down")), calibration)


def main(steps: int = 200, tokens: int = 1024, vocab: int = 4000):
    import torch
    cfg = synth.scaled(synth.CONFIGS[1], d_model=512, d_ff=2752, n_centres=16)
    source = synth.make_token_source(cfg)
    rng = torch.Generator().manual_seed(5)
    dtype = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
    head = Head(torch.randn(vocab, cfg.d_model, generator=rng) * 0.05, dtype)
    dense = Dense(*synth.make_weights(cfg), head)
    says = torch.randn(cfg.d_model, vocab, generator=rng).cuda()            # the token that follows is a function of x

    def batch(i):
        x = torch.from_numpy(source.eval_batch(i, n=tokens)).to("cuda", dtype)
        return x, torch.zeros_like(x), (x.float() @ says).argmax(1).to(torch.int32)

    def loss_of(out, targets):
        loss = torch.empty(len(out), dtype=torch.float32, device="cuda")
        binding.head_loss_forward(out, head.weight, targets, loss)
        return float(loss.mean())

    x, residual, targets = batch(10 ** 6)
    losses = [loss_of(dense.forward(x, residual)[0], targets)]
    for i in range(steps):
        dense.step(*batch(i))
    losses.append(loss_of(dense.forward(x, residual)[0], targets))
    block = recovery.Block(dense.restructured(cfg, source.calibration()), p=0.0, form=dense.form, eps=dense.eps, seed=0)
    block.params["weight"].copy_(dense.params["weight"])
    block._cast()
    losses.append(loss_of(block.serve(x, residual)[0], targets))
    for i in range(steps):
        block.step_tokens(*batch(i), head)
    losses.append(loss_of(block.serve(x, residual)[0], targets))
    print("loss per token on tokens of their own: %.3f; dense block trained %.3f; restructured %.3f; recovered %.3f" % tuple(losses))
    return losses


if __name__ == "__main__":
    main()
