"""What restructuring loses, recovered with low-rank adapters beside the restructured layer (paper Sec. 5.1: rank 8, alpha 32).

A block is what a transformer has there:

    out = norm(residual + drop(ffn(x) + adapters(drop(x)))) * weight

`Block.step` trains the adapters and the norm's weight towards given outputs, by the package's own forward and backward operators; the
feed-forward layer is frozen.  `Block.serve` runs the block for a batch of requests, each token with an adapter of the bank or none.

    python -m paper_2502_04416_amd.recovery        # on an MI355X: a small layer, the distance to its dense form before and after
"""
from __future__ import annotations

import itertools
from typing import Optional

from . import binding, synth

_blocks = itertools.count()


class Block:
    """A restructured layer (binding.Layer, uploaded), a bank of adapters beside it and the norm that follows.

    seed: of the adapters' first values and of the dropout masks, another for every block of a model, or two of them drop the same
    elements in the same step.  None: the number of blocks made without one before this, which a program that makes its blocks in the same
    order finds again."""

    def __init__(self, layer: binding.Layer, n_adapters: int = 1, rank: int = 8, alpha: float = 32.0, p: float = 0.05, form: str = "rms",
                 eps: float = 1e-5, seed: Optional[int] = None):
        import torch
        if seed is None:
            seed = next(_blocks)
        self.layer, self.form, self.eps, self.p, self.seed, self.steps = layer, form, eps, p, seed, 0
        d = layer.cfg.d_model
        self.dtype = torch.bfloat16 if layer.bf16 else torch.float32
        rng = torch.Generator().manual_seed(seed)
        # trained in fp32; the operators read them in the layer's type
        self.params = {"a": (torch.randn(n_adapters, rank, d, generator=rng) * d ** -0.5).cuda(), "b": torch.zeros(n_adapters, d, rank, device="cuda"),
                       "weight": torch.ones(d, device="cuda")}
        self.scale = torch.full((n_adapters,), alpha / rank, device="cuda")
        self.moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in self.params.items()}
        self._cast()

    def _cast(self):
        self.a, self.b, self.weight = (self.params[k].to(self.dtype) for k in ("a", "b", "weight"))

    def serve(self, x, residual, ids=None):
        """(out, stream): [tokens, d] of the layer's type; ids: [tokens] int32 (no adapter where it is not in the bank), None: adapter 0."""
        import torch
        z, out = torch.empty_like(x), torch.empty_like(x)
        self.layer.forward_device(x, z)
        binding.adapters_forward(x, z, self.a, self.b, self.scale, ids=ids, base=z)
        binding.norm_forward(z, out, self.weight, form=self.form, eps=self.eps, residual=residual, sum_out=z)
        return out, z

    def gradients(self, x, residual, target, ids=None):
        """(mean squared distance of the block's outputs to the target, gradients of a, b and weight)."""
        import torch
        t, d = x.shape
        f32 = dict(dtype=torch.float32, device="cuda")
        before, after = (binding.Dropout(self.p, self.seed, 2 * self.steps + i) for i in (0, 1))
        z, s, out, dz = (torch.empty_like(x) for _ in range(4))
        u, mean, rstd = torch.empty(t, self.a.shape[1], **f32), torch.empty(t, **f32), torch.empty(t, **f32)
        self.layer.forward_device(x, z)
        binding.adapters_forward(x, z, self.a, self.b, self.scale, ids=ids, base=z, dropout=before, u=u)
        binding.norm_forward(z, out, self.weight, form=self.form, eps=self.eps, residual=residual, dropout=after, sum_out=s, mean=mean, rstd=rstd)
        off = out.float() - target.float()
        dy = (off * (2.0 / off.numel())).to(self.dtype)
        grads = {k: torch.empty_like(v) for k, v in self.params.items()}
        binding.norm_backward(dy, s, dz, mean, rstd, self.weight, form=self.form, dropout=after, dweight=grads["weight"])
        binding.adapters_backward(dz, x, u, self.a, self.b, self.scale, ids=ids, dropout=before, da=grads["a"], db=grads["b"])
        return (off * off).mean(), grads

    def step(self, x, residual, target, ids=None, lr: float = 1e-3, betas=(0.9, 0.95)):
        """One step of Adam; the loss before it (on the device)."""
        loss, grads = self.gradients(x, residual, target, ids)
        self.steps += 1
        for k, g in grads.items():
            m, v = self.moments[k]
            m.lerp_(g, 1 - betas[0])
            v.lerp_(g * g, 1 - betas[1])
            self.params[k] -= lr * (m / (1 - betas[0] ** self.steps)) / ((v / (1 - betas[1] ** self.steps)).sqrt() + 1e-12)
        self._cast()
        return loss


def main(steps: int = 200, tokens: int = 1024):
    import torch
    cfg = synth.scaled(synth.CONFIGS[1], d_model=512, d_ff=2752, n_centres=16)
    weights, source = synth.make_weights(cfg), synth.make_token_source(cfg)
    layer = binding.Layer.build(cfg, *weights, source.calibration())
    block = Block(layer, seed=0)

    def batch(i):
        x = torch.from_numpy(source.eval_batch(i, n=tokens)).to("cuda", block.dtype)
        residual = torch.zeros_like(x)
        dense, target = torch.empty_like(x), torch.empty_like(x)
        layer.dense_forward_device(x, dense)
        binding.norm_forward(dense, target, form=block.form, eps=block.eps)
        return x, residual, target

    def distance():
        x, residual, target = batch(10 ** 6)
        return float((block.serve(x, residual)[0].float() - target.float()).square().mean())

    first = distance()
    for i in range(steps):
        block.step(*batch(i))
    last = distance()
    print("mean squared distance to the dense layer on tokens of their own: %.4f before, %.4f after %d steps of %d tokens" % (first, last, steps, tokens))
    return first, last


if __name__ == "__main__":
    main()
