"""Several recovery blocks of one model, and what the adapters of one do."""
import pytest
import torch

from paper_2502_04416_amd import binding, recovery, synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layer():
    binding.load()
    cfg = synth.scaled(synth.CONFIGS[1], d_model=512, d_ff=2752, n_centres=16)
    source = synth.make_token_source(cfg)
    made = binding.Layer.build(cfg, *synth.make_weights(cfg), source.calibration())
    made.source = source
    yield made
    made.close()


def test_blocks_of_a_model_drop_elements_of_their_own(layer, monkeypatch):
    """No two batches of three steps of two blocks share a seed and an offset."""
    used = []
    for name in ("adapters_forward", "norm_forward"):
        def spy(*args, entry=getattr(binding, name), **kw):
            used.append((kw["dropout"].seed, kw["dropout"].offset))
            return entry(*args, **kw)
        monkeypatch.setattr(binding, name, spy)
    blocks = [recovery.Block(layer) for _ in range(2)]
    x, residual, target = (torch.randn(8, 512, device="cuda").to(blocks[0].dtype) for _ in range(3))
    for _ in range(3):
        for block in blocks:
            block.step(x, residual, target)
    assert len(used) == 12 and len(set(used)) == 12, used


def test_a_block_with_a_seed_keeps_its_masks(layer):
    a, b = recovery.Block(layer, seed=5), recovery.Block(layer, seed=5)
    assert a.seed == b.seed == 5 and torch.equal(a.params["a"], b.params["a"])


class Frozen(recovery.Block):
    """Only the norm's weight is trained."""

    def gradients(self, *args, **kw):
        loss, grads = super().gradients(*args, **kw)
        return loss, {k: g if k == "weight" else torch.zeros_like(g) for k, g in grads.items()}


def test_it_is_the_adapters_that_recover(layer):
    """Against a block whose adapters stay as they were, on tokens that neither was trained on.

    Without adapters the norm's weight can only scale: of a distance 2 - 2 c (c: cosine of the outputs, of unit mean square) it leaves
    1 - c^2 or so, 0.38 of 0.43.  Less than three quarters of that is the adapters' work."""
    def batch(i, dtype):
        x = torch.from_numpy(layer.source.eval_batch(i, n=1024)).to("cuda", dtype)
        dense, target = torch.empty_like(x), torch.empty_like(x)
        layer.dense_forward_device(x, dense)
        binding.norm_forward(dense, target, form="rms")
        return x, torch.zeros_like(x), target

    def distance(block, ids=None):
        x, residual, target = batch(10 ** 6, block.dtype)
        return float((block.serve(x, residual, ids)[0].float() - target.float()).square().mean())

    trained, frozen = recovery.Block(layer, seed=0), Frozen(layer, seed=0)
    first = distance(trained)
    assert distance(frozen) == first                         # (b is 0: no adapter yet)
    for i in range(200):
        for block in (trained, frozen):
            block.step(*batch(i, block.dtype))
    last, without = distance(trained), distance(frozen)
    none = distance(trained, torch.full((1024,), -1, dtype=torch.int32, device="cuda"))
    print("distance: %.4f at first, %.4f after training, %.4f with frozen adapters, %.4f of the trained block without its adapter" % (first, last, without, none))
    assert last < 0.75 * without and last < 0.75 * none
