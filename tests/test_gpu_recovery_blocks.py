"""Several recovery blocks of one model."""
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
