"""bf16 batches whose outputs are small differences: products with the factors that are kept in fp32 are those of all their 24 bits."""
import pytest
import torch

import operator_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2502_04416_amd import binding as b
    b.load()
    return b


def cancelling(t, d_in, d_out, rank, p, seed, device):
    """(x, dy, a, b, scale, ids, base, dx_base, mask): the bases are the rounded negatives of what the adapters add, so that an output is what rounding left."""
    from paper_2502_04416_amd.binding import Dropout
    rng = torch.Generator().manual_seed(seed)

    def bf16(*shape, std=1.0):
        return (torch.randn(*shape, generator=rng) * std).to(device, torch.bfloat16)

    x, dy, a, b = bf16(t, d_in), bf16(t, d_out), bf16(2, rank, d_in), bf16(2, d_out, rank)
    scale = (torch.rand(2, generator=rng) + 1).to(device)
    ids = (torch.arange(t) % 2).tolist()
    drop = Dropout(p, seed, 3) if p > 0 else None
    mask = O.mask(t, d_in, drop, device)
    want, _ = O.adapters(x, dy, a, b, scale, ids, None, None, mask)
    return x, dy, a, b, scale, ids, (-want["y"]).to(torch.bfloat16), (-want["dx"]).to(torch.bfloat16), drop, mask


@pytest.mark.parametrize("t,d_in,d_out,rank,p", [
    # narrow contractions, whose own roundings are few: of u over 8 and 16 values, of v likewise; every form of rows and block of ranks
    (24, 8, 520, 8, 0.0), (24, 520, 8, 8, 0.0), (600, 16, 264, 16, 0.25), (600, 264, 16, 16, 0.25), (9, 9, 515, 12, 0.0), (700, 515, 9, 3, 0.0),
    (40, 8, 256, 32, 0.0), (530, 8, 256, 64, 0.0), (8192, 8, 64, 40, 0.0),
])
def test_small_differences_of_the_base_and_the_adapter(B, monkeypatch, t, d_in, d_out, rank, p):
    x, dy, a, b, scale, ids, base, dx_base, drop, mask = cancelling(t, d_in, d_out, rank, p, t + rank, "cuda")
    monkeypatch.setattr(O, "SPLIT", 0.0)                     # no more than fp32 arithmetic may be off
    want, tol = O.adapters(x, dy, a, b, scale, ids, base, dx_base, mask)
    at = torch.tensor(ids, dtype=torch.int32, device="cuda")
    y, u, dx = torch.empty_like(base), torch.empty(t, rank, device="cuda"), torch.empty_like(dx_base)
    B.adapters_forward(x, y, a, b, scale, ids=at, base=base, dropout=drop, u=u)
    B.adapters_backward(dy, x, u, a, b, scale, ids=at, dx=dx, dx_base=dx_base, dropout=drop)
    O.check(y, want["y"], tol["y"], "y")
    O.check(dx, want["dx"], tol["dx"], "dx")
