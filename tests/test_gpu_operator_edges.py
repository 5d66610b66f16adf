"""Calls of the operators around the feed-forward layer at the edges of their buffers, against the 64-bit oracle.  Where the loads of such calls
begin is gone through on the host (test_operator_reads_cpu.py)."""
import pytest
import torch

import operator_oracle as O
import test_gpu_operators as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2502_04416_amd import binding as b
    b.load()
    return b


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", [
    # a tile whose last rows are one token with the bank's last adapter, widths that end 8 to 32 values past a multiple of 64
    (1, 96, 96, 8, 1, "one", 0.0, True), (513, 96, 72, 8, 2, "one", 0.1, True), (5, 64, 96, 1, 2, "one", 0.0, True),
    (1, 8, 8, 8, 1, "one", 0.0, True), (1, 72, 32, 16, 2, "one", 0.1, False), (1, 800, 1376, 8, 3, "one", 0.0, True), (1, 4128, 96, 32, 2, "one", 0.1, True),
    (17, 32, 8, 8, 2, "one", 0.0, True), (3, 16, 16, 2, 2, "one", 0.1, True), (4, 24, 8, 1, 1, "one", 0.0, True), (513, 200, 136, 8, 5, "one", 0.1, True),
    (529, 72, 72, 24, 2, "one", 0.0, True), (8193, 72, 96, 64, 2, "one", 0.1, True),
], ids=lambda c: "-".join(map(str, c)))
def test_adapters_of_a_last_token(B, dtype, case):
    T.test_adapters(B, dtype, case)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", [
    # widths and buffers below eight values, wide ranks: most rows of a unit of b lie behind its last column
    (1, 4, 40, 64, 1, "one", 0.0, True), (3, 5, 33, 64, 2, "mixed", 0.2, True), (600, 7, 1, 33, 3, "one", 0.1, True), (1, 640, 3, 64, 1, "one", 0.0, False),
], ids=lambda c: "-".join(map(str, c)))
def test_adapters_of_tiny_widths(B, dtype, case):
    T.test_adapters(B, dtype, case)


def test_gradients_of_a_bank_of_many_wide_adapters(B):
    """More sums than one axis of a launch takes (2^32 threads): every adapter without a token has gradients of 0."""
    n, d_in, d_out, t = 8191, 8, 65568, 2
    z = dict(device="cuda")
    ids = torch.tensor([n - 1, 0], dtype=torch.int32, **z)
    rng = torch.Generator().manual_seed(4)
    dy, x = (torch.randn(t, d, generator=rng).to("cuda", torch.bfloat16) for d in (d_out, d_in))
    u, scale = torch.randn(t, 1, generator=rng).cuda(), torch.full((n,), 2.0, **z)
    a, b = torch.ones(n, 1, d_in, dtype=torch.bfloat16, **z), torch.zeros(n, d_out, 1, dtype=torch.bfloat16, **z)
    da, db = torch.full((n, 1, d_in), float("nan"), **z), torch.full((n, d_out, 1), float("nan"), **z)
    B.adapters_backward(dy, x, u, a, b, scale, ids=ids, da=da, db=db)
    assert not da.any()                                     # (b is 0)
    for i, k in enumerate(ids.tolist()):                    # one product of three roundings
        want = 2.0 * dy[i].double() * u[i].double()
        assert bool(((db[k, :, 0].double() - want).abs() <= 4 * O.U32 * want.abs()).all()), k
    assert not db[1:n - 1].any()
