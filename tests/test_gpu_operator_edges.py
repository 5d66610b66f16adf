"""Calls of the operators around the feed-forward layer at the edges of their buffers, against the 64-bit oracle.  Where the loads of such calls
begin is gone through on the host (test_operator_reads_cpu.py)."""
import pytest

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
