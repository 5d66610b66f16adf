"""Sizes that the entry points of the operators cannot take, on the CPU."""
import pytest
import torch

from paper_2502_04416_amd import binding

WIDE = [(1 << 31), (1 << 32) + 8]      # cut off to 32 bits: negative, and 8


def wide(*shape):
    return torch.empty(*shape, dtype=torch.bfloat16, device="meta")


@pytest.mark.parametrize("cols", WIDE)
def test_widths_beyond_32_bits_are_refused(cols):
    x = wide(1, cols)
    a, b, scale = wide(1, 1, cols), wide(1, 8, 1), torch.empty(1, device="meta")
    for call in (lambda: binding.dropout(x, x, binding.Dropout(0.5, 1)), lambda: binding.norm_forward(x, x),
                 lambda: binding.norm_backward(x, x, x, None, None), lambda: binding.adapters_forward(x, wide(1, 8), a, b, scale),
                 lambda: binding.adapters_backward(wide(1, 8), x, None, a, b, scale),
                 lambda: binding.adapters_backward(wide(1, cols), None, None, wide(1, 1, 8), wide(1, cols, 1), scale)):
        with pytest.raises(binding.CmoeError, match="32 bits"):
            call()


@pytest.mark.parametrize("eps", [1e39, 1e300, float("inf"), float("nan"), -1e-9])
def test_eps_that_is_no_fp32_number_is_refused(eps):
    with pytest.raises(binding.CmoeError, match="eps"):
        binding.norm_forward(wide(2, 8), wide(2, 8), eps=eps)
