"""Clipping where the factor's definition has to say what it is, on the GPU."""
import pytest
import torch

from test_gpu_operators import Arena

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2502_04416_amd import binding as b
    b.load()
    return b


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("max_norm", [0.0, 1.0, float("inf")])
def test_zeros_stay_zeros_where_norm_and_eps_are_zero(B, in_place, max_norm):
    m = Arena(1)
    grads, norm = [m.put(torch.zeros(40)), m.put(torch.zeros(3000, dtype=torch.bfloat16))], m.out(1)
    out = grads if in_place else [m.out(*g.shape, dtype=g.dtype) for g in grads]
    B.clip_gradients(grads, norm, max_norm, eps=0.0, out=None if in_place else out)
    assert float(norm) == 0 and all(bool((o == 0).all()) for o in out)
    m.intact()


def test_a_limit_of_zero_without_eps_clips_to_zeros_and_passes_nan_on(B):
    m = Arena(2)
    g, norm, out = m.normal(100), m.out(1), m.out(100)
    B.clip_gradients([g], norm, 0.0, eps=0.0, out=[out])
    assert float(norm) > 0 and bool((out == 0).all())
    g[5] = float("nan")
    B.clip_gradients([g], norm, 0.0, eps=0.0, out=[out])
    assert bool(torch.isnan(norm).all()) and bool(torch.isnan(out).all())
    m.intact()
