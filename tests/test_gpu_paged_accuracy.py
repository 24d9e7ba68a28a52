"""The attention over pages within bounds as narrow as what its kernels keep (tests/paged_accuracy.py): a key of a shared latent in two bf16
parts everywhere, probabilities in two for single and proposed tokens of up to 32 rows."""
import pytest
import torch

from paged_accuracy import CASES, attention, batch, bounds, half_step
from test_gpu_paged import Context, attend, on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("name", sorted(CASES))
def test_narrow_bounds(name, shared):
    _, _, _, heads, r, two = CASES[name]
    b = batch(name, shared)
    ref = attention(b, 64)
    to, tl, mean = bounds(b, *ref)
    with Context(heads, r, r, "bf16", shared=shared) as c:
        O, L = attend(c, b, *on_gpu(b))
    err = L.cpu().double() - ref[1]
    assert (err.abs() <= tl).all(), f"lse: {float((err.abs() / tl).max()):.3g} of its bound"
    assert err.square().mean().sqrt() <= mean, f"lse: {float(err.square().mean().sqrt() / mean):.3g} of its mean bound"
    if two:
        over = (O.cpu().double() - ref[0]).abs() / (half_step(ref[0]) + to)
        assert over.max() <= 1, f"O: {float(over.max()):.3g} of its bound"
