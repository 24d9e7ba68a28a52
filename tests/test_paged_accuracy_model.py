"""The bounds of tests/paged_accuracy.py hold what the kernels keep and fail what they could lose (no GPU: 64 bits with the roundings put in)."""
import pytest
import torch

from paged_accuracy import CASES, attention, batch, bounds, half_step


@pytest.mark.parametrize("name", sorted(CASES))
def test_a_shared_latents_key_in_two_parts_and_in_one(name):
    b = batch(name, True)
    ref = attention(b, 64)
    to, tl, mean = bounds(b, *ref)
    two, one = (attention(b, 64, key_parts=parts)[1] - ref[1] for parts in (2, 1))
    assert (two.abs() <= tl / 2).all() and two.square().mean().sqrt() <= mean / 2
    assert one.square().mean().sqrt() > 2 * mean


@pytest.mark.parametrize("name,shared", [(n, s) for n, c in sorted(CASES.items()) if c[5] for s in (False, True) if (n, s) != ("split", True)])
def test_a_probability_in_two_parts_and_in_one(name, shared):
    b = batch(name, shared)
    ref = attention(b, 64)
    to, _, _ = bounds(b, *ref)
    for parts, ok in ((2, True), (1, False)):
        O = attention(b, 64, p_parts=parts)[0].bfloat16().double()
        over = ((O - ref[0]).abs() > half_step(ref[0]) + to).double().mean()
        assert (over == 0) == ok
