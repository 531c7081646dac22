"""Weights of the sampler next to where they round to nothing."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [3, 5000])
def test_the_smallest_weight_is_half_a_unit(V):
    """exp(x) is held in multiples of 2^-42: above -43 log(2) it is one of them, below it is none.  With u of 1 the token is the last
    one that has any weight."""
    from paper_2412_01034_b200 import api
    edge = -43 * math.log(2.0)
    u, t = torch.tensor([1.0], device="cuda"), torch.tensor([1.0], device="cuda")
    for x, has_weight in ((edge + 1e-4, True), (edge + 0.003, True), (-29.801, True), (-29.5, True), (edge - 1e-4, False), (edge - 1.0, False)):
        logits = torch.full((1, V), -1e9)
        logits[0, 0], logits[0, V - 1] = 0.0, x
        for more in ({}, dict(top_k=torch.tensor([V - 1], dtype=torch.int32, device="cuda"))):
            assert api.sample(logits.cuda(), u, t, **more).item() == (V - 1 if has_weight else 0), (x, more)
