"""Attention over the quantised cache near the ends of fp32's range."""
import pytest
import torch

from tests.test_gpu_layer_ops import gen
from tests.test_gpu_quant_cache import check_quant_attention, quant_attention_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available()
    from paper_2412_01034_b200 import api as a
    return a


def scaled(cache, side, power):
    """The cache with a side's scales times 2^power (exact: they stay normal numbers)."""
    s = getattr(cache, side).clone()
    (s if cache.bits == 8 else s[..., 0]).mul_(2.0 ** power)
    return cache._replace(**{side: s})


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("most", [2.0 ** 125, 2.0 ** 126, 1e38, 3e38])
@pytest.mark.parametrize("q_lens,kv_lens", [([1], [500]), ([6, 1], [77, 300]), ([12], [40]), ([200], [260])])
def test_queries_near_the_largest_number(api, q_lens, kv_lens, most, bits):
    """Every query row has an element of this size, keys are as small as queries are large: scores of ordinary size."""
    H, Hk, D = 2, 1, 128
    q, cache, table, tab = quant_attention_inputs(api, gen(1400), q_lens, kv_lens, H, Hk, D, 16, bits, poison=False)
    q = (q.double() / q.double().abs().amax(dim=2, keepdim=True) * most).to(torch.bfloat16)
    assert torch.isfinite(q).all() and (q.double().abs().amax(dim=2) > most * (1 - 2.0 ** -7)).all()
    cache = scaled(cache, "k_scale", -117)
    check_quant_attention(api, q, cache, table, tab, q_lens, kv_lens, scale=2.0 ** -6)
