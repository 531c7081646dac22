"""Attention over the quantised cache near the ends of fp32's range."""
import numpy as np
import pytest
import torch

from tests.test_gpu_layer_ops import f64, gen, ints, starts
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


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("q_lens,kv_lens,D", [([1, 5], [300, 129], 128), ([200], [260], 128), ([130, 1], [1000, 70], 64)])
def test_scores_too_small_for_their_factor(api, q_lens, kv_lens, D, bits):
    """Keys and queries so small that a score's factor is no number above zero: weights are all the same, as they are with a scale
    of zero."""
    q, cache, table, tab = quant_attention_inputs(api, gen(1410), q_lens, kv_lens, 4, 2, D, 32, bits, q_std=1e-13)
    cache = scaled(cache, "k_scale", -110)
    args = (ints(starts(q_lens)), ints(kv_lens), table, max(q_lens), max(kv_lens))
    assert torch.equal(api.attn_paged_q(q, cache, *args), api.attn_paged_q(q, cache, *args, scale=0.0))
    check_quant_attention(api, q, cache, table, tab, q_lens, kv_lens)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("q_lens,kv_lens,D", [([200], [500], 128), ([60, 40], [510, 333], 64), ([200], [700], 128), ([60, 40], [3000, 2500], 64)])
def test_values_near_the_smallest_number(api, q_lens, kv_lens, D, bits):
    """Of prompts, in one part of the cache and in several: values by a power of two smaller give results by that power smaller, up
    to bf16's own smallest step."""
    q, cache, table, _ = quant_attention_inputs(api, gen(1420), q_lens, kv_lens, 2, 2, D, 64, bits, q_std=0.1)
    args = (ints(starts(q_lens)), ints(kv_lens), table, max(q_lens), max(kv_lens))
    if bits == 8:   # values of one sign: results of their size
        cache.v.clamp_(min=0)
    else:
        cache.v_scale[..., 1] = 0
    power = 119 if bits == 8 else 122   # (scales of 2^-126 to 2^-124)
    want = api.attn_paged_q(q, cache, *args)
    got = api.attn_paged_q(q, scaled(cache, "v_scale", -power), *args)
    # results below 2^-126 are whole numbers of 2^-133: each is off by half of one, and the two roundings by one together
    assert np.abs(f64(got) * 2.0 ** power - f64(want)).max() <= 2.0 ** (power - 133)
