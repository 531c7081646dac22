"""Attention of prompts over the quantised cache against what the codes stand for, (q - z) s in 64 bits: nothing of the reference is
rounded as the kernel rounds, and what its rounding may cost is derived here.

With u = 2^-11, half a step of fp16: a key's element is off by u of it, and so a score by u sum_d |q_d k_d| |scale| (a query has
bf16's 8 bits, of which fp16 holds all down to 2^-14 of the row's largest element, and steps of 2^-25 of it below), next to fp32's
products and sums.  Scores off by e at most change a weight, over its sum, by a factor of exp(2 e) at most.  A weight and a value are off
by u each, exp2 and the sums in fp32 by 2^-14 together, a weight below 2^-14 of the reference by 2^-25; then the result's own rounding.
"""
import numpy as np
import pytest
import torch

from oracle import np_layer, np_quant_cache
from tests.test_gpu_layer_ops import BF16_HALF_ULP, assert_within, f64, gen, ints, starts
from tests.test_gpu_quant_cache import parts_of, quant_attention_inputs

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -11


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available()
    from paper_2412_01034_b200 import api as a
    return a


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("q_std", [0.25, 1.0, 4.0, 16.0, 30.0])
@pytest.mark.parametrize("q_lens,kv_lens,H,Hk,D,page", [([200], [500], 2, 1, 128, 32), ([100, 33], [100, 290], 4, 4, 64, 16), ([40, 20], [2600, 300], 8, 2, 128, 64),
                                                        ([1, 60, 0, 300], [9, 61, 5, 300], 3, 1, 64, 128)])
def test_prompts_against_the_values_of_the_codes(api, q_lens, kv_lens, H, Hk, D, page, q_std, bits):
    q, cache, table, tab = quant_attention_inputs(api, gen(1500 + D + len(q_lens)), q_lens, kv_lens, H, Hk, D, page, bits, q_std=q_std)
    cu, G, scale = starts(q_lens), H // Hk, D ** -0.5
    got = f64(api.attn_paged_q(q, cache, ints(cu), ints(kv_lens), table, max(q_lens), max(kv_lens)))
    qd = f64(q)
    sides = [np_quant_cache.values(*p, bits) for p in parts_of(cache)]
    for b, (n, kv) in enumerate(zip(q_lens, kv_lens)):
        if n * G <= 16:
            continue
        rows = slice(cu[b], cu[b] + n)
        k, v = (np_layer.gather_cache(side, tab[b], kv) for side in sides)
        want, spread, absdot = np_layer.attn(qd[rows], k, v, kv - n, scale)
        sizes = np.repeat(np.abs(k).sum(axis=2).max(axis=0), G)[None] * np.abs(qd[rows]).max(axis=2) * scale
        e = (HALF + (D + 8) * 2.0 ** -24) * absdot + 2.0 ** -25 * sizes
        factor = np.exp(2 * e)[:, :, None]
        off = (factor - 1 + factor * (2 * HALF + 2.0 ** -14)) * spread + 2.0 ** -25 * np.repeat(np.abs(v).sum(axis=0), G, axis=0)[None]
        assert_within(got[rows], want, off + BF16_HALF_ULP * (np.abs(want) + off) + 1e-30)
