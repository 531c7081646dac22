"""The layer operators where a call's numbers are wrong or its values are no numbers: what is promised then, and nothing else
touched.  Tolerances are those of the parity tests."""
import numpy as np
import pytest
import torch

from .test_gpu_layer_ops import api, attention_inputs, check_attention, draw, f64, gen, ints, starts  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q_lens,kv_lens,max_q", [([0] * 15 + [16], [0] * 15 + [2100], 1), ([1] * 8 + [0] * 7 + [9], [2100, 700] * 4 + [0] * 7 + [3000], 1),
                                                  ([2, 3, 1, 5, 2, 3, 1, 3], [2500] * 8, 3)])
def test_attn_paged_more_new_tokens_than_the_bound(api, q_lens, kv_lens, max_q):  # noqa: F811
    """Requests with more tokens than max_q_len: the others' results stand, and the memory around the workspace, which ends
    where its stated size ends, is left alone; the next call on it is right."""
    H, D = 32, 64
    q, kc, vc, table, tab = attention_inputs(gen(700), q_lens, kv_lens, H, H, D, 64, poison=False)
    T, B, max_kv = sum(q_lens), len(q_lens), 4096
    size = api.attn_paged_workspace_size(T, B, H, H, D, max_q, max_kv)
    assert size > 1 << 18                                        # (there are parts in it)
    around = torch.full((size + (64 << 10),), 0x5A, dtype=torch.uint8, device="cuda")
    ws = around[32 << 10:(32 << 10) + size]
    ws.zero_()
    args = (q, kc, vc, ints(starts(q_lens)), ints(kv_lens), table, max_q, max_kv)
    out = torch.zeros_like(q)
    api.attn_paged(*args, out=out, workspace=ws)
    assert around[:32 << 10].eq(0x5A).all() and around[(32 << 10) + size:].eq(0x5A).all()
    want = api.attn_paged(*args[:6], max(q_lens), max_kv)
    cu = starts(q_lens)
    for b, n in enumerate(q_lens):
        if n <= max_q:
            np.testing.assert_allclose(f64(out[cu[b]:cu[b + 1]]), f64(want[cu[b]:cu[b + 1]]), atol=2.0 ** -7)
    ones = [min(n, 1) for n in q_lens]
    few = q[:sum(ones)]
    check_attention(api, few, kc, vc, table, tab, ones, kv_lens, workspace=ws)
