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


# (requests, heads, key heads, dim, new tokens, cached tokens): the ways in which a request's parts are joined
JOINS = {"one_block": (1, 4, 2, 128, 1, 90), "cluster": (1, 8, 2, 128, 3, 700), "workspace": (8, 32, 32, 64, 1, 1000), "workspace_drafts": (9, 32, 32, 128, 4, 1500),
         "prompt": (2, 8, 2, 64, 70, 300), "prompt_parts": (1, 4, 2, 128, 60, 3000)}


@pytest.mark.parametrize("how", list(JOINS))
def test_attn_paged_nan_queries(api, how):  # noqa: F811
    """A query with a NaN gives NaN, on every way through the kernels; nothing else does."""
    B, H, Hk, D, n, kv = JOINS[how]
    q_lens, kv_lens = [n] * B, [kv - 3 * b for b in range(B)]
    q, kc, vc, table, _ = attention_inputs(gen(710), q_lens, kv_lens, H, Hk, D, 64)
    call = lambda: api.attn_paged(q, kc, vc, ints(starts(q_lens)), ints(kv_lens), table, n, kv)  # noqa: E731
    want, bad = call(), torch.zeros(B * n, H, dtype=torch.bool, device="cuda")
    assert torch.isfinite(want).all()
    for t, h in ((0, H - 1), (B * n - 1, 0), (B * n // 2, H // 2)):
        q[t, h, (5 * t + h) % D] = float("nan")
        bad[t, h] = True
    got = call()
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])


@pytest.mark.parametrize("B,H,D,chunk,max_kv", [(8, 32, 64, 896, 1000), (9, 32, 128, 1472, 1500), (40, 8, 64, 2048, 2100), (1, 2, 128, 128, 188)])
def test_attn_paged_a_nan_key_alone_in_its_part(api, B, H, D, chunk, max_kv):  # noqa: F811
    """The last cached token, which may be the only one of a block's part (parts of `chunk` tokens), has a key with a NaN: whoever sees it gets NaN."""
    for kv in (chunk, chunk + 1, chunk + 2):
        kv_lens = [kv] + [max_kv] * (B - 1)
        q, kc, vc, table, tab = attention_inputs(gen(720), [1] * B, kv_lens, H, H, D, 64)
        kc[tab[0, (kv - 1) // 64], 1, (kv - 1) % 64, 7] = float("nan")
        got = api.attn_paged(q, kc, vc, ints(starts([1] * B)), ints(kv_lens), table, 1, max_kv)
        bad = torch.zeros(B, H, dtype=torch.bool, device="cuda")
        bad[0, 1] = True
        assert torch.isnan(got[bad]).all() and torch.isfinite(got[~bad]).all(), kv


@pytest.mark.parametrize("q_lens,kv_lens,max_q,H,Hk", [([1, 40, 2], [90, 300, 7], 2, 4, 4), ([3, 100, 1, 9], [33, 500, 300, 9], 9, 8, 2), ([50, 120], [50, 130], 50, 4, 4)])
def test_attn_paged_one_request_beyond_the_bound(api, q_lens, kv_lens, max_q, H, Hk):  # noqa: F811
    """More rows in all than the bound on each allows: the requests that keep to it have their results."""
    q, kc, vc, table, tab = attention_inputs(gen(730), q_lens, kv_lens, H, Hk, 64, 16)
    want = check_attention(api, q, kc, vc, table, tab, q_lens, kv_lens)
    cu, out = starts(q_lens), torch.full_like(q, 77.0)
    api.attn_paged(q, kc, vc, ints(cu), ints(kv_lens), table, max_q, max(kv_lens), out=out)
    for b, n in enumerate(q_lens):
        if n <= max_q:
            np.testing.assert_allclose(f64(out[cu[b]:cu[b + 1]]), f64(want[cu[b]:cu[b + 1]]), atol=2.0 ** -6, err_msg=str(b))


def test_lora_batch_without_adapters_in_a_chain(api):  # noqa: F811
    """Prompts of which none has an adapter, in place (the second kernel has nothing to do), between work that changes what the
    call before and after reads: adapters, rows and workspace.  As in calls one by one."""
    g = gen(740)
    q_lens, K, N, r, n = [300, 17, 200, 90], 2048, 1024, 32, 2
    M, cu = sum(q_lens), ints(starts(q_lens))
    a, b, scales = draw(g, n, r, K, std=K ** -0.5), draw(g, n, N, r), torch.tensor([0.5, -1.0], device="cuda")
    picks = [ints(p) for p in ([-1] * 4, [0, -1, 1, 0], [-1, 2, 7, -5], [1, 1, 0, -1])]
    x0, y0 = draw(g, M, K), draw(g, M, N)
    size = api.lora_batch_workspace_size(M, len(q_lens), r)

    def chain(after):
        x, y, ad, ws = x0.clone(), y0.clone(), picks[0].clone(), api.new_workspace(size)
        for i in range(24):
            ad.copy_(picks[i % 4])
            after()
            api.lora_batch_add(x, a, b, y, cu, ad, scales, workspace=ws)
            after()
            ws.fill_(0xFF)
            x.mul_(-1.0)
            after()
        return y

    want = chain(torch.cuda.synchronize)
    assert torch.equal(chain(lambda: None), want) and torch.isfinite(want).all() and not torch.equal(want, y0)


def dirty_memory():
    """What the allocator hands out next is full of 0xFF."""
    torch.cuda.empty_cache()
    for n in (1 << 8, 1 << 12, 1 << 16, 1 << 18, 1 << 20, 1 << 22, 1 << 24, 1 << 26):
        block = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(3)]
        del block


def test_calls_without_a_workspace_clear_what_has_to_be_zero_and_no_more(api):  # noqa: F811
    """In memory that others have used: the results stand, and nothing but the counters of the attention is filled."""
    g = gen(750)
    q_lens, kv_lens = [1] * 8 + [60], [1000 - 7 * i for i in range(8)] + [4000]
    q, kc, vc, table, tab = attention_inputs(g, q_lens, kv_lens, 32, 32, 64, 64)
    attn = (q, kc, vc, ints(starts(q_lens)), ints(kv_lens), table, 60, 4000)
    M, K, N, r = 340, 2048, 1024, 64
    x, y, a, b = draw(g, M, K), draw(g, M, N), draw(g, 1, r, K, std=K ** -0.5), draw(g, 1, N, r)
    lora = (x, a, b, y, ints([0, M]), ints([0]), torch.ones(1, device="cuda"))
    out = torch.empty_like(y)
    want_l = api.lora_batch_add(*lora, out=torch.empty_like(y), workspace=api.new_workspace(api.lora_batch_workspace_size(M, 1, r)))
    want = check_attention(api, q, kc, vc, table, tab, q_lens, kv_lens,
                           workspace=api.new_workspace(api.attn_paged_workspace_size(sum(q_lens), 9, 32, 32, 64, 60, 4000)))
    for _ in range(3):
        dirty_memory()
        assert torch.equal(api.attn_paged(*attn), want) and torch.equal(api.lora_batch_add(*lora, out=out), want_l)
    # the fills that the calls enqueue
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA], acc_events=True) as prof:
        api.lora_batch_add(*lora, out=out)
        torch.cuda.synchronize()
    names = [e.key for e in prof.key_averages()]
    assert not [n for n in names if "fill" in n.lower() or "memset" in n.lower()], names


def test_lora_batch_single_rows_of_tensors_of_any_width(api):  # noqa: F811
    """One row of a matrix whose rows are no multiple of 8 long: the stride is of no account."""
    g = gen(760)
    K, N = 256, 128
    a, b, scales = draw(g, 1, 8, K, std=K ** -0.5), draw(g, 1, N, 8), torch.ones(1, device="cuda")
    x, y = draw(g, 1, K), draw(g, 1, N)
    want = api.lora_batch_add(x, a, b, y, ints([0, 1]), ints([0]), scales, out=torch.empty_like(y))
    for pad in (4, 13):
        wide_x, wide_y, wide_o = (torch.zeros(3, n + pad, dtype=torch.bfloat16, device="cuda") for n in (K, N, N))
        wide_x[:1, :K], wide_y[:1, :N] = x, y
        out = wide_o[:1, :N]
        api.lora_batch_add(wide_x[:1, :K], a, b, wide_y[:1, :N], ints([0, 1]), ints([0]), scales, out=out)
        assert torch.equal(out, want) and not wide_o[1:].any() and not wide_o[:, N:].any()
        api.lora_batch_add(wide_x[:1, :K], a, b, wide_y[:1, :N], ints([0, 1]), ints([0]), scales)
        assert torch.equal(wide_y[:1, :N], want) and not wide_y[1:].any() and not wide_y[:, N:].any()
        with pytest.raises(api.QilError):
            api.lora_batch_add(wide_x[:2, :K], a, b, draw(g, 2, N), ints([0, 2]), ints([0]), scales)


def test_attn_paged_bounds_are_not_cut_to_32_bits(api):  # noqa: F811
    q, kc, vc, table, _ = attention_inputs(gen(770), [1], [20], 4, 4, 64, 16)
    for max_q, max_kv in ((1 - 2 ** 32, 20), (1 + 2 ** 32, 20), (1, 20 - 2 ** 32), (1, 20 + 2 ** 32)):
        with pytest.raises(ValueError, match="32 bits"):
            api.attn_paged(q, kc, vc, ints([0, 1]), ints([20]), table, max_q, max_kv)
    for max_q, max_kv in ((-1, 20), (0, 20), (1, 0)):
        with pytest.raises(api.QilError):
            api.attn_paged(q, kc, vc, ints([0, 1]), ints([20]), table, max_q, max_kv, workspace=api.new_workspace(1 << 20))


@pytest.mark.parametrize("q_lens", [[1, 3, 2], [40, 100, 33]])
@pytest.mark.parametrize("r", [8, 16, 24, 32, 64])
def test_lora_batch_inner_products_beyond_bf16(api, q_lens, r):  # noqa: F811
    """Inner products that are infinite, or finite and larger than bf16's largest number, enter the second product as such."""
    g = gen(780 + r)
    K, N, M, cu = 264, 72, sum(q_lens), starts(q_lens)
    x, y = draw(g, M, K), draw(g, M, N)
    a, b = draw(g, 1, r, K, std=K ** -0.5), draw(g, 1, N, r).abs() * 2.0 ** -70
    a[0, :, 5], a[0, :, 77] = 3.38953139e38, 1e36
    x[:, 5] = x[:, 77] = 0
    big, inf = cu[1], cu[2] - 1
    x[big] = 0
    x[big, 5] = x[big, 77] = 1.0      # 3.3995e38: fp32 holds it, bf16 rounds it to infinity
    x[inf, 100] = float("inf")
    a[0, :, 100] = 0.5
    out = api.lora_batch_add(x, a, b, y, ints(cu), ints([0] * len(q_lens)), torch.ones(1, device="cuda"), out=torch.empty_like(y))
    t = f64(x[big:big + 1]) @ f64(a[0]).T
    assert (t > 3.3896e38).all() and (t < 3.4028e38).all()
    want = f64(y[big:big + 1]) + t @ f64(b[0]).T
    got = f64(out)
    assert np.all(np.abs(got[big] - want) <= (2.0 ** -8 + (K + 2 * r + 8) * 2.0 ** -24 + 2.0 ** -16) * np.abs(want))
    assert np.all(got[inf] == np.inf)
    assert np.all(np.isfinite(np.delete(got, inf, axis=0)))


@pytest.mark.parametrize("K", [64, 4096, 20000])
@pytest.mark.parametrize("x_std,w_std,eps", [(1e-35, 1.0, 1e-5), (2e-37, 1.0, 1e-5), (1e-37, 1.0, 1e-5), (1e-36, 1e-2, 1e-5), (1.0, 1e-35, 1e-5), (1e-18, 1e-20, 1e-6),
                                             (1e-17, 3e-18, 1e-6)])
@pytest.mark.parametrize("with_residual", [False, True])
def test_rmsnorm_codes_of_tiny_rows(api, K, x_std, w_std, eps, with_residual):  # noqa: F811
    """Rows near the end of fp32's range: their codes are those of the formula, or, below the stated limit, those of zeros.  (The
    sum x + residual and the product with the weight round to fp32, 2^-23 of the largest, or to multiples of 2^-149.)"""
    from oracle import np_layer
    g = gen(790 + K)
    x, w = draw(g, 9, K, std=x_std), draw(g, K, std=w_std)
    r = draw(g, 9, K, std=x_std) if with_residual else None
    v, h = np_layer.rmsnorm(f64(x), f64(w), eps, None if r is None else f64(r))
    top = np.abs(h * f64(w)).max(axis=1)
    both = torch.empty_like(x)
    codes, scales, *_ = api.rmsnorm_a8(x, w, eps, residual=r, out=both)
    s, got, codes = np_layer.a8_scale(v), f64(scales), f64(codes)
    zero, full = top < 2.0 ** -119 * (1 - 2.0 ** -20), top > 2.0 ** -119 * (1 + 2.0 ** -20)
    assert not codes[zero].any() and np.all(got[zero] == 1)
    assert np.all(np.abs(got - s)[full] <= 2.0 ** -17 * s[full])
    assert np.all(np.abs(codes - v / s[:, None])[full] <= 0.5 + 127 * (2.0 ** -16 + 2.0 ** -149 / top[full, None]))
    assert np.all(np.abs(f64(both) - v) <= (2.0 ** -8 + 2.0 ** -16) * np.abs(v) + 2.0 ** -134)


@pytest.mark.parametrize("K", [64, 4096, 20000])
def test_rmsnorm_nan_rows_have_nan_scales(api, K):  # noqa: F811
    """A NaN anywhere in a row, or everywhere, shows in the row's scale and norm; the other rows are as without it."""
    g = gen(800 + K)
    x, w = draw(g, 4, K), draw(g, K)
    _, want = api.rmsnorm_a8(x, w)
    y = api.rmsnorm(x, w)
    x[1], x[3, K // 2] = float("nan"), float("nan")
    both = torch.empty_like(x)
    _, scales = api.rmsnorm_a8(x, w, out=both)
    assert torch.isnan(scales[[1, 3]]).all() and torch.equal(scales[[0, 2]], want[[0, 2]])
    assert torch.isnan(both[[1, 3]]).all() and torch.equal(both[[0, 2]], y[[0, 2]])
