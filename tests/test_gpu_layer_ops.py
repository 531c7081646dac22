"""GPU parity of the operators between the linears of a decoder layer, against the 64-bit oracle.

Tolerances follow from the arithmetic: a bf16 result carries half a unit of its 8 significant bits (2^-8 of its value);
what is added to it is stated at each test.
"""
import numpy as np
import pytest
import torch

from oracle import np_layer

pytestmark = pytest.mark.gpu

BF16_HALF_ULP = 2.0 ** -8


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available()
    from paper_2412_01034_b200 import api as a
    return a


def draw(g, *shape, std=1.0):
    return (torch.randn(shape, generator=g) * std).to(torch.bfloat16).cuda()


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def starts(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(int).tolist()


def assert_within(got, want, tol):
    err = np.abs(got - want)
    assert np.all(np.isfinite(got))
    assert np.all(err <= tol), f"{(err / np.maximum(tol, 1e-300)).max():.3f} of the tolerance at {np.unravel_index((err - tol).argmax(), err.shape)}"


# ------------------------------------------------------------------------------------------------------------------
# residual norm
# ------------------------------------------------------------------------------------------------------------------
NORM_SHAPES = [(1, 4096), (1, 8), (3, 24), (7, 2176), (280, 4096), (33, 1000), (2, 11008), (5, 8200), (2, 32768), (3, 16392), (700, 256)]


# The fp32 chain of a value: the sum of squares (at most 40 dependent additions per thread and 10 over the block), the
# root, the division and two products: under 64 roundings of 2^-24 each, 2^-18 of the value.
@pytest.mark.parametrize("M,K", NORM_SHAPES)
@pytest.mark.parametrize("with_residual", [True, False])
def test_rmsnorm(api, M, K, with_residual):
    g = gen(M * 7 + K)
    x, w = draw(g, M, K), draw(g, K)
    r = draw(g, M, K, std=2.0) if with_residual else None
    x[0] *= 100.0
    v, h = np_layer.rmsnorm(f64(x), f64(w), 1e-5, None if r is None else f64(r))
    got = api.rmsnorm(x, w, 1e-5, residual=r)
    y = got[0] if with_residual else got
    assert_within(f64(y), v, (BF16_HALF_ULP + 2.0 ** -16) * np.abs(v))
    if with_residual:
        assert torch.equal(got[1], (x.float() + r.float()).to(torch.bfloat16))
    # the quantised form: the scale is fp32 arithmetic, a code is within half a step of v / s plus 127 times that error
    both = torch.empty_like(x)
    codes, scales, *rest = api.rmsnorm_a8(x, w, 1e-5, residual=r, out=both)
    assert torch.equal(both, y)
    s = np_layer.a8_scale(v)
    assert_within(f64(scales), s, 2.0 ** -17 * s)
    assert_within(f64(codes), v / s[:, None], np.full_like(v, 0.5 + 127 * 2.0 ** -16))
    assert int(codes.abs().max()) == 127
    if with_residual:
        assert torch.equal(rest[0], got[1])
    else:
        assert not rest


def test_rmsnorm_in_place_zero_rows_and_eps(api):
    g = gen(5)
    x, w = draw(g, 4, 512), draw(g, 512)
    r = -x.clone()
    r[2] = 0
    y, h = api.rmsnorm(x, w, 1e-5, residual=r, residual_out=r)
    assert h is r and torch.equal(h[2], x[2]) and not h[[0, 1, 3]].any()
    assert not y[[0, 1, 3]].any() and y[2].any()
    codes, scales = api.rmsnorm_a8(h, w, 1e-5)
    assert scales[[0, 1, 3]].eq(1).all() and not codes[[0, 1, 3]].any()
    # a row far below eps: the norm is x / sqrt(eps)
    tiny = torch.full((1, 64), 2.0 ** -40, dtype=torch.bfloat16, device="cuda")
    y = api.rmsnorm(tiny, torch.ones(64, dtype=torch.bfloat16, device="cuda"), 1.0)
    assert_within(f64(y), np.full((1, 64), 2.0 ** -40), np.full((1, 64), 2.0 ** -48))


def test_rmsnorm_codes_feed_the_w8a8_linear(api):
    g = gen(6)
    x, w = draw(g, 40, 512), draw(g, 512)
    qw = torch.randint(-128, 128, (96, 512), generator=g, dtype=torch.int8).cuda()
    sw = (torch.rand(96, generator=g) * 0.01 + 0.001).cuda()
    codes, scales = api.rmsnorm_a8(x, w)
    y, acc = api.linear_w8a8(codes, scales, qw, sw, want_acc=True)
    assert torch.equal(acc.cpu().long(), codes.cpu().long() @ qw.cpu().long().t())


# ------------------------------------------------------------------------------------------------------------------
# rotary embedding and append
# ------------------------------------------------------------------------------------------------------------------
def paged(g, kv_lens, page, spare=3, garbage=True):
    """A block table over shuffled pages; entries past a request's last page are garbage."""
    need = [-(-n // page) for n in kv_lens]
    order = torch.randperm(sum(need) + spare, generator=g).tolist()
    width = max(max(need), 1) + 1
    table = np.full((len(kv_lens), width), 2 ** 31 - 1 if garbage else 0, dtype=np.int64)
    table[::2, -1] = -7
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return ints(table.tolist()), table, sum(need) + spare


ROPE_CASES = [  # (q_lens, kv_lens, H, Hk, D, page)
    ([1], [1], 4, 4, 128, 16),
    ([1, 1, 1], [40, 7, 129], 8, 2, 128, 32),
    ([5, 0, 17, 1], [5, 9, 60, 1], 7, 1, 64, 64),
    ([33, 70], [33, 200], 32, 32, 128, 128),
    ([4, 3], [2, 3], 2, 2, 64, 16),          # more new tokens than cached ones: the first have no place
    ([1] * 70, list(range(1, 71)), 3, 1, 64, 16),
]


@pytest.mark.parametrize("case", range(len(ROPE_CASES)))
def test_rope_append(api, case):
    q_lens, kv_lens, H, Hk, D, page = ROPE_CASES[case]
    g = gen(100 + case)
    table, tab, pages = paged(g, kv_lens, page)
    T, cu = sum(q_lens), starts(q_lens)
    qkv = draw(g, T, (H + 2 * Hk) * D)
    kc, vc = draw(g, pages, Hk, page, D), draw(g, pages, Hk, page, D)
    k0, v0 = kc.clone(), vc.clone()
    cs = api.rope_table(max(kv_lens), D)
    q = api.rope_append(qkv, cs, kc, vc, ints(cu), ints(kv_lens), table, H)
    x = f64(qkv).reshape(T, H + 2 * Hk, D)
    want_k, want_v, touched = f64(k0), f64(v0), np.zeros((pages, page), dtype=bool)
    tol_k = np.zeros_like(want_k)
    for t, (b, p) in enumerate(zip(*np_layer.positions(cu, kv_lens))):
        if p < 0:
            assert not q[t].any()
            continue
        turned = np_layer.rope_rotate(x[t, : H + Hk], p, 10000.0)
        # the table's fp32 entries (2^-24 each), two products and a sum of the pair's values
        pair = np.abs(x[t, : H + Hk, : D // 2]) + np.abs(x[t, : H + Hk, D // 2:])
        tol = BF16_HALF_ULP * np.abs(turned) + 2.0 ** -22 * np.concatenate([pair, pair], axis=1)
        assert_within(f64(q[t]), turned[:H], tol[:H])
        pg, slot = tab[b, p // page], p % page
        want_k[pg, :, slot], want_v[pg, :, slot], tol_k[pg, :, slot] = turned[H:], x[t, H + Hk:], tol[H:]
        touched[pg, slot] = True
    assert_within(f64(kc), want_k, tol_k)
    np.testing.assert_array_equal(f64(vc), want_v)
    same = torch.from_numpy(~touched).cuda()[:, None, :, None].expand_as(kc)
    assert torch.equal(kc[same], k0[same]) and torch.equal(vc[same], v0[same])


def test_rope_append_skips_what_has_no_place(api):
    """Positions past the angle table, past the block table and in pages that do not exist: skipped, nothing else written."""
    g = gen(9)
    H, Hk, D, page, pages = 2, 1, 64, 16, 4
    qkv = draw(g, 6, (H + 2 * Hk) * D)
    kc, vc = api.new_kv_cache(pages, Hk, page, D)
    table = ints([[0, 99], [-1, 1], [2, 3]])
    cs = api.rope_table(33, D)
    q = api.rope_append(qkv, cs, kc, vc, ints([0, 2, 4, 6]), ints([18, 18, 34]), table, H)
    # request 0: positions 16, 17 in page 99; request 1: 16, 17 in page 1; request 2: 32 beyond its two pages, 33 beyond the angles
    assert vc[1, 0, :2].any() and not vc[1, 0, 2:].any()
    assert not vc[[0, 2, 3]].any() and not kc[[0, 2, 3]].any()
    assert q[:5].any(dim=2).all() and not q[5].any()


# ------------------------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------------------------
LENGTHS = {
    "single": ([1], [1]),
    "decode": ([1, 1, 1, 1, 1], [1, 2, 17, 130, 611]),
    "empty_requests": ([0, 1, 3, 0, 2], [5, 1, 200, 0, 2]),
    "rows_that_see_nothing": ([5, 1, 9], [3, 0, 9]),
    "prompts": ([1, 127, 128, 129, 300], [1, 127, 128, 129, 300]),
    "chunks": ([64, 1, 200], [1000, 513, 257]),
    "mixed": ([150, 1, 1, 1, 2], [150, 400, 1, 33, 90]),
    "prompt_that_sees_little": ([140], [130]),
    "few_new_tokens": ([4, 2, 8, 3], [257, 2, 8, 1500]),
}


def attention_inputs(g, q_lens, kv_lens, H, Hk, D, page, q_std=1.0, poison=True):
    table, tab, pages = paged(g, kv_lens, page)
    q = draw(g, sum(q_lens), H, D, std=q_std)
    kc, vc = draw(g, pages, Hk, page, D), draw(g, pages, Hk, page, D)
    if poison:   # everything that belongs to no cached token is infinite or NaN
        live = np.zeros((pages, page), dtype=bool)
        for b, n in enumerate(kv_lens):
            for j in range(n):
                live[tab[b, j // page], j % page] = True
        dead = torch.from_numpy(~live).cuda()
        for c, bad in ((kc, float("inf")), (vc, float("nan"))):
            c.masked_fill_(dead[:, None, :, None], bad)
        kc[dead[:, None, :].expand(-1, Hk, -1)] *= torch.tensor([1.0, -1.0], device="cuda").repeat(D // 2).to(torch.bfloat16)
    return q, kc, vc, table, tab


def check_attention(api, q, kc, vc, table, tab, q_lens, kv_lens, scale=None, out=None, **kw):
    cu, D = starts(q_lens), q.shape[2]
    got = api.attn_paged(q, kc, vc, ints(cu), ints(kv_lens), table, max(max(q_lens), 1), max(max(kv_lens), 1), scale=scale, **kw)
    scale = D ** -0.5 if scale is None else scale
    qd, kd, vd, gd = f64(q), f64(kc), f64(vc), f64(got)
    for b, (n, kv) in enumerate(zip(q_lens, kv_lens)):
        if n == 0:
            continue
        lo = cu[b]
        want, spread, absdot = np_layer.attn(qd[lo:lo + n], np_layer.gather_cache(kd, tab[b], kv), np_layer.gather_cache(vd, tab[b], kv),
                                             kv - n, scale)
        # scores: fp32 sums of D products, each off by at most D 2^-24 of the absolute sum; a weight changes by as much,
        # relatively, once in the numerator and once in the sum.  Weights rounded to bf16 (2^-8 of each), exp2 and the
        # sums of weights and products in fp32 (2^-14 covers 1024 roundings).
        weight = BF16_HALF_ULP + 2 * (D + 4) * 2.0 ** -24 * absdot[:, :, None] + 2.0 ** -14
        assert_within(gd[lo:lo + n], want, BF16_HALF_ULP * np.abs(want) + weight * spread + 1e-30)
    return got


@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("H,Hk,D,page", [(4, 4, 128, 16), (8, 2, 128, 64), (7, 1, 64, 32), (6, 2, 64, 128), (3, 3, 64, 16), (12, 3, 128, 128)])
def test_attn_paged(api, lengths, H, Hk, D, page):
    q_lens, kv_lens = LENGTHS[lengths]
    g = gen(1000 + H * 10 + D + page)
    args = attention_inputs(g, q_lens, kv_lens, H, Hk, D, page)
    check_attention(api, *args, q_lens, kv_lens)


@pytest.mark.parametrize("H,Hk", [(32, 1), (40, 2), (17, 1)])
def test_attn_paged_wide_groups(api, H, Hk):
    q_lens, kv_lens = [1, 9, 1], [300, 77, 5]
    args = attention_inputs(gen(H), q_lens, kv_lens, H, Hk, 64, 16)
    check_attention(api, *args, q_lens, kv_lens)


@pytest.mark.parametrize("q_std,scale", [(30.0, None), (1.0, 0.0), (1.0, -0.5), (0.01, 1.0), (60.0, 1.0)])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [700, 65]), ([200], [500])])
def test_attn_paged_scores_of_every_size(api, q_std, scale, q_lens, kv_lens):
    args = attention_inputs(gen(77), q_lens, kv_lens, 4, 2, 128, 32, q_std=q_std)
    check_attention(api, *args, q_lens, kv_lens, scale=scale)


@pytest.mark.parametrize("q_lens", [[1], [130]])
def test_attn_paged_growing_scores(api, q_lens):
    """Scores that grow along the cache: the running maximum changes in every step."""
    kv = 1500
    q, kc, vc, table, tab = attention_inputs(gen(78), q_lens, [kv], 2, 2, 128, 16)
    ramp = torch.linspace(0.0, 20.0, kv)
    for j in range(kv):
        kc[tab[0, j // 16], :, j % 16] = 0
        kc[tab[0, j // 16], :, j % 16, 0] = ramp[j].item()
    q[:, :, 0] = 10.0
    check_attention(api, q, kc, vc, table, tab, q_lens, [kv], scale=1.0)


@pytest.mark.parametrize("q_lens,kv_lens", [([1], [20011]), ([1, 1], [9000, 3]), ([130], [6100]), ([20, 20], [5000, 2600])])
def test_attn_paged_long_caches_are_split(api, q_lens, kv_lens):
    args = attention_inputs(gen(79), q_lens, kv_lens, 2, 1, 128, 64, poison=False)
    check_attention(api, *args, q_lens, kv_lens)


def test_attn_paged_is_deterministic_and_its_workspace_is_reusable(api):
    cases = [([1] * 6, [900, 33, 2000, 1, 64, 700], 8, 8), ([70, 1], [3000, 20], 8, 2), ([1], [5000], 2, 1), ([300], [300], 4, 4)]
    size = max(api.attn_paged_workspace_size(sum(q), len(q), H, Hk, 128, max(q), max(kv)) for q, kv, H, Hk in cases)
    ws = api.new_workspace(size)
    first = []
    for again in range(2):
        for i, (q_lens, kv_lens, H, Hk) in enumerate(cases):
            args = attention_inputs(gen(80 + i), q_lens, kv_lens, H, Hk, 128, 16)
            if again:
                got = api.attn_paged(args[0], args[1], args[2], ints(starts(q_lens)), ints(kv_lens), args[3], max(q_lens), max(kv_lens), workspace=ws)
                assert torch.equal(got, first[i])
            else:
                first.append(check_attention(api, *args, q_lens, kv_lens, workspace=ws))
    assert int(ws[:4].view(torch.int32)[0]) == 0


@pytest.mark.parametrize("q_len,kv,H,Hk,D,page", [(6, 300, 4, 2, 128, 16), (16, 16, 3, 3, 64, 32), (5, 4100, 3, 1, 128, 64), (16, 700, 2, 2, 64, 16),
                                                  (300, 500, 2, 2, 128, 16), (280, 280, 4, 1, 64, 64), (70, 70, 6, 2, 128, 128), (130, 6100, 2, 1, 128, 64)])
@pytest.mark.parametrize("scale", [None, -0.1, 0.0])
def test_attn_paged_values_that_are_not_finite_stay_out_of_earlier_tokens(api, q_len, kv, H, Hk, D, page, scale):
    """A new token's value holds a NaN and an infinity, the last one's key is infinite: the new tokens before them are as if
    they were not there, the others get them in their columns (the last one everywhere)."""
    q, kc, vc, table, tab = attention_inputs(gen(90 + q_len + D), [q_len], [kv], H, Hk, D, page)
    bad = kv - q_len + q_len // 2
    vc[tab[0, bad // page], :, bad % page, 5] = float("nan")
    vc[tab[0, bad // page], :, bad % page, D - 3] = float("inf")
    kc[tab[0, (kv - 1) // page], :, (kv - 1) % page] = float("inf")
    got = f64(api.attn_paged(q, kc, vc, ints([0, q_len]), ints([kv]), table, q_len, kv, scale=scale))
    s = D ** -0.5 if scale is None else scale
    with np.errstate(all="ignore"):
        want, spread, absdot = np_layer.attn(f64(q), np_layer.gather_cache(f64(kc), tab[0], kv), np_layer.gather_cache(f64(vc), tab[0], kv), kv - q_len, s)
    before, n = kv - 1 - (kv - q_len), q_len // 2
    weight = BF16_HALF_ULP + 2 * (D + 4) * 2.0 ** -24 * absdot[:before, :, None] + 2.0 ** -14
    clean = np.ones(D, dtype=bool)
    clean[[5, D - 3]] = False
    tol = BF16_HALF_ULP * np.abs(want[:before]) + weight * spread[:before] + 1e-30
    assert_within(got[:n], want[:n], tol[:n])
    assert_within(got[n:before][:, :, clean], want[n:before][:, :, clean], tol[n:][:, :, clean])
    assert not np.isfinite(got[n:][:, :, ~clean]).any()
    if s != 0.0:
        assert not np.isfinite(got[before]).any()


def test_attn_paged_workspace_of_calls_of_every_size(api):
    """Calls with many and with few rows of the cache take turns on one workspace: the counters of one must not lie where
    another keeps its parts."""
    cases = [([1] * 5, [3000, 2500, 2900, 31, 2999], 32, 32), ([1], [20000], 1, 1), ([1] * 3, [2999] * 3, 64, 64), ([40, 1], [4000, 9], 2, 1)]
    size = max(api.attn_paged_workspace_size(sum(q), len(q), H, Hk, 64, max(q), max(kv)) for q, kv, H, Hk in cases)
    ws = api.new_workspace(size)
    made = [attention_inputs(gen(180 + i), *c, 64, 64, poison=False) for i, c in enumerate(cases)]

    def call(i, workspace):
        (q, kc, vc, table, _), (q_lens, kv_lens, _, _) = made[i], cases[i]
        return api.attn_paged(q, kc, vc, ints(starts(q_lens)), ints(kv_lens), table, max(q_lens), max(kv_lens), workspace=workspace)

    want = [call(i, None) for i in range(len(cases))]
    for i in (0, 1, 0, 3, 2, 1, 2, 0, 3, 0):
        out = call(i, ws)
        assert torch.equal(out, want[i]), i


def test_attn_paged_bounds_may_be_loose(api):
    q_lens, kv_lens = [1, 2, 1], [100, 300, 7]
    q, kc, vc, table, tab = attention_inputs(gen(81), q_lens, kv_lens, 4, 4, 128, 16)
    want = check_attention(api, q, kc, vc, table, tab, q_lens, kv_lens)
    for max_q, max_kv in ((2, 5000), (500, 300), (64, 100000)):
        got = api.attn_paged(q, kc, vc, ints(starts(q_lens)), ints(kv_lens), table, max_q, max_kv)
        np.testing.assert_allclose(f64(got), f64(want), atol=2.0 ** -5)


@pytest.mark.parametrize("n_new", [1, 40])
def test_attn_and_append_in_a_cache_beyond_32_bit_offsets(api, n_new):
    """Elements past 2^31 (4 GiB) of either cache."""
    H, Hk, D, page, kv = 4, 4, 128, 64, 200
    pages = (2 ** 31) // (Hk * page * D) + 40
    kc = torch.empty((pages, Hk, page, D), dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    g = gen(82)
    use = [pages - 1, pages - 9, 3, pages - 30]
    for p in use:
        kc[p] = draw(g, Hk, page, D)
        vc[p] = draw(g, Hk, page, D)
    table = ints([use])
    qkv = draw(g, n_new, (H + 2 * Hk) * D)
    q = api.rope_append(qkv, api.rope_table(kv, D), kc, vc, ints([0, n_new]), ints([kv]), table, H)
    small_k, small_v = kc[use].clone(), vc[use].clone()
    want_v = qkv.view(n_new, -1, D)[:, H + Hk:]
    for i in range(n_new):
        p = kv - n_new + i
        assert torch.equal(small_v[p // page, :, p % page], want_v[i])
    got = api.attn_paged(q, kc, vc, ints([0, n_new]), ints([kv]), table, n_new, kv)
    del kc, vc
    torch.cuda.empty_cache()
    tab = np.arange(4)[None, :]
    want = check_attention(api, q, small_k, small_v, ints(tab.tolist()), tab, [n_new], [kv])
    assert torch.equal(got, want)


# ------------------------------------------------------------------------------------------------------------------
# adapters of many requests
# ------------------------------------------------------------------------------------------------------------------
LORA_CASES = [  # (q_lens, adapters of the requests, n, K, N, r)
    ([1], [0], 1, 8, 8, 8),
    ([1] * 9, [0, 1, 2, -1, 2, 0, 1, 3, 99], 4, 4096, 1000, 16),
    ([3, 0, 17, 64, 65], [1, 0, -1, 0, 1], 2, 1000, 520, 32),
    ([130, 1, 40], [2, 0, 1], 3, 520, 264, 64),
    ([40, 33], [0, 1], 2, 264, 72, 24),
    ([280], [0], 1, 11008, 4096, 40),
    ([100, 28], [1, 0], 2, 4096, 24, 8),
    ([1] * 70, [i % 5 - 1 for i in range(70)], 4, 136, 40, 48),
    ([2] * 20, [i % 3 for i in range(20)], 3, 640, 256, 8),
    ([15, 17, 90], [0, 0, 1], 2, 2176, 328, 16),
]


@pytest.mark.parametrize("case", range(len(LORA_CASES)))
def test_lora_batch_add(api, case):
    q_lens, adapter, n, K, N, r = LORA_CASES[case]
    g = gen(200 + case)
    M, cu = sum(q_lens), starts(q_lens)
    x, y = draw(g, M, K), draw(g, M, N)
    a, b = draw(g, n, r, K, std=K ** -0.5), draw(g, n, N, r)
    scales = (torch.rand(n, generator=g) * 2 - 1).cuda()
    side, absside = np_layer.lora_batch(f64(x), f64(a), f64(b), cu, adapter, f64(scales))
    want = f64(y) + side
    # two fp32 inner products (K and 2 r terms), the first rounded to 16 significant bits (2^-16)
    tol = BF16_HALF_ULP * np.abs(want) + ((K + 2 * r + 8) * 2.0 ** -24 + 2.0 ** -16) * absside + 2.0 ** -22 * np.abs(f64(y))
    out = torch.full_like(y, float("nan"))
    got = api.lora_batch_add(x, a, b, y, ints(cu), ints(adapter), scales, out=out)
    assert got is out
    assert_within(f64(out), want, tol)
    for i, ad in enumerate(adapter):
        if not 0 <= ad < n:
            assert torch.equal(out[cu[i]:cu[i + 1]], y[cu[i]:cu[i + 1]])
    # in place, on column slices of wider tensors
    wide_x, wide_y = draw(g, M, K + 16), draw(g, M, N + 24)
    wide_x[:, 8:8 + K], wide_y[:, 16:16 + N] = x, y
    keep = wide_y.clone()
    api.lora_batch_add(wide_x[:, 8:8 + K], a, b, wide_y[:, 16:16 + N], ints(cu), ints(adapter), scales)
    assert torch.equal(wide_y[:, 16:16 + N], out)
    assert torch.equal(wide_y[:, :16], keep[:, :16]) and torch.equal(wide_y[:, 16 + N:], keep[:, 16 + N:])


def test_lora_batch_agrees_with_the_single_adapter_path(api):
    g = gen(300)
    M, K, N, r = 33, 1024, 512, 16
    x, y, a, b = draw(g, M, K), draw(g, M, N), draw(g, 1, r, K, std=0.03), draw(g, 1, N, r)
    one = api.lora_side_add(x, a[0], b[0], y.clone(), 0.5)
    many = api.lora_batch_add(x, a, b, y.clone(), ints([0, 10, M]), ints([0, 0]), torch.tensor([0.5], device="cuda"))
    np.testing.assert_allclose(f64(many), f64(one), rtol=2.0 ** -7, atol=2.0 ** -12)


def test_every_operator_runs_on_the_stream_it_is_given(api):
    """Inputs are produced, late, on a side stream; the results are read there."""
    g = gen(400)
    s = torch.cuda.Stream()
    x0, w = draw(g, 64, 512), draw(g, 512)
    want = api.rmsnorm(x0 * 2, w)
    kc, vc = api.new_kv_cache(8, 2, 16, 64)
    q0, table, cu, kv = draw(g, 40, 4, 64), ints([list(range(8))]), ints([0, 40]), ints([100])
    kc.copy_(draw(g, 8, 2, 16, 64))
    vc.copy_(draw(g, 8, 2, 16, 64))
    want_o = api.attn_paged(q0 * 2, kc, vc, cu, kv, table, 40, 100)
    a, b, scales = draw(g, 1, 8, 512), draw(g, 1, 64, 8), torch.ones(1, device="cuda")
    y0 = draw(g, 64, 64)
    want_l = api.lora_batch_add(x0 * 2, a, b, y0.clone(), ints([0, 64]), ints([0]), scales)
    cu64, zero = ints([0, 64]), ints([0])
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)
            x, q, y = x0 * 2, q0 * 2, y0.clone()
        got = api.rmsnorm(x, w, stream=s)
        got_o = api.attn_paged(q, kc, vc, cu, kv, table, 40, 100, stream=s)
        got_l = api.lora_batch_add(x, a, b, y, cu64, zero, scales, stream=s)
        s.synchronize()
        assert torch.equal(got, want) and torch.equal(got_o, want_o) and torch.equal(got_l, want_l)


# ------------------------------------------------------------------------------------------------------------------
# chains: the kernels come up early and wait for what is before them
# ------------------------------------------------------------------------------------------------------------------
class Chain:
    """Each call reads what the call before it wrote, in place where that is possible; shapes short enough that launches, not
    work, fill the time."""

    def __init__(self, api, q_lens, kv_lens, seed):
        g = gen(seed)
        self.api, self.H, self.Hk, self.D, hidden = api, 8, 4, 64, 512
        self.q_lens, self.T = q_lens, sum(q_lens)
        self.table, _, pages = paged(g, kv_lens, 16)
        self.kc, self.vc = draw(g, pages, self.Hk, 16, self.D), draw(g, pages, self.Hk, 16, self.D)
        self.cu, self.kv, self.kv_lens = ints(starts(q_lens)), ints(kv_lens), kv_lens
        self.h, self.residual, self.w = draw(g, self.T, hidden), draw(g, self.T, hidden), draw(g, hidden)
        wide = (self.H + 2 * self.Hk) * self.D
        self.a, self.b = draw(g, 2, 16, hidden, std=0.05), draw(g, 2, wide, 16, std=0.3)
        self.scales, self.adapter = torch.tensor([0.5, -1.0], device="cuda"), ints([i % 3 - 1 for i in range(len(q_lens))])
        self.cs = api.rope_table(max(kv_lens), self.D)
        self.ws = api.new_workspace(api.attn_paged_workspace_size(self.T, len(q_lens), self.H, self.Hk, self.D, max(q_lens), max(kv_lens)))
        self.lora_ws = api.new_workspace(api.lora_batch_workspace_size(self.T, len(q_lens), 16))
        self.qkv, self.x = torch.empty(self.T, wide, dtype=torch.bfloat16, device="cuda"), torch.empty_like(self.h)
        self.q, self.o = (torch.empty(self.T, self.H, self.D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.state = [self.h, self.residual, self.kc, self.vc]

    def step(self, after=lambda: None):
        api = self.api
        api.rmsnorm(self.h, self.w, residual=self.residual, out=self.x, residual_out=self.residual)
        after()
        self.qkv.zero_()
        after()
        api.lora_batch_add(self.x, self.a, self.b, self.qkv, self.cu, self.adapter, self.scales, workspace=self.lora_ws)
        after()
        api.rope_append(self.qkv, self.cs, self.kc, self.vc, self.cu, self.kv, self.table, self.H, out=self.q)
        after()
        api.attn_paged(self.q, self.kc, self.vc, self.cu, self.kv, self.table, max(self.q_lens), max(self.kv_lens), out=self.o, workspace=self.ws)
        after()
        api.rmsnorm(self.o.view(self.T, -1), self.w, residual=self.residual, out=self.h, residual_out=self.residual)
        after()


CHAINS = [([1] * 5, [30, 1, 200, 77, 650]), ([70, 1, 1, 130], [700, 33, 500, 130]), ([200], [2000])]


@pytest.mark.parametrize("case", range(len(CHAINS)))
def test_chains_of_calls_equal_calls_one_by_one(api, case):
    q_lens, kv_lens = CHAINS[case]
    one, many = Chain(api, q_lens, kv_lens, 500 + case), Chain(api, q_lens, kv_lens, 500 + case)
    for _ in range(20):
        one.step(after=torch.cuda.synchronize)
    torch.cuda.synchronize()
    for _ in range(20):
        many.step()
    torch.cuda.synchronize()
    for a, b in zip(one.state, many.state):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert torch.isfinite(many.h).all()


@pytest.mark.parametrize("case", range(len(CHAINS)))
def test_a_captured_chain_replays(api, case):
    q_lens, kv_lens = CHAINS[case]
    one, many = Chain(api, q_lens, kv_lens, 600 + case), Chain(api, q_lens, kv_lens, 600 + case)
    start = [t.clone() for t in many.state]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        many.step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        many.step()
        many.step()
    for t, v in zip(many.state, start):
        t.copy_(v)
    for _ in range(5):
        graph.replay()
    torch.cuda.synchronize()
    for _ in range(10):
        one.step()
    for a, b in zip(one.state, many.state):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_attn_paged_many_requests_of_every_kind(api):
    """More requests than a warp looks at in one go, those with many rows and those with none anywhere among them."""
    q_lens = [1] * 40 + [0] * 3 + [33, 1, 0, 5] + [1] * 30 + [130] + [2] * 5
    kv_lens = [1 + (37 * i) % 150 for i in range(len(q_lens))]
    kv_lens = [max(kv, q) for kv, q in zip(kv_lens, q_lens)]
    args = attention_inputs(gen(90), q_lens, kv_lens, 4, 2, 64, 16)
    check_attention(api, *args, q_lens, kv_lens)
