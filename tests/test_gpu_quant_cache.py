"""GPU parity of the quantised paged cache: append, read-back and attention over the codes, against the plain oracle.

Codes, scales and zero points are defined to the bit; the read-back is one rounding of a product.  Tolerances of the attention
are those of the bf16 cache, with what is added stated at the check.
"""
import numpy as np
import pytest
import torch

from oracle import np_layer, np_quant_cache
from tests.test_gpu_layer_ops import BF16_HALF_ULP, LENGTHS, ROPE_CASES, assert_within, draw, f64, gen, ints, paged, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available()
    from paper_2412_01034_b200 import api as a
    return a


def parts_of(cache):
    """(codes as whole numbers, scale, zero) of either side, numpy."""
    out = []
    for codes, scales in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        s = scales.float().cpu().numpy()
        if cache.bits == 8:
            out.append((codes.cpu().numpy().astype(np.int64), s, np.zeros_like(s)))
        else:
            out.append((np_quant_cache.unpack(codes.cpu().numpy()), s[..., 0], s[..., 1]))
    return out


def random_cache(api, g, pages, Hk, page, D, bits, spread=1.0):
    """Every code, scales around spread, whole zero points; the codes of real heads would use their range in the same way."""
    cache = api.new_kv_cache_q(pages, Hk, page, D, bits)
    for codes, scales in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        raw = torch.randint(-2 ** 31, 2 ** 31, codes.shape if bits == 4 else codes.shape[:-1] + (D // 4,), generator=g, dtype=torch.int64)
        codes.copy_(raw.to(torch.int32).cuda() if bits == 4 else raw.to(torch.int32).cuda().view(torch.int8))
        s = (0.5 + torch.rand(scales.shape[:3], generator=g)) * spread / (60 if bits == 8 else 5)
        if bits == 8:
            scales.copy_(s)
        else:
            scales.copy_(torch.stack([s, torch.randint(5, 11, s.shape, generator=g).float()], dim=-1))
    return cache


# ------------------------------------------------------------------------------------------------------------------
# append
# ------------------------------------------------------------------------------------------------------------------
def check_append(api, g, qkv, q_lens, kv_lens, H, Hk, D, page, bits):
    table, tab, pages = paged(g, kv_lens, page)
    T, cu = sum(q_lens), starts(q_lens)
    cache = random_cache(api, g, pages, Hk, page, D, bits)
    want = [[x.copy() for x in side] for side in parts_of(cache)]
    cs = api.rope_table(max(kv_lens), D)
    q = api.rope_append_q(qkv, cs, cache, ints(cu), ints(kv_lens), table, H)
    x = qkv.float().cpu().numpy().reshape(T, H + 2 * Hk, D)
    angles = cs.cpu().numpy()
    with np.errstate(all="ignore"):
        for t, (b, p) in enumerate(zip(*np_layer.positions(cu, kv_lens))):
            if p < 0:
                assert not q[t].any()
                continue
            turned = np_quant_cache.rotate32(x[t, : H + Hk], angles[p, : D // 2], angles[p, D // 2:])
            np.testing.assert_array_equal(q[t].float().cpu().numpy(), np_quant_cache.bf16(turned[:H]))
            pg, slot = tab[b, p // page], p % page
            for side, heads in enumerate((turned[H:], x[t, H + Hk:])):
                for held, made in zip(want[side], np_quant_cache.quantise(heads, bits)):
                    held[pg, :, slot] = made
    for got, wanted in zip(parts_of(cache), want):
        for a, b in zip(got, wanted):
            np.testing.assert_array_equal(a, b)
    return cache


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("case", range(len(ROPE_CASES)))
def test_append(api, case, bits):
    q_lens, kv_lens, H, Hk, D, page = ROPE_CASES[case]
    g = gen(1100 + case)
    qkv = draw(g, sum(q_lens), (H + 2 * Hk) * D)
    check_append(api, g, qkv, q_lens, kv_lens, H, Hk, D, page, bits)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("D", [64, 128])
def test_append_of_heads_of_every_kind(api, D, bits):
    """Zeros, heads of one sign, one large value among small ones, the ends of the range, values that are not finite."""
    H, Hk = 2, 2
    g = gen(1120 + D)
    rows = 24
    x = draw(g, rows, H + 2 * Hk, D)
    x[0] = 0
    x[1] = x[1].abs()
    x[2] = -x[2].abs()
    x[3, :, 7] = 1000.0
    x[4, :, 5] = -1000.0
    x[5] *= 1e-37                       # scales near the smallest normal number, some above it, some below
    x[6] *= 2.0 ** -124
    x[7] *= 1e-39
    x[8, :, 3] = float("inf")
    x[9, :, D - 1] = float("-inf")
    x[10, :, 0] = float("nan")
    x[11, 2, 9] = float("nan")          # one key head alone
    x[12, 5, 9] = float("inf")          # one value head alone
    x[13] = 0.75
    x[14] = -0.75
    x[15] = torch.arange(D, device="cuda").float().sub(D / 2).to(torch.bfloat16)
    x[16] *= 1e36
    x[17, :, 0], x[17, :, 1] = 3e38, -3e38   # the 4-bit range is beyond fp32
    x[18] = 0
    x[18, :, 11] = 1.0
    x[19] = (x[19] * 4).round() / 8     # many values half way between two codes
    x[20] = torch.tensor([-127.5, 127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 126.5], device="cuda").to(torch.bfloat16).repeat(D // 8)
    check_append(api, g, x.view(rows, -1), [rows], [rows], H, Hk, D, 16, bits)


@pytest.mark.parametrize("bits", [8, 4])
def test_append_of_values_half_way_between_codes(api, bits):
    """Keys whose quotient by the scale is a half, or a few units in the last place beside one: the fp32 division decides.  (Cosines
    that are the keys themselves and sines of zero give any fp32 key.)"""
    rows, Hk, D, page = 400, 1, 128, 16
    rng = np.random.default_rng(7)
    top = 127 if bits == 8 else 15
    table = np.zeros((rows, D), dtype=np.float32)
    for t in range(rows):
        s = np.float32(np_quant_cache.bf16(np.float32([2.0 ** rng.uniform(-20, 20)]))[0])
        k = rng.integers(0, top, D // 2)
        v = ((k + 0.5) * np.float64(s)).astype(np.float32)
        v = (v.view(np.int32) + rng.integers(-3, 4, D // 2).astype(np.int32)).view(np.float32)
        v[0] = np.float32(top) * s   # (the scale is s)
        table[t, : D // 2] = v
    cs = torch.from_numpy(table).cuda()
    qkv = torch.ones(rows, 3 * D, dtype=torch.bfloat16, device="cuda")
    cache = api.new_kv_cache_q(rows // page, Hk, page, D, bits)
    pages = ints([list(range(rows // page))])
    api.rope_append_q(qkv, cs, cache, ints([0, rows]), ints([rows]), pages, 1)
    keys = np.concatenate([table[:, : D // 2], table[:, : D // 2]], axis=1)[:, None]
    got = parts_of(cache)[0]
    for held, made in zip(got, np_quant_cache.quantise(keys, bits)):
        np.testing.assert_array_equal(held.transpose(0, 2, 1, *range(3, held.ndim)).reshape(made.shape), made)


@pytest.mark.parametrize("bits", [8, 4])
def test_append_skips_what_has_no_place(api, bits):
    g = gen(1130)
    H, Hk, D, page, pages = 2, 1, 64, 16, 4
    qkv = draw(g, 6, (H + 2 * Hk) * D)
    cache = api.new_kv_cache_q(pages, Hk, page, D, bits)
    table = ints([[0, 99], [-1, 1], [2, 3]])
    q = api.rope_append_q(qkv, api.rope_table(33, D), cache, ints([0, 2, 4, 6]), ints([18, 18, 34]), table, H)
    for codes, scales in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        assert codes[1, 0, :2].any() and not codes[1, 0, 2:].any() and not codes[[0, 2, 3]].any()
        assert scales[1, 0, :2].any() and not scales[1, 0, 2:].any() and not scales[[0, 2, 3]].any()
    assert q[:5].any(dim=2).all() and not q[5].any()


# ------------------------------------------------------------------------------------------------------------------
# read-back
# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("Hk,D,page", [(1, 64, 16), (4, 128, 64), (32, 128, 16), (7, 64, 128), (3, 128, 32)])
def test_read_back(api, Hk, D, page, bits):
    """Whole contexts, the last tokens of one, none of one, more rows than tokens; rows behind the last request."""
    rows, kv_lens = [40, 5, 0, 1, 20], [40, 129, 7, 1, 18]
    g = gen(1140 + Hk)
    table, tab, pages = paged(g, kv_lens, page)
    cache = random_cache(api, g, pages, Hk, page, D, bits)
    cache.k_scale[tab[0, 0], 0, 3] = float("nan")
    out = [torch.full((sum(rows) + 3, Hk, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    k, v = api.kv_read_q(cache, ints(starts(rows)), ints(kv_lens), table, sum(rows) + 3, out=out)
    assert k is out[0] and v is out[1]
    for got, (codes, s, z) in zip((k, v), parts_of(cache)):
        # (fewer than 17 significant bits times 8: exact in fp32, then one rounding)
        held = np_quant_cache.bf16(np_quant_cache.values(codes, s, z, bits).astype(np.float32))
        got = got.float().cpu().numpy()
        for t, (b, p) in enumerate(zip(*np_layer.positions(starts(rows), kv_lens))):
            want = held[tab[b, p // page], :, p % page] if p >= 0 else np.zeros((Hk, D))
            np.testing.assert_array_equal(got[t], want)
        assert (got[sum(rows):] == 7.0).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_read_back_of_an_append(api, bits):
    """What is read back is within half a step of what was appended (and the clamp's: the scale is rounded to 8 bits)."""
    g = gen(1150)
    H, Hk, D, page, kv = 4, 2, 128, 32, 100
    qkv = draw(g, kv, (H + 2 * Hk) * D)
    cache = api.new_kv_cache_q(8, Hk, page, D, bits)
    table = ints([[5, 0, 7, 2]])
    cs = api.rope_table(kv, D)
    api.rope_append_q(qkv, cs, cache, ints([0, kv]), ints([kv]), table, H)
    k, v = api.kv_read_q(cache, ints([0, kv]), ints([kv]), table, kv)
    x = f64(qkv).reshape(kv, H + 2 * Hk, D)
    turned = np.stack([np_layer.rope_rotate(x[t, H:H + Hk], t, 10000.0) for t in range(kv)])
    for got, want in ((k, turned), (v, x[:, H + Hk:])):
        a = np.abs(want).max(axis=-1, keepdims=True)
        span = np.maximum(want.max(axis=-1, keepdims=True), 0) - np.minimum(want.min(axis=-1, keepdims=True), 0)
        # the step; half of it, or where a rounded-down scale (2^-8) cuts the end off what is beyond the last code; with 4 bits
        # the zero point is rounded as well, so that either end may be half a step beyond; the value's own rounding
        step = (a / 127 if bits == 8 else span / 15) * (1 + BF16_HALF_ULP)
        beyond = 127 * BF16_HALF_ULP if bits == 8 else 0.5 + 15 * BF16_HALF_ULP
        assert_within(f64(got), want, step * max(0.5, beyond + 0.5) + BF16_HALF_ULP * (np.abs(want) + step) + 2.0 ** -20 * a)


# ------------------------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------------------------
def quant_attention_inputs(api, g, q_lens, kv_lens, H, Hk, D, page, bits, q_std=1.0, poison=True):
    table, tab, pages = paged(g, kv_lens, page)
    q = draw(g, sum(q_lens), H, D, std=q_std)
    cache = random_cache(api, g, pages, Hk, page, D, bits)
    if poison:   # the scales of everything that belongs to no cached token are NaN or infinite
        live = np.zeros((pages, page), dtype=bool)
        for b, n in enumerate(kv_lens):
            for j in range(n):
                live[tab[b, j // page], j % page] = True
        dead = torch.from_numpy(~live).cuda()[:, None, :]
        for s, bad in ((cache.k_scale, float("inf")), (cache.v_scale, float("nan"))):
            s.masked_fill_(dead if bits == 8 else dead[..., None], bad)
    return q, cache, table, tab


def check_quant_attention(api, q, cache, table, tab, q_lens, kv_lens, scale=None, bounds=None, **kw):
    cu, D, bits = starts(q_lens), q.shape[2], cache.bits
    G = q.shape[1] // cache.k.shape[1]
    bounds = bounds or (max(max(q_lens), 1), max(max(kv_lens), 1))
    got = api.attn_paged_q(q, cache, ints(cu), ints(kv_lens), table, *bounds, scale=scale, **kw)
    scale = D ** -0.5 if scale is None else scale
    qd, gd = f64(q), f64(got)
    sides = [(np_quant_cache.values(*p, bits), p[1].astype(np.float64)) for p in parts_of(cache)]
    for b, (n, kv) in enumerate(zip(q_lens, kv_lens)):
        if n == 0:
            continue
        lo = cu[b]
        k, v = (np_layer.gather_cache(side[0], tab[b], kv) for side in sides)
        if n * G > 16 and kv > 0:   # (values and weights have fp16's 11 bits; the largest value is near the end of its range)
            k, v = (np.ldexp(np.ldexp(x, -e).astype(np.float16).astype(np.float64), e)
                    for x, e in ((x, int(np.floor(np.log2(np.abs(x).max()))) - 14) for x in (k, v)))
        want, spread, absdot = np_layer.attn(qd[lo:lo + n], k, v, kv - n, scale)
        # as for the bf16 cache: fp32 sums of D products, once in the numerator and once in the sum; a weight times its value's
        # scale rounded to bf16 (a weight alone to fp16); exp2 and the sums in fp32
        weight = (BF16_HALF_ULP if n * G <= 16 else 2.0 ** -11) + 2 * (D + 8) * 2.0 ** -24 * absdot[:, :, None] + 2.0 ** -14
        tol = BF16_HALF_ULP * np.abs(want) + weight * spread + 1e-30
        if n * G <= 16 and kv > 0:
            # a query row in steps of 1 / 32512 of its largest element is off by half of one, 2^-16 of that element to within
            # 2^-6 of it, at each d: a score by 2^-16 max |q| sum |k_d| |scale|, in the numerator and in the sum
            sizes = np.repeat(np.abs(k).sum(axis=2).max(axis=0), G)[None] * np.abs(qd[lo:lo + n]).max(axis=2) * abs(scale)
            tol += 2 * (1 + 2.0 ** -6) * 2.0 ** -16 * sizes[:, :, None] * spread
        if n * G > 16 and kv > 0:   # a weight below 2^-14 of the reference is off by 2^-25 of it, whatever its size
            tol += 2.0 ** -25 * np.repeat(np.abs(v).sum(axis=0), G, axis=0)[None]
        assert_within(gd[lo:lo + n], want, tol)
    return got


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("H,Hk,D,page", [(4, 4, 128, 16), (8, 2, 128, 64), (7, 1, 64, 32), (6, 2, 64, 128), (12, 3, 128, 128)])
def test_attention(api, lengths, H, Hk, D, page, bits):
    q_lens, kv_lens = LENGTHS[lengths]
    args = quant_attention_inputs(api, gen(1200 + H * 10 + D + page), q_lens, kv_lens, H, Hk, D, page, bits)
    check_quant_attention(api, *args, q_lens, kv_lens)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("H,Hk", [(32, 1), (40, 2), (17, 1), (16, 1), (9, 1)])
def test_attention_wide_groups(api, H, Hk, bits):
    q_lens, kv_lens = [1, 9, 1], [300, 77, 5]
    args = quant_attention_inputs(api, gen(1210 + H), q_lens, kv_lens, H, Hk, 64, 16, bits)
    check_quant_attention(api, *args, q_lens, kv_lens)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("B,kv,D", [(55, 257, 64), (37, 385, 128), (28, 513, 64), (22, 700, 64), (18, 769, 128), (15, 1000, 64), (150, 300, 64)])
def test_attention_blocks_of_a_request(api, B, kv, D, bits):
    """One to eight blocks to a request and key head, of which shorter requests have no work for some."""
    q_lens, kv_lens = [1 + (b % 3 == 1) for b in range(B)], [kv] + [2 + (b * 131) % (kv - 1) for b in range(B - 1)]
    args = quant_attention_inputs(api, gen(1215 + B), q_lens, kv_lens, 6, 3, D, 32, bits)
    check_quant_attention(api, *args, q_lens, kv_lens)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("D", [128, 64])
def test_attention_single_tokens_beside_a_prompt(api, D, bits):
    """Requests of 4, 8, 12 and 16 rows in blocks of their own beside one of 80; the workspace twice."""
    q_lens, kv_lens = [1, 20, 2, 1, 3, 0, 4, 1], [2300, 2500, 1025, 1024, 1500, 9, 2049, 1]
    q, cache, table, tab = quant_attention_inputs(api, gen(1216 + D), q_lens, kv_lens, 8, 2, D, 64, bits)
    ws = api.new_workspace(api.attn_paged_q_workspace_size(sum(q_lens), len(q_lens), 8, 2, D, bits, max(q_lens), max(kv_lens)))
    first = check_quant_attention(api, q, cache, table, tab, q_lens, kv_lens, workspace=ws)
    second = check_quant_attention(api, q, cache, table, tab, q_lens, kv_lens, workspace=ws)
    assert torch.equal(first, second)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("q_std,scale", [(30.0, None), (1.0, 0.0), (1.0, -0.5), (0.01, 1.0)])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [700, 65]), ([200], [500])])
def test_attention_scores_of_every_size(api, q_std, scale, q_lens, kv_lens, bits):
    args = quant_attention_inputs(api, gen(1220), q_lens, kv_lens, 4, 2, 128, 32, bits, q_std=q_std)
    check_quant_attention(api, *args, q_lens, kv_lens, scale=scale)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("q_lens", [[1], [12], [130]])
def test_attention_growing_scores(api, q_lens, bits):
    """Scores that grow along the cache: the running reference changes all the time."""
    kv = 1500
    q, cache, table, tab = quant_attention_inputs(api, gen(1230), q_lens, [kv], 1, 1, 128, 16, bits)
    ramp = torch.linspace(0.01, 20.0, kv).to(torch.bfloat16)
    cache.k.zero_()
    for j in range(kv):
        at = (int(tab[0, j // 16]), slice(None), j % 16)
        if bits == 8:
            cache.k[at + (0,)] = 1
            cache.k_scale[at] = ramp[j]
        else:
            cache.k[at + (0,)] = 2
            cache.k_scale[at + (0,)] = ramp[j] / 2
            cache.k_scale[at + (1,)] = 0
    q[:, :, 0] = 10.0
    check_quant_attention(api, q, cache, table, tab, q_lens, [kv], scale=1.0)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("q_lens,kv_lens", [([1], [20011]), ([1, 1], [9000, 3]), ([130], [6100]), ([20, 20], [5000, 2600]), ([9], [4100])])
def test_attention_long_caches_are_split(api, q_lens, kv_lens, bits):
    args = quant_attention_inputs(api, gen(1240), q_lens, kv_lens, 2, 1, 128, 64, bits, poison=False)
    check_quant_attention(api, *args, q_lens, kv_lens)


@pytest.mark.parametrize("bits", [8, 4])
def test_attention_scales_of_very_different_size(api, bits):
    """Heads whose scales differ by factors of a million, among them heads of zeros."""
    q_lens, kv_lens = [1, 40], [400, 300]
    q, cache, table, tab = quant_attention_inputs(api, gen(1250), q_lens, kv_lens, 2, 1, 128, 16, bits)
    g = gen(1251)
    for s in (cache.v_scale,):
        of = s if bits == 8 else s[..., 0]
        of.mul_((10.0 ** (6 * torch.rand(of.shape, generator=g) - 3)).cuda().to(torch.bfloat16))
    zero = tab[0, 3]
    if bits == 8:
        cache.k[zero], cache.v[zero], cache.k_scale[zero], cache.v_scale[zero] = 0, 0, 1, 1
    check_quant_attention(api, q, cache, table, tab, q_lens, kv_lens)


@pytest.mark.parametrize("bits", [8, 4])
def test_attention_is_deterministic_and_its_workspace_is_reusable(api, bits):
    cases = [([1] * 6, [900, 33, 2000, 1, 64, 700], 8, 8), ([70, 1], [3000, 20], 8, 2), ([1], [5000], 2, 1), ([300], [300], 4, 4), ([1] * 5, [3000] * 5, 32, 32)]
    size = max(max(api.attn_paged_q_workspace_size(sum(q), len(q), H, Hk, 128, bits, max(q), max(kv)),
                   api.attn_paged_workspace_size(sum(q), len(q), H, Hk, 128, max(q), max(kv))) for q, kv, H, Hk in cases)
    ws = api.new_workspace(size)
    made = [quant_attention_inputs(api, gen(1260 + i), q, kv, H, Hk, 128, 16, bits) for i, (q, kv, H, Hk) in enumerate(cases)]
    first = [check_quant_attention(api, *made[i], cases[i][0], cases[i][1]) for i in range(len(cases))]
    for i in (0, 4, 1, 0, 2, 3, 4, 2, 0):
        (q, cache, table, _), (q_lens, kv_lens, H, Hk) = made[i], cases[i]
        args = (ints(starts(q_lens)), ints(kv_lens), table, max(q_lens), max(kv_lens))
        # (the bf16 cache's attention takes turns on the workspace)
        bf = torch.zeros(cache.k.shape[:3] + (128,), dtype=torch.bfloat16, device="cuda")
        api.attn_paged(q, bf, bf, *args, workspace=ws)
        assert torch.equal(api.attn_paged_q(q, cache, *args, workspace=ws), first[i]), i
    assert int(ws[:4].view(torch.int32)[0]) == 0


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("q_len,kv,H,Hk,D,page", [(6, 300, 4, 2, 128, 16), (16, 16, 3, 3, 64, 32), (5, 4100, 3, 1, 128, 64), (300, 500, 2, 2, 128, 16),
                                                  (280, 280, 4, 1, 64, 64), (130, 6100, 2, 1, 128, 64)])
def test_heads_that_are_no_numbers_stay_out_of_earlier_tokens(api, q_len, kv, H, Hk, D, page, bits):
    """A new token's value head is NaN, the last one's key head as well: the tokens before them are as if they were not there, the
    others are NaN."""
    q, cache, table, tab = quant_attention_inputs(api, gen(1270 + q_len + D), [q_len], [kv], H, Hk, D, page, bits)
    clean = check_quant_attention(api, q, cache, table, tab, [q_len], [kv])
    bad = kv - q_len + q_len // 2
    cache.v_scale[tab[0, bad // page], :, bad % page] = float("nan")
    cache.k_scale[tab[0, (kv - 1) // page], :, (kv - 1) % page] = float("nan")
    got = api.attn_paged_q(q, cache, ints([0, q_len]), ints([kv]), table, q_len, kv)
    n = q_len // 2
    assert torch.equal(got[:n], clean[:n])
    assert got[n:].isnan().all()


@pytest.mark.parametrize("bits", [8, 4])
def test_attention_bounds_may_be_loose(api, bits):
    q_lens, kv_lens = [1, 2, 1], [100, 300, 7]
    args = quant_attention_inputs(api, gen(1280), q_lens, kv_lens, 4, 4, 128, 16, bits)
    for bounds in ((2, 300), (2, 5000), (500, 300), (64, 100000)):
        check_quant_attention(api, *args, q_lens, kv_lens, bounds=bounds)


@pytest.mark.parametrize("bits", [8, 4])
def test_requests_beyond_the_bounds_leave_the_others_alone(api, bits):
    q_lens, kv_lens = [1, 12, 1, 40], [700, 300, 900, 60]
    q, cache, table, tab = quant_attention_inputs(api, gen(1285), q_lens, kv_lens, 4, 4, 128, 16, bits)
    want = check_quant_attention(api, q, cache, table, tab, q_lens, kv_lens)
    got = api.attn_paged_q(q, cache, ints(starts(q_lens)), ints(kv_lens), table, 1, 900)
    for at in (0, 13):
        np.testing.assert_allclose(f64(got[at]), f64(want[at]), atol=2.0 ** -5)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("n_new", [1, 40])
def test_append_read_and_attention_beyond_32_bit_offsets(api, n_new, bits):
    """Bytes past 2^32 of either side's codes."""
    H, Hk, D, page, kv = 4, 4, 128, 64, 200
    pages = (2 ** 32) // (Hk * page * D * bits // 8) + 40
    cache = api.new_kv_cache_q(pages, Hk, page, D, bits)
    g = gen(1290)
    use = [pages - 1, pages - 9, 3, pages - 30]
    some = random_cache(api, g, 4, Hk, page, D, bits)
    for big, small in zip(cache, some):
        big[use] = small
    table, cu, lens = ints([use]), ints([0, n_new]), ints([kv])
    qkv = draw(g, n_new, (H + 2 * Hk) * D)
    cs = api.rope_table(kv, D)
    q = api.rope_append_q(qkv, cs, cache, cu, lens, table, H)
    read = api.kv_read_q(cache, ints([0, kv]), lens, table, kv)
    got = api.attn_paged_q(q, cache, cu, lens, table, n_new, kv)
    del cache, big
    torch.cuda.empty_cache()
    near = ints([[0, 1, 2, 3]])
    assert torch.equal(q, api.rope_append_q(qkv, cs, some, cu, lens, near, H))
    for a, b in zip(read, api.kv_read_q(some, ints([0, kv]), lens, near, kv)):
        assert torch.equal(a, b)
    assert torch.equal(got, check_quant_attention(api, q, some, near, np.arange(4)[None, :], [n_new], [kv]))


@pytest.mark.parametrize("bits", [8, 4])
def test_many_requests_of_every_kind(api, bits):
    q_lens = [1] * 40 + [0] * 3 + [33, 1, 0, 5] + [1] * 30 + [130] + [2] * 5
    kv_lens = [max(1 + (37 * i) % 150, q) for i, q in enumerate(q_lens)]
    args = quant_attention_inputs(api, gen(1300), q_lens, kv_lens, 4, 2, 64, 16, bits)
    check_quant_attention(api, *args, q_lens, kv_lens)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("q_lens,kv_lens", [([1] * 5, [30, 1, 200, 77, 650]), ([70, 1, 1, 130], [700, 33, 500, 130])])
def test_chains_streams_and_graphs_give_the_same(api, q_lens, kv_lens, bits):
    """Append, read-back and attention in a chain: one by one, on a side stream, and captured and replayed."""
    H, Hk, D, page = 8, 4, 64, 16
    g = gen(1310)
    table, _, pages = paged(g, kv_lens, page)
    T, cu, lens = sum(q_lens), ints(starts(q_lens)), ints(kv_lens)
    start = random_cache(api, g, pages, Hk, page, D, bits)
    qkv, cs = draw(g, T, (H + 2 * Hk) * D), api.rope_table(max(kv_lens), D)
    ws = api.new_workspace(api.attn_paged_q_workspace_size(T, len(q_lens), H, Hk, D, bits, max(q_lens), max(kv_lens)))

    def step(cache, x, after=lambda: None):
        outs = []
        for _ in range(3):
            q = api.rope_append_q(x, cs, cache, cu, lens, table, H)
            after()
            k, v = api.kv_read_q(cache, cu, lens, table, T)
            after()
            o = api.attn_paged_q(q, cache, cu, lens, table, max(q_lens), max(kv_lens), workspace=ws)
            after()
            outs += [q, k, v, o]
            x = torch.cat([o, k, v], dim=1).view(T, -1)
            after()
        return outs

    want = step(type(start)(*[t.clone() for t in start]), qkv, torch.cuda.synchronize)
    assert all(torch.isfinite(t).all() for t in want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step(type(start)(*[t.clone() for t in start]), qkv)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    cache = type(start)(*[t.clone() for t in start])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(cache, qkv)
    for _ in range(3):
        for t, v in zip(cache, start):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
