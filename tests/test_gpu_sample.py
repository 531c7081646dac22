"""The choice of the next token against the plain oracle: equal tokens, whatever the settings, sizes and values."""
import math

import numpy as np
import pytest
import torch

from oracle import np_sample

pytestmark = pytest.mark.gpu

OFF = dict(top_k=0, top_p=1.0, min_p=0.0)
SETTINGS = {
    "temperature": dict(temperature=0.7),
    "hot": dict(temperature=50.0),
    "cold": dict(temperature=0.01),
    "greedy": dict(temperature=0.0),
    "top_k": dict(temperature=1.0, top_k=40),
    "top_k_large": dict(temperature=1.5, top_k=3000),
    "top_k_one": dict(temperature=1.0, top_k=1),
    "top_k_beyond": dict(temperature=1.0, top_k=10 ** 9),
    "top_p": dict(temperature=1.0, top_p=0.9),
    "top_p_of_nearly_all": dict(temperature=3.0, top_p=0.9999),
    "top_p_small": dict(temperature=1.0, top_p=1e-4),
    "top_p_zero": dict(temperature=1.0, top_p=0.0),
    "min_p": dict(temperature=1.0, min_p=0.05),
    "min_p_one": dict(temperature=1.0, min_p=1.0),
    "all": dict(temperature=0.8, top_k=50, top_p=0.95, min_p=0.01),
    "all_large": dict(temperature=4.0, top_k=6000, top_p=0.9, min_p=0.001),
}


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available()
    from paper_2412_01034_b200 import api as a
    return a


def f32(v):
    return torch.tensor(v, dtype=torch.float32, device="cuda")


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def check(api, x, u, rows, **kw):
    """rows: the settings of every row, as dicts."""
    rows = [dict(OFF, **r) for r in rows]
    u = torch.tensor(u, dtype=torch.float32)
    got = api.sample(x, u.cuda(), f32([r["temperature"] for r in rows]), i32([min(r["top_k"], 2 ** 31 - 1) for r in rows]),
                     f32([r["top_p"] for r in rows]), f32([r["min_p"] for r in rows]), **kw)
    host, tokens = x.double().cpu().numpy(), got.cpu().tolist()
    single = lambda v: float(np.float32(v))  # noqa: E731 (what the kernel is given)
    for b, r in enumerate(rows):
        want, gap = np_sample.pick(host[b], float(u[b]), single(r["temperature"]), r["top_k"], single(r["top_p"]), single(r["min_p"]))
        # sums of up to 2^18 weights, each off by 2^-43 of the largest at most: within 2^-25 of the total of a border either side is right
        if gap > 2.0 ** -25:
            assert tokens[b] == want, (b, r, float(u[b]), tokens[b], want, gap)
    return got


def bell(g, B, V, std=2.0, ahead=6):
    x = torch.randn(B, V, generator=g) * std
    return x.scatter_add_(1, torch.randint(0, V, (B, ahead), generator=g), 4.0 + 5.0 * torch.rand(B, ahead, generator=g))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V", [1, 2, 31, 256, 1000, 4096, 4097, 9001, 32000, 128003])
def test_every_setting(api, V, dtype):
    g = torch.Generator().manual_seed(V)
    rows = list(SETTINGS.values())
    x = bell(g, len(rows), V).to(dtype).cuda()
    for _ in range(3):
        check(api, x, torch.rand(len(rows), generator=g).tolist(), rows)


@pytest.mark.parametrize("V", [5000, 262144])
def test_flat_rows(api, V):
    """All logits alike, or of few values: the order of the indices decides, and steps of the histogram hold thousands."""
    g = torch.Generator().manual_seed(1)
    rows = [dict(temperature=1.0), dict(temperature=1.0, top_k=2000), dict(temperature=1.0, top_p=0.5), dict(temperature=1.0, top_k=3000, top_p=0.6),
            dict(temperature=0.5, top_p=0.97, min_p=0.01), dict(temperature=1.0, top_k=4000, min_p=0.5)] * 2
    x = torch.full((len(rows), V), -3.5)
    x[6:] = torch.randint(0, 4, (6, V), generator=g).float()
    for u in (0.0, 0.25, 0.7371, 1 - 2.0 ** -24):
        check(api, x.cuda(), [u] * len(rows), rows)


def test_rows_that_are_nearly_empty(api):
    """Masks of -inf and of the type's lowest value, NaN, infinities, rows with nothing."""
    g = torch.Generator().manual_seed(2)
    V = 7000
    x = bell(g, 12, V)
    x[0] = -math.inf
    x[1] = math.nan
    x[2] = -math.inf
    x[2, 6543] = -1e30
    x[3, :-5] = torch.finfo(torch.float32).min
    x[4] = torch.finfo(torch.float32).min
    x[5, ::2] = math.nan
    x[6, [3, 77, 4200]] = math.inf
    x[7, 100] = 3e38
    x[7, 200] = -3e38
    x[8, 10:] = -math.inf
    x[9] *= 1e-38
    x[10] = -0.0
    x[10, 1::2] = 0.0
    x[11] *= 1e37
    for r in (dict(temperature=1.0), dict(temperature=1.0, top_k=5), dict(temperature=1.0, top_p=0.8), dict(temperature=0.0), dict(temperature=1e30, top_p=0.5),
              dict(temperature=1e-30, top_k=9), dict(temperature=math.inf, top_k=2000), dict(temperature=1.0, top_k=3000, top_p=0.9, min_p=0.1)):
        got = check(api, x.cuda(), torch.rand(12, generator=g).tolist(), [r] * 12).tolist()
        assert got[0] == got[1] == -1 and got[2] == 6543 and got[6] in (3, 77, 4200) and 0 <= got[8] < 10
    for r in (dict(temperature=math.nan), dict(temperature=-1.0), dict(temperature=1.0, min_p=1.5), dict(temperature=1.0, min_p=math.nan), dict(temperature=1.0, top_p=-0.5)):
        got = check(api, x[8:9].cuda(), [0.9], [dict(r, temperature=0.0)]).tolist()
        raw = dict(OFF, **r)
        one = api.sample(x[8:9].cuda(), f32([0.9]), f32([raw["temperature"]]), i32([raw["top_k"]]), f32([raw["top_p"]]), f32([raw["min_p"]]))
        assert one.tolist() == got
    # top_p that is no number is off; u outside [0, 1)
    a = api.sample(x[8:9].cuda(), f32([0.3]), f32([1.0]), None, f32([math.nan]), None)
    assert a.tolist() == api.sample(x[8:9].cuda(), f32([0.3]), f32([1.0])).tolist()
    ends = api.sample(x[8:9].cuda().expand(4, V), f32([-1.0, math.nan, 1.0, 5.0]), f32([1.0] * 4))
    assert ends.tolist() == [0, 0, 9, 9]


def test_steps_that_have_to_be_cut_again(api):
    """Values so close together, beside some far away, that one step of the histogram holds more than the list."""
    g = torch.Generator().manual_seed(3)
    V = 20000
    x = torch.rand(6, V, generator=g) * 1e-4
    x[:, 17] = 25.0
    x[:, 18] = 25.0 - 1e-5
    x[2:4] = (x[2:4] * 1e6).round() / 1e6
    x[4:, 1000:] = 3.0
    rows = [dict(temperature=1.0, top_k=9000), dict(temperature=20.0, top_p=0.7), dict(temperature=20.0, top_k=15000, top_p=0.3), dict(temperature=30.0, top_k=1500),
            dict(temperature=20.0, top_p=0.5), dict(temperature=20.0, top_k=12345, top_p=0.9)]
    for u in (0.11, 0.5, 0.93):
        check(api, x.cuda(), [u] * 6, rows)


def test_strides_alignment_and_slices(api):
    g = torch.Generator().manual_seed(4)
    for dtype in (torch.float32, torch.bfloat16):
        wide = bell(g, 9, 40013).to(dtype).cuda()
        for lo, hi in ((0, 40013), (1, 40000), (31744, 32000), (3, 4), (7, 9011)):
            x = wide[:, lo:hi]
            rows = [dict(temperature=0.9, top_k=30), dict(temperature=1.0, top_p=0.8), dict(temperature=0.0)] * 3
            u = torch.rand(9, generator=g).tolist()
            got = check(api, x, u, rows)
            assert torch.equal(got, check(api, x.contiguous(), u, rows))
            assert torch.equal(got[1:2], check(api, x[1:2], u[1:2], rows[1:2]))


def test_shares_of_tokens_follow_the_weights(api):
    """u on an even grid: every token comes as often as its share says, give or take one at either end of its range."""
    x = torch.tensor([1.0, -2.0, 3.0, 2.5, 0.0, 2.9, -8.0])
    B = 4000
    u = (torch.arange(B) + 0.5) / B
    for r in (dict(temperature=1.0), dict(temperature=2.0, top_k=4), dict(temperature=1.0, top_p=0.7), dict(temperature=1.0, min_p=0.5)):
        got = check(api, x.expand(B, 7).cuda(), u.tolist(), [r] * B).cpu().numpy()
        index, w = np_sample.distribution(x.double().numpy(), r["temperature"], r.get("top_k", 0), r.get("top_p", 1.0), r.get("min_p", 0.0))
        share = np.zeros(7)
        share[index] = w / w.sum()
        assert (np.abs(np.bincount(got, minlength=7) - share * B) <= 1).all()
        assert (np.diff(got) >= 0).all()


def test_rows_are_their_own_business(api):
    """A row's token is the same alone, in any batch, on any stream, and in a replayed graph; twice the same."""
    g = torch.Generator().manual_seed(5)
    rows = list(SETTINGS.values()) * 20
    B, V = len(rows), 9001
    x, u = bell(g, B, V).to(torch.bfloat16).cuda(), torch.rand(B, generator=g)
    want = check(api, x, u.tolist(), rows)
    args = [f32([dict(OFF, **r)[n] for r in rows]) for n in ("temperature", "top_p", "min_p")]
    k = i32([min(dict(OFF, **r)["top_k"], 2 ** 31 - 1) for r in rows])
    uc = u.cuda()
    for b in (0, 5, B - 1):
        assert torch.equal(api.sample(x[b:b + 1], uc[b:b + 1], args[0][b:b + 1], k[b:b + 1], args[1][b:b + 1], args[2][b:b + 1]), want[b:b + 1])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        late = x * 1
    got = api.sample(late, uc, args[0], k, args[1], args[2], stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    out = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert api.sample(x, uc, args[0], k, args[1], args[2], out=out) is out
    for _ in range(3):
        out.fill_(-9)
        graph.replay()
        assert torch.equal(out, want)
