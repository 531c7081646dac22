"""The workspaces of a decoder layer over its lifetime: captured steps, growing batches."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, DIM, FFN, PAGE, WIDTH = 512, 8, 64, 768, 16, 72


def make(adapters=True, max_tokens=256):
    from paper_2412_01034_b200.decoder_layer import DecoderLayer
    g = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda std, *s: torch.randn(s, generator=g, device="cuda") * std  # noqa: E731
    w = {"norm1": 1 + normal(0.1, HIDDEN), "norm2": 1 + normal(0.1, HIDDEN), "qkv": normal(0.04, 3 * HEADS * DIM, HIDDEN),
         "o": normal(0.04, HIDDEN, HEADS * DIM), "gate": normal(0.04, FFN, HIDDEN), "up": normal(0.04, FFN, HIDDEN), "down": normal(0.04, HIDDEN, FFN)}
    ad = (normal(HIDDEN ** -0.5, 3, 8, HIDDEN).bfloat16(), normal(0.3, 3, 3 * HEADS * DIM, 8).bfloat16(), torch.tensor([0.5, 1.0, -0.7], device="cuda"))
    layer = DecoderLayer(w, HEADS, HEADS, DIM, num_pages=40 * WIDTH, page_size=PAGE, max_pos=1152, max_tokens=max_tokens, adapters=ad if adapters else None)
    for c in (layer.k_cache, layer.v_cache):
        c.normal_(generator=g)
    return layer, normal


def batch(normal, q_lens, kv_lens):
    """Requests on pages of their own (request b on pages b WIDTH ...) and their rows."""
    from paper_2412_01034_b200.decoder_layer import Requests
    tables = [list(range(b * WIDTH, (b + 1) * WIDTH)) for b in range(len(q_lens))]
    return Requests.of(q_lens, kv_lens, tables, [b % 4 - 1 for b in range(len(q_lens))]), normal(1.0, sum(q_lens), HIDDEN).bfloat16()


def capture(layer, x, b):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.forward(x, None, b)
    return graph, out


def both(pair):
    return torch.cat([t.clone() for t in pair])


def test_a_captured_step_outlives_larger_batches():
    """A step is captured, larger batches run, other tensors take whatever memory is free: the replay is what it was, and
    writes nowhere else."""
    layer, normal = make()
    small, x = batch(normal, [1] * 20, [900 - b for b in range(20)])    # (20 x 8 rows of the cache in two parts each)
    want = both(layer.forward(x, None, small))
    caches = layer.k_cache.clone(), layer.v_cache.clone()
    graph, out = capture(layer, x, small)
    graph.replay()
    assert torch.equal(both(out), want)
    for n, kv in ((30, 1000), (40, 1150), (1, 700), (40, 1150)):
        other, xo = batch(normal, [1] * n, [kv] * n)
        layer.forward(xo, None, other)
        other, xo = batch(normal, [3 * n], [kv])
        layer.forward(xo, None, other)
    layer.k_cache.copy_(caches[0])   # (the larger batches append to the same requests)
    layer.v_cache.copy_(caches[1])
    torch.cuda.synchronize()
    held = [torch.full((1 << k,), 0xFF, dtype=torch.uint8, device="cuda") for k in (10, 16, 18, 20, 20, 21, 21, 22, 22, 23, 23, 24) for _ in range(4)]
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(both(out), want) and all(bool(t.eq(0xFF).all()) for t in held)


def test_a_step_captured_before_its_workspace_was_made():
    """The first batch of its kind runs in a capture, and outside before the graph has ever run."""
    layer, normal = make()
    b, x = batch(normal, [1] * 40, [1100 - 3 * i for i in range(40)])
    ready, xr = batch(normal, [2], [5])
    layer.forward(xr, None, ready)          # (kernels are loaded; this needs hardly any workspace)
    graph, out = capture(layer, x, b)
    want = both(layer.forward(x, None, b))
    graph.replay()
    assert torch.equal(both(out), want) and torch.equal(both(layer.forward(x, None, b)), want)
    fresh, _ = make()
    fresh.k_cache.copy_(layer.k_cache)
    fresh.v_cache.copy_(layer.v_cache)
    assert torch.equal(both(fresh.forward(x, None, b)), want)


def test_reserved_batches_allocate_no_workspace():
    layer, normal = make()
    b, x = batch(normal, [1] * 40, [1100] * 40)
    layer.reserve(40, 40, 1, 1100)
    before = [t.data_ptr() for t in layer._attn_workspaces]
    layer.forward(x, None, b)
    assert before and [t.data_ptr() for t in layer._attn_workspaces] == before


@pytest.mark.parametrize("n", [1, 16, 17, 100, 255, 256, 300])
def test_adapters_of_every_row_count_have_room(n):
    """One request with all rows, and the same rows as many requests (300: more than max_tokens)."""
    layer, normal = make()
    one, x = batch(normal, [n], [n])
    h, r = layer.forward(x, None, one)
    assert torch.isfinite(h).all()
    many, x = batch(normal, [n // 5] * 4 + [n - n // 5 * 4], [max(n, 1)] * 5)
    h, r = layer.forward(x, None, many)
    assert torch.isfinite(h).all()


def test_recorded_failures_are_seen():
    """A status word that a kernel has set (here: the test) is raised, by the function and by the layer."""
    from paper_2412_01034_b200 import api
    ws = api.new_workspace(1 << 10)
    api.check_workspace(ws)
    ws[:4].view(torch.int32).fill_(api.ERR_TIMEOUT)
    with pytest.raises(api.QilError, match="timed out"):
        api.check_workspace(ws)
    layer, normal = make()
    b, x = batch(normal, [60, 1], [900, 30])
    layer.forward(x, None, b)
    layer.check()
    for held in (layer.workspace, layer._attn_workspaces[0]):
        held[:4].view(torch.int32).fill_(api.ERR_TIMEOUT)
        with pytest.raises(api.QilError, match="timed out"):
            layer.check()
        held[:4].zero_()
        layer.check()


def test_more_rows_than_the_layer_was_made_for():
    """A layer for one row takes batches of 2 to 40: as a layer with room for them, up to the order of the GEMMs' sums."""
    small, normal = make(max_tokens=1)
    large, _ = make(max_tokens=256)
    for n in (2, 7, 8, 9, 40):
        b, x = batch(normal, [n], [n])
        got, want = both(small.forward(x, None, b)), both(large.forward(x, None, b))
        assert float((got.float() - want.float()).abs().max()) <= 2.0 ** -5 * float(want.float().abs().max()), n
    small.check()
