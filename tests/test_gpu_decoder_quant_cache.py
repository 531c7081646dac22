"""Decoder layers over a quantised cache, and the token head: append, attention, read-back and the choice of tokens together,
as a server runs them."""
import numpy as np
import pytest
import torch

from oracle import np_layer, np_sample
from tests.test_gpu_decoder_layer import DIM, FFN, HEADS, HIDDEN, KV_HEADS, PAGE, dequantised

pytestmark = pytest.mark.gpu

VOCAB = 600


def make(kv_bits, layers=2, seed=0):
    from paper_2412_01034_b200.decoder_layer import DecoderLayer, TokenHead
    g = torch.Generator().manual_seed(seed)
    normal = lambda std, *s: (torch.randn(s, generator=g) * std).cuda()  # noqa: E731
    made = []
    for _ in range(layers):
        w = {"norm1": 1 + normal(0.1, HIDDEN), "norm2": 1 + normal(0.1, HIDDEN), "qkv": normal(0.04, (HEADS + 2 * KV_HEADS) * DIM, HIDDEN),
             "o": normal(0.04, HIDDEN, HEADS * DIM), "gate": normal(0.04, FFN, HIDDEN), "up": normal(0.04, FFN, HIDDEN), "down": normal(0.04, HIDDEN, FFN)}
        made.append(DecoderLayer(w, HEADS, KV_HEADS, DIM, num_pages=64, page_size=PAGE, max_pos=400, max_tokens=256, kv_bits=kv_bits))
    head = TokenHead(1 + normal(0.1, HIDDEN), normal(0.08, VOCAB, HIDDEN), max_requests=8)
    return made, head, normal(1.0, VOCAB, HIDDEN).bfloat16()


def reference(layers, held, x):
    """One request from its first token on, x [n][HIDDEN] float64, with the keys and values that the layers' caches hold; the
    worst distance of a held head from what it was made of, over its step (or, where it is more, its bf16 inputs' error)."""
    n, worst = len(x), 0.0
    for layer, (k, v) in zip(layers, held):
        y, _ = np_layer.rmsnorm(x, layer.norm1.double().cpu().numpy(), layer.eps)
        t = (y @ dequantised(layer.qkv).T).reshape(n, -1, DIM)
        turned = np.stack([np_layer.rope_rotate(t[i, : HEADS + KV_HEADS], i, 10000.0) for i in range(n)])
        for got, made in ((k, turned[:, HEADS:]), (v, t[:, HEADS + KV_HEADS:])):
            span = np.maximum(made.max(axis=2), 0) - np.minimum(made.min(axis=2), 0) if layer.kv_bits == 4 else np.abs(made).max(axis=2)
            step = span / (15 if layer.kv_bits == 4 else 127)
            # (what goes in is off by 2^-5 of the row's largest value at most, as the outputs of a layer)
            worst = max(worst, float((np.abs(got - made).max(axis=2) / (step + 2.0 ** -5 * np.abs(made).max(axis=2))).max()))
        att, _, _ = np_layer.attn(turned[:, :HEADS], k, v, 0, DIM ** -0.5)
        x = x + att.reshape(n, -1) @ dequantised(layer.o).T
        y, _ = np_layer.rmsnorm(x, layer.norm2.double().cpu().numpy(), layer.eps)
        gu = y @ dequantised(layer.gate_up).T
        x = x + (gu[:, 0::2] / (1 + np.exp(-gu[:, 0::2])) * gu[:, 1::2]) @ dequantised(layer.down).T
    return x, worst


@pytest.mark.parametrize("kv_bits", [8, 4])
def test_layers_serve_requests_step_by_step(kv_bits):
    """A prompt at once, a prompt in two chunks next to single tokens, one that joins later; then the tokens of the last step.
    The tolerance is that of the layers over a bf16 cache: the reference reads the same keys and values."""
    from paper_2412_01034_b200.decoder_layer import Requests
    layers, head, _ = make(kv_bits)
    g = torch.Generator().manual_seed(1)
    lengths, pages = [37, 150, 21], [[5, 9, 0], [3, 1, 2, 7, 11, 12, 20, 21, 22, 33], [40, 41]]
    x = [torch.randn((n, HIDDEN), generator=g).bfloat16().cuda() for n in lengths]
    steps = [[(0, 0, 35), (1, 0, 100)], [(0, 35, 1), (1, 100, 49), (2, 0, 20)], [(0, 36, 1), (1, 149, 1), (2, 20, 1)]]
    got = [torch.zeros(n, HIDDEN, dtype=torch.float64) for n in lengths]
    for step in steps:
        batch = Requests.of([n for _, _, n in step], [s + n for _, s, n in step], [pages[r] for r, _, _ in step], [-1] * len(step))
        h, residual = torch.cat([x[r][s:s + n] for r, s, n in step]), None
        for layer in layers:
            h, residual = layer.forward(h, residual, batch)
            layer.check()
        out, at = (h.double() + residual.double()).cpu(), 0
        for r, s, n in step:
            got[r][s:s + n] = out[at:at + n]
            at += n
    held = [[t.double().cpu().numpy() for t in layer.read_cache(lengths, pages)] for layer in layers]
    at = 0
    for r, n in enumerate(lengths):
        want, worst = reference(layers, [[t[at:at + n] for t in pair] for pair in held], x[r].double().cpu().numpy())
        at += n
        tol = 2.0 ** -5 * np.abs(want).max(axis=1, keepdims=True)
        assert np.all(np.abs(got[r].numpy() - want) <= tol), float((np.abs(got[r].numpy() - want) / tol).max())
        assert worst <= 1.0, worst
    # the tokens: those of the logits that the head forms, which are its rows' to bf16
    logits = head.logits(h, residual, batch)
    rows = (h.double() + residual.double()).cpu().numpy()
    y, _ = np_layer.rmsnorm(rows, head.norm.double().cpu().numpy(), head.eps)
    want = y @ dequantised(head.head).T
    assert np.all(np.abs(logits.double().cpu().numpy() - want) <= 2.0 ** -5 * np.abs(want).max(axis=1, keepdims=True))
    u, t, k, p = (torch.tensor(v, device="cuda") for v in ([0.1, 0.6, 0.93], [0.0, 0.7, 1.3], [0, 20, 0], [1.0, 1.0, 0.8]))
    tokens = head.forward(h, residual, batch, u, t, k.int(), p).tolist()
    for b in range(3):
        assert tokens[b] == np_sample.pick(logits[b].double().cpu().numpy(), float(u[b]), float(t[b]), int(k[b]), float(p[b]))[0]


@pytest.mark.parametrize("kv_bits", [16, 8, 4])
def test_a_policy_decodes_from_its_action_tokens(kv_bits):
    """Prompts, then eight captured single-token steps that feed one another; eager steps give the same tokens."""
    from paper_2412_01034_b200.decoder_layer import Requests, TokenHead
    layers, full, table = make(kv_bits, seed=3)
    head = TokenHead(full.norm.float(), torch.randn(VOCAB, HIDDEN, generator=torch.Generator().manual_seed(4)).cuda() * 0.08, 8, tokens=(500, 600))
    g = torch.Generator().manual_seed(5)
    lengths, pages = [20, 33], [[0, 1, 2, 3], [9, 8, 7, 6]]
    prompt = torch.randn(sum(lengths), HIDDEN, generator=g).bfloat16().cuda()
    us = torch.rand(9, 2, generator=g).cuda()
    t, k = torch.tensor([1.0, 0.0], device="cuda"), torch.tensor([30, 0], dtype=torch.int32, device="cuda")

    def step(x, batch, u):
        h, residual = x, None
        for layer in layers:
            h, residual = layer.forward(h, residual, batch)
        return head.forward(h, residual, batch, u, t, k)

    runs = []
    for captured in (False, True):
        tokens = [step(prompt, Requests.of(lengths, lengths, pages, [-1, -1]), us[0])]
        one = Requests.of([1, 1], [n + 8 for n in lengths], pages, [-1, -1])
        token, u, lens = tokens[0].clone(), us[1].clone(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
        for layer in layers:
            layer.reserve(2, 2, one.max_q, one.max_kv)

        def next_token():
            one.kv_len.copy_(lens)
            return step(table.index_select(0, token), one, u)

        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = next_token()
        for i in range(8):
            lens.add_(1)
            u.copy_(us[1 + i])
            if captured:
                graph.replay()
            else:
                out = next_token()
            token.copy_(out)
            tokens.append(out.clone())
        runs.append(torch.stack(tokens))
        for layer in layers:
            layer.check()
    assert torch.equal(runs[0], runs[1])
    assert ((runs[0] >= 500) & (runs[0] < 600)).all()


def test_refusals():
    from paper_2412_01034_b200.decoder_layer import DecoderLayer, TokenHead
    layers, head, _ = make(16, layers=1)
    with pytest.raises(ValueError, match="bf16 cache"):
        layers[0].read_cache([4], [[0]])
    with pytest.raises(ValueError, match="kv_bits"):
        DecoderLayer({}, 8, 4, 64, 4, 16, 64, 64, kv_bits=6)
    with pytest.raises(ValueError, match="tokens"):
        TokenHead(torch.ones(128, device="cuda"), torch.ones(64, 128, device="cuda"), 1, tokens=(10, 65))
