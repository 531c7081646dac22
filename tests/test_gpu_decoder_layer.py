"""The layer operators together with the quantised linears: a decoder layer that serves requests in several steps against
one pass over the whole sequences in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import np_layer

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, KV_HEADS, DIM, FFN, PAGE = 512, 8, 4, 64, 768, 16


def dequantised(lin):
    codes, s, z = (t.double().cpu().numpy() for t in (lin.codes, lin.scales, lin.zeros))
    return (codes - np.repeat(z, 128, axis=1)) * np.repeat(s, 128, axis=1)


def make(bits, adapters, layers=2, seed=0):
    from paper_2412_01034_b200.decoder_layer import DecoderLayer
    g = torch.Generator().manual_seed(seed)
    normal = lambda std, *s: (torch.randn(s, generator=g) * std).cuda()  # noqa: E731
    made = []
    for _ in range(layers):
        w = {"norm1": 1 + normal(0.1, HIDDEN), "norm2": 1 + normal(0.1, HIDDEN), "qkv": normal(0.04, (HEADS + 2 * KV_HEADS) * DIM, HIDDEN),
             "o": normal(0.04, HIDDEN, HEADS * DIM), "gate": normal(0.04, FFN, HIDDEN), "up": normal(0.04, FFN, HIDDEN),
             "down": normal(0.04, HIDDEN, FFN)}
        ad = None
        if adapters:
            ad = (normal(HIDDEN ** -0.5, 3, 8, HIDDEN).bfloat16(), normal(0.3, 3, w["qkv"].shape[0], 8).bfloat16(),
                  torch.tensor([0.5, 1.0, -0.7], device="cuda"))
        made.append((DecoderLayer(w, HEADS, KV_HEADS, DIM, num_pages=64, page_size=PAGE, max_pos=400, max_tokens=256, qkv_bits=bits,
                                  adapters=ad), w))
    return made


def reference(layers, x, adapter):
    """One request from its first token on: x [n][HIDDEN] float64."""
    n = len(x)
    for layer, w in layers:
        v, _ = np_layer.rmsnorm(x, layer.norm1.double().cpu().numpy(), layer.eps)
        if layer.qkv_bits == 8:
            codes, scales = (t.double().cpu().numpy() for t in layer.qkv8)
            qkv = v @ (codes * scales[:, None]).T
        else:
            qkv = v @ dequantised(layer.qkv).T
        if layer.adapters:
            a, b, scales = (t.double().cpu().numpy() for t in layer.adapters)
            qkv += np_layer.lora_batch(v, a, b, [0, n], [adapter], scales)[0]
        t = qkv.reshape(n, -1, DIM)
        turned = np.stack([np_layer.rope_rotate(t[i, : HEADS + KV_HEADS], i, 10000.0) for i in range(n)])
        att, _, _ = np_layer.attn(turned[:, :HEADS], turned[:, HEADS:], t[:, HEADS + KV_HEADS:], 0, DIM ** -0.5)
        x = x + att.reshape(n, -1) @ dequantised(layer.o).T
        v, _ = np_layer.rmsnorm(x, layer.norm2.double().cpu().numpy(), layer.eps)
        gu = v @ dequantised(layer.gate_up).T
        x = x + (gu[:, 0::2] / (1 + np.exp(-gu[:, 0::2])) * gu[:, 1::2]) @ dequantised(layer.down).T
    return x


@pytest.mark.parametrize("bits,adapters", [(4, False), (4, True), (8, True), (8, False)])
def test_decoder_layers_serve_requests_step_by_step(bits, adapters):
    """Three requests: a prompt at once, a prompt in two chunks next to single tokens, and one that joins later.

    Two layers, in each of which about ten results are rounded to bf16 (2^-9 of their size on average, independent of one
    another), or to 127 steps of the row's maximum (int8); the residual stream carries the sum: 2^-5 of the largest value
    of a row (2^-4 with int8 projections) is more than ten standard deviations of it."""
    from paper_2412_01034_b200.decoder_layer import Requests
    layers = make(bits, adapters)
    g = torch.Generator().manual_seed(1)
    lengths, adapter = [37, 150, 21], [2, -1, 0]
    x = [torch.randn((n, HIDDEN), generator=g).bfloat16().cuda() for n in lengths]
    pages = [[5, 9, 0], [3, 1, 2, 7, 11, 12, 20, 21, 22, 33], [40, 41]]
    steps = [  # (request, first token, tokens) of every step
        [(0, 0, 35), (1, 0, 100)],
        [(0, 35, 1), (1, 100, 49), (2, 0, 20)],
        [(0, 36, 1), (1, 149, 1), (2, 20, 1)],
    ]
    got = [torch.zeros(n, HIDDEN, dtype=torch.float64) for n in lengths]
    for step in steps:
        batch = Requests.of([n for _, _, n in step], [s + n for _, s, n in step], [pages[r] for r, _, _ in step],
                            [adapter[r] for r, _, _ in step])
        h, residual = torch.cat([x[r][s:s + n] for r, s, n in step]), None
        for layer, _ in layers:
            h, residual = layer.forward(h, residual, batch)
        out, at = (h.double() + residual.double()).cpu(), 0
        for r, s, n in step:
            got[r][s:s + n] = out[at:at + n]
            at += n
    for r in range(3):
        want = reference(layers, x[r].double().cpu().numpy(), adapter[r])
        tol = (2.0 ** -4 if bits == 8 else 2.0 ** -5) * np.abs(want).max(axis=1, keepdims=True)
        err = np.abs(got[r].numpy() - want)
        assert np.all(err <= tol), float((err / tol).max())
