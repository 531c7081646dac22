"""A decoder layer of the Llama-2-7B backbone's sizes, where the projections are split along K: prompts and single tokens take
turns on one layer, against one pass over the whole sequences in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, DIM, FFN, PAGE = 4096, 32, 128, 11008, 16


def dequantised(lin):
    codes, s, z = lin.codes.double(), lin.scales.double(), lin.zeros.double()
    return (codes - z.repeat_interleave(128, dim=1)) * s.repeat_interleave(128, dim=1)


def rms(x, layer, weight):
    return x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + layer.eps) * weight.double()


def reference(layer, x):
    """One request from its first token on: x [n][HIDDEN] float64."""
    n = x.shape[0]
    t = (rms(x, layer, layer.norm1) @ dequantised(layer.qkv).t()).view(n, 3, HEADS, DIM)
    angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(DIM // 2, device="cuda").double() / (DIM // 2))
    wave = torch.polar(torch.ones_like(angle), angle)[:, None]
    turn = lambda v: torch.view_as_real(torch.complex(*v.split(DIM // 2, dim=2)) * wave).transpose(2, 3).reshape(n, HEADS, DIM)  # noqa: E731
    q, k, v = turn(t[:, 0]), turn(t[:, 1]), t[:, 2]
    score = torch.einsum("ihd,jhd->hij", q, k) * DIM ** -0.5
    hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
    att = torch.einsum("hij,jhd->ihd", score.masked_fill(hidden, float("-inf")).softmax(dim=2), v)
    x = x + att.reshape(n, -1) @ dequantised(layer.o).t()
    gu = rms(x, layer, layer.norm2) @ dequantised(layer.gate_up).t()
    return x + (torch.nn.functional.silu(gu[:, 0::2]) * gu[:, 1::2]) @ dequantised(layer.down).t()


@pytest.mark.parametrize("max_tokens", [300, 512])
def test_prompts_and_single_tokens_take_turns(max_tokens):
    """Single tokens after a prompt, a prompt beside a token after single tokens, and so on.

    About ten results are rounded to bf16 on the way (2^-9 of their size on average, independent of one another; the weights
    of the tensor-core GEMM as well); 2^-5 of the largest value of a row is more than ten standard deviations of the sum."""
    from paper_2412_01034_b200.decoder_layer import DecoderLayer, Requests
    g = torch.Generator(device="cuda").manual_seed(7)
    normal = lambda std, *s: torch.randn(s, generator=g, device="cuda") * std  # noqa: E731
    w = {"norm1": 1 + normal(0.1, HIDDEN), "norm2": 1 + normal(0.1, HIDDEN), "qkv": normal(0.016, 3 * HIDDEN, HIDDEN),
         "o": normal(0.016, HIDDEN, HIDDEN), "gate": normal(0.016, FFN, HIDDEN), "up": normal(0.016, FFN, HIDDEN),
         "down": normal(0.01, HIDDEN, FFN)}
    layer = DecoderLayer(w, HEADS, HEADS, DIM, num_pages=40, page_size=PAGE, max_pos=320, max_tokens=max_tokens)
    lengths = [47, 284, 12]
    pages = [list(range(0, 3)), list(range(20, 38)), [5]]
    x = [normal(1.0, n, HIDDEN).bfloat16() for n in lengths]
    steps = [[(0, 0, 40)], [(0, 40, 1)], [(0, 41, 1)], [(0, 42, 1), (1, 0, 280)], [(1, 280, 1)], [(0, 43, 1), (1, 281, 1)],
             [(0, 44, 1), (2, 0, 11)], [(0, 45, 1), (1, 282, 1), (2, 11, 1)], [(0, 46, 1), (1, 283, 1)]]
    got = [torch.zeros(n, HIDDEN, dtype=torch.float64, device="cuda") for n in lengths]
    for step in steps:
        batch = Requests.of([n for _, _, n in step], [s + n for _, s, n in step], [pages[r] for r, _, _ in step], [-1] * len(step))
        h, residual = layer.forward(torch.cat([x[r][s:s + n] for r, s, n in step]), None, batch)
        out, at = h.double() + residual.double(), 0
        for r, s, n in step:
            got[r][s:s + n] = out[at:at + n]
            at += n
    for r in range(len(lengths)):
        want = reference(layer, x[r].double())
        tol = 2.0 ** -5 * want.abs().amax(dim=1, keepdim=True)
        err = (got[r] - want).abs()
        assert torch.isfinite(got[r]).all() and (err <= tol).all(), (r, float((err / tol).max()), (err > tol).any(dim=1).nonzero().flatten().tolist())
