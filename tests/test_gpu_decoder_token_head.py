"""The token head's rows without a choice."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HIDDEN, VOCAB = 256, 600


@pytest.mark.parametrize("tokens", [None, (0, 600), (1, 2), (500, 600)])
def test_rows_without_a_choice_keep_their_mark(tokens):
    """A hidden row that is no number has no logit above -inf: -1, whatever range the head chooses from; eager and captured."""
    from paper_2412_01034_b200.decoder_layer import Requests, TokenHead
    g = torch.Generator().manual_seed(7)
    head = TokenHead(torch.ones(HIDDEN, device="cuda"), torch.randn(VOCAB, HIDDEN, generator=g).cuda() * 0.1, 4, tokens=tokens)
    first, end = tokens or (0, VOCAB)
    batch = Requests.of([2, 1, 1], [2, 1, 1], [[0], [1], [2]], [-1] * 3)
    h = torch.randn(4, HIDDEN, generator=g).bfloat16().cuda()
    h[1, 9] = math.nan   # the last row of request 0
    h[3] = math.nan
    residual = torch.zeros_like(h)
    u, t = torch.tensor([0.3, 0.6, 0.9], device="cuda"), torch.tensor([0.0, 1.0, 1.0], device="cuda")
    top_p = torch.tensor([1.0, 0.9, 0.9], device="cuda")

    def run():
        return head.forward(h, residual, batch, u, t, top_p=top_p)

    token = run()
    assert token.dtype == torch.int32 and token[0] == -1 and first <= token[1] < end and token[2] == -1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    graph.replay()
    assert torch.equal(captured, token)
