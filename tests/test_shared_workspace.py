"""One workspace, zero-filled once, for calls of different shapes that take turns on it."""
import pytest
import torch

from paper_2412_01034_b200 import _lib, build

COUNTERS = 16384   # one int for each of the 4096 row tiles that a split linear may have


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


@pytest.mark.parametrize("M,N,K,G", [(1, 22016, 4096, 128), (8, 22016, 4096, 128), (1, 28672, 4096, 128), (3, 11264, 2048, 128),
                                     (4, 9472, 4096, 128), (1, 1536, 512, 128), (1, 64, 128, 128), (5, 96, 192, 64), (2, 40, 24, 8),
                                     (12, 40, 24, 8)])
def test_the_gated_mlps_scratch_lies_behind_the_split_k_counters(lib, M, N, K, G):
    """For the shapes that are not fused the bf16 products are the last 2 M N bytes of the workspace; counters that other
    linears have begin where the workspace of a linear that does not split ends."""
    split_k = lib.qil_linear_w4a16_workspace_size(1, 22016, 4096, 128)
    assert lib.qil_linear_w4a16_workspace_size(1, 40000, 4096, 128) == split_k
    assert lib.qil_linear_w4a16_workspace_size(1, 4096, 11008, 128) > split_k + COUNTERS   # (this one splits)
    assert lib.qil_linear_w4a16_swiglu_workspace_size(M, N, K, G) - 2 * M * N >= split_k + COUNTERS


def weights(api, g, N, K, G=128):
    codes, scales, zeros = api.quantize_rtn_w4((torch.randn(N, K, generator=g) * 0.03).cuda(), G)
    return api.pack_w4(codes), scales, zeros


@pytest.mark.gpu
def test_linears_and_the_gated_mlp_take_turns_on_one_workspace():
    """Single tokens and prompts through the gated MLP and the projections around it (Llama-2-7B's sizes): the results are
    those of calls with a workspace of their own, bit for bit."""
    from paper_2412_01034_b200 import api
    g = torch.Generator().manual_seed(31)
    hidden, ffn = 4096, 11008
    gate_up, down, o = weights(api, g, 2 * ffn, hidden), weights(api, g, hidden, ffn), weights(api, g, hidden, hidden)
    odd = weights(api, g, 96, 192, 64)   # (K is no multiple of 128: the general kernel, no workspace of its own)
    calls = {}
    for M in (1, 8, 9, 40, 280):
        x, t = torch.randn(M, hidden, generator=g).bfloat16().cuda(), torch.randn(M, ffn, generator=g).bfloat16().cuda()
        u = torch.randn(M, 192, generator=g).bfloat16().cuda()
        calls[M, "gate_up"] = lambda ws, x=x: api.linear_w4a16_swiglu(x, *gate_up, 2 * ffn, 128, workspace=ws)
        calls[M, "down"] = lambda ws, t=t: api.linear_w4a16(t, *down, hidden, 128, workspace=ws)
        calls[M, "o"] = lambda ws, x=x: api.linear_w4a16(x, *o, hidden, 128, workspace=ws)
        calls[M, "odd"] = lambda ws, u=u: api.linear_w4a16_swiglu(u, *odd, 96, 64, workspace=ws)
    want = {k: f(None) for k, f in calls.items()}
    size = max(max(api.linear_w4a16_swiglu_workspace_size(M, 2 * ffn, hidden, 128), api.linear_w4a16_workspace_size(M, hidden, ffn, 128),
                   api.linear_w4a16_workspace_size(M, hidden, hidden, 128), api.linear_w4a16_swiglu_workspace_size(M, 96, 192, 64))
               for M in (1, 8, 9, 40, 280))
    ws = api.new_workspace(size)
    for M in (280, 1, 1, 40, 8, 9, 1, 280, 8, 40):
        for name in ("o", "gate_up", "odd", "down", "gate_up", "o", "down"):
            assert torch.equal(calls[M, name](ws), want[M, name]), (M, name)
    assert int(ws[:4].view(torch.int32)[0]) == 0


@pytest.mark.parametrize("max_tokens", [1, 7, 8, 200, 300, 512, 768, 1024])
def test_the_decoder_layers_workspace_serves_every_row_count(lib, max_tokens):
    """No batch of up to max_tokens rows needs more than the layer has (the GEMM would take a slower way without a word)."""
    from paper_2412_01034_b200 import decoder_layer
    hidden, ffn, qkv = 4096, 11008, 12288
    size = decoder_layer.linear_workspace_size(max_tokens, [(hidden, hidden), (hidden, ffn), (qkv, hidden)], (2 * ffn, hidden))
    for M in range(1, max_tokens + 1):
        for N, K in ((hidden, hidden), (hidden, ffn), (qkv, hidden)):
            assert lib.qil_linear_w4a16_workspace_size(M, N, K, 128) <= size, (M, N, K)
        assert lib.qil_linear_w4a16_swiglu_workspace_size(M, 2 * ffn, hidden, 128) <= size, M
    with8 = decoder_layer.linear_workspace_size(max_tokens, [(hidden, hidden)], (2 * ffn, hidden), [(qkv, hidden)])
    assert with8 >= lib.qil_linear_w4a4_workspace_size(max_tokens, qkv, hidden)


@pytest.mark.parametrize("max_tokens", [1, 2, 5])
def test_layers_made_for_a_few_rows_take_what_the_unfused_gated_mlp_takes(lib, max_tokens):
    """The row counts of the unfused form (up to 8) always have room for its scratch, which is a must; the GEMM above has a way
    without its parts."""
    from paper_2412_01034_b200 import decoder_layer
    size = decoder_layer.linear_workspace_size(max_tokens, [(4096, 4096), (4096, 11008), (12288, 4096)], (22016, 4096))
    for M in range(1, 10):
        assert lib.qil_linear_w4a16_swiglu_workspace_size(M, 22016, 4096, 128) <= size, M
