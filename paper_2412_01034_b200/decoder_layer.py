"""One decoder layer of a Llama-2 style backbone (the OpenVLA language model, App. A.4.2) over quantised linears, for a batch
of requests that are at different places: prompts, chunks of prompts and single tokens together.

The linears are the library's (4-bit weight-only; the fused query / key / value projection optionally W8A8), and what lies
between them runs on its layer operators: residual norm, rotary embedding with append to the paged cache, attention over
the cache, low-rank adapters per request.  Weights are quantised on the device once; ``forward`` only enqueues kernels.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import api

GROUP = 128


@dataclass
class Requests:
    """A batch as the kernels read it (packed rows, lengths, pages, adapters) and the bounds that the host knows."""
    cu_q: torch.Tensor          # int32 [B + 1]
    kv_len: torch.Tensor        # int32 [B], the new tokens included
    block_table: torch.Tensor   # int32 [B][max_pages]
    adapter: torch.Tensor       # int32 [B], -1: none
    max_q: int
    max_kv: int

    @staticmethod
    def of(q_lens, kv_lens, tables, adapters, device="cuda") -> "Requests":
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=device)  # noqa: E731
        starts = [0]
        for n in q_lens:
            starts.append(starts[-1] + n)
        width = max(1, max(len(t) for t in tables))
        return Requests(ints(starts), ints(kv_lens), ints([list(t) + [0] * (width - len(t)) for t in tables]), ints(adapters),
                        max(q_lens), max(kv_lens))


class Linear4:
    """A 4-bit weight-only linear on the canonical layout."""

    def __init__(self, w):
        self.N, self.K = w.shape
        self.codes, self.scales, self.zeros = api.quantize_rtn_w4(w, GROUP)
        self.packed = api.pack_w4(self.codes)

    def __call__(self, x, workspace):
        return api.linear_w4a16(x, self.packed, self.scales, self.zeros, self.N, GROUP, workspace=workspace)


def linear_workspace_size(max_tokens, linears, gate_up, linears8=()):
    """Bytes that serve batches of 1 ... max_tokens rows (and of up to 9) through the 4-bit linears, the gated MLP and the W8A8
    linears of these (N, K).  Every row count is asked for: the prefill GEMM's need grows and shrinks with the tiles that the rows
    are cut into (at 4096 x 11008, 280 rows need more than 1000 do), and with less it falls back to whole tiles on part of the
    GPU."""
    size = 256
    for M in range(1, max(max_tokens, 9) + 1):   # (more rows than max_tokens run too, but the gated MLP's scratch has to be there)
        size = max(size, api.linear_w4a16_swiglu_workspace_size(M, *gate_up, GROUP),
                   *(api.linear_w4a16_workspace_size(M, N, K, GROUP) for N, K in linears),
                   *(api.linear_w4a4_workspace_size(M, N, K) for N, K in linears8))
    return size


class DecoderLayer:
    """weights: fp32 CUDA tensors norm1, norm2 [hidden], qkv [(H + 2 Hk) D][hidden], o [hidden][H D], gate, up [ffn][hidden],
    down [hidden][ffn].  adapters: None or (a [n][r][hidden], b [n][(H + 2 Hk) D][r], scales [n]) beside the qkv projection.
    The caches and workspaces are the layer's own: its calls belong on one stream, or have to be ordered by the caller.
    Steps may be captured in CUDA graphs."""

    def __init__(self, weights, heads, kv_heads, head_dim, num_pages, page_size, max_pos, max_tokens, qkv_bits=4, adapters=None,
                 eps=1e-5, theta=10000.0):
        self.heads, self.kv_heads, self.head_dim, self.eps, self.qkv_bits = heads, kv_heads, head_dim, eps, qkv_bits
        self.norm1, self.norm2 = (weights[n].to(torch.bfloat16) for n in ("norm1", "norm2"))
        if qkv_bits == 8:
            codes, scales, _ = api.quantize_rtn_w8(weights["qkv"], weights["qkv"].shape[1], symmetric=True)
            self.qkv8 = (codes, scales.reshape(-1).contiguous())
        else:
            self.qkv = Linear4(weights["qkv"])
        self.o, self.down = Linear4(weights["o"]), Linear4(weights["down"])
        self.gate_up = Linear4(api.interleave_rows(weights["gate"], weights["up"]))
        self.adapters = adapters
        self.cos_sin = api.rope_table(max_pos, head_dim, theta)
        self.k_cache, self.v_cache = api.new_kv_cache(num_pages, kv_heads, page_size, head_dim)
        # one workspace for all linears of the layer (they run one after another)
        self.workspace = api.new_workspace(linear_workspace_size(
            max_tokens, [(lin.N, lin.K) for lin in (self.o, self.down) + (() if qkv_bits == 8 else (self.qkv,))],
            (self.gate_up.N, self.gate_up.K), [tuple(weights["qkv"].shape)] if qkv_bits == 8 else []))
        # the adapters' need is greatest for one request with all the rows (more requests: fewer slices of K)
        self.max_tokens = max_tokens
        self.lora_workspace = None
        if adapters:
            need = max(api.lora_batch_workspace_size(M, 1, adapters[0].shape[1]) for M in range(1, max_tokens + 1))
            self.lora_workspace = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        self._attn_workspaces = []

    def _attn_workspace(self, tokens, requests, max_q, max_kv):
        """The attention's workspace for such a batch: the newest one if it is large enough, or a larger one.  The older ones
        stay (each is at least twice the one before), because a captured graph may hold them."""
        need = api.attn_paged_workspace_size(tokens, requests, self.heads, self.kv_heads, self.head_dim, max_q, max_kv)
        held = self._attn_workspaces[-1].numel() if self._attn_workspaces else 0
        if held < need:
            if torch.cuda.is_current_stream_capturing():
                return None   # (one of the graph's own: what is cleared in a capture is only cleared when the graph runs)
            self._attn_workspaces.append(api.new_workspace(max(need, 2 * held)))
        return self._attn_workspaces[-1]

    def reserve(self, tokens, requests, max_q, max_kv):
        """Makes room for batches of up to this many new tokens and requests with these bounds, so that ``forward`` need not
        (before a capture, say).  Batches that differ in shape may need more than a larger one: reserve each kind."""
        self._attn_workspace(tokens, requests, max_q, max_kv)

    def check(self):
        """Waits for the current stream and raises QilError if a kernel of an earlier step has recorded a failure."""
        for workspace in (self.workspace, *self._attn_workspaces):
            api.check_workspace(workspace)

    def _qkv(self, h, residual, batch):
        """The norm and the fused projection with the requests' adapters: (qkv, the residual stream)."""
        if self.qkv_bits == 8:
            x = torch.empty_like(h) if self.adapters else None   # the adapters read the norm in bf16
            codes, scales, *rest = api.rmsnorm_a8(h, self.norm1, self.eps, residual=residual, out=x)
            qkv = api.linear_w8a8(codes, scales, *self.qkv8, workspace=self.workspace)
            residual = rest[0] if rest else h
        else:
            x = api.rmsnorm(h, self.norm1, self.eps, residual=residual)
            x, residual = x if residual is not None else (x, h)
            qkv = self.qkv(x, self.workspace)
        if self.adapters:
            a, b, scales = self.adapters
            api.lora_batch_add(x, a, b, qkv, batch.cu_q, batch.adapter, scales,
                               workspace=self.lora_workspace if x.shape[0] <= self.max_tokens else None)
        return qkv, residual

    def forward(self, h, residual, batch: Requests):
        """h [T][hidden]: the layer's input (residual None) or the part of it that is still to be added to residual.
        Returns the same pair for the next layer."""
        qkv, residual = self._qkv(h, residual, batch)
        q = api.rope_append(qkv, self.cos_sin, self.k_cache, self.v_cache, batch.cu_q, batch.kv_len, batch.block_table, self.heads)
        a = api.attn_paged(q, self.k_cache, self.v_cache, batch.cu_q, batch.kv_len, batch.block_table, batch.max_q, batch.max_kv,
                           workspace=self._attn_workspace(q.shape[0], batch.kv_len.shape[0], batch.max_q, batch.max_kv))
        o = self.o(a.view(a.shape[0], -1), self.workspace)
        x, residual = api.rmsnorm(o, self.norm2, self.eps, residual=residual)
        g = api.linear_w4a16_swiglu(x, self.gate_up.packed, self.gate_up.scales, self.gate_up.zeros, self.gate_up.N, GROUP,
                                    workspace=self.workspace)
        return self.down(g, self.workspace), residual
