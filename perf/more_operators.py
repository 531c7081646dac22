"""Operators of a serving step over a quantised key / value cache, and the choice of the next token, as cases that can be
timed and compared.

The cache holds every key and value head in 8 or 4 bits with one scale (4 bits: and one zero point) per token and head: the
rotary embedding's append quantises as it writes, a read-back gives the cached tokens as bf16 rows, and the attention of
prompts, chunks and single tokens reads the codes.  At the end of a step the logits become tokens: temperature, top-k,
top-p and min-p, with the uniform numbers given.

A case is a dict of plain values; ``prepare`` makes what a serving program has in hand, ``run`` is one call of the
operator, ``exact`` the same result from the definition in 64 bits.  With ``own`` false ``run`` computes the plain form in
elementary torch operations; with ``own`` true it calls this library.
"""
import math
import random

import numpy as np
import torch

own = False

THETA = 10000.0
DEV = "cuda"


# ------------------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # 32 requests in their decode phase, one new token each, into an 8-bit cache; the new tokens are read back
        {"name": "append8_decode_32", "op": "append", "bits": 8, "batch": 32, "mode": "decode", "q_len": 1, "kv_len": 287, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 16},
        # seven prompts of different lengths into a 4-bit cache, read back
        {"name": "append4_prompts_7", "op": "append", "bits": 4, "batch": 7, "mode": "prompt", "q_len": 1111, "kv_len": 1111, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 64},
        # one robot's short context leaves the cache (a request that moves to another worker)
        {"name": "read8_context_1", "op": "read", "bits": 8, "batch": 1, "mode": "decode", "q_len": 1, "kv_len": 287, "heads": 32, "kv_heads": 32,
         "dim": 128, "page": 16},
        # the contexts of 24 requests, grouped heads, 4 bits
        {"name": "read4_contexts_24", "op": "read", "bits": 4, "batch": 24, "mode": "decode", "q_len": 1, "kv_len": 2111, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 64},
        # one robot's action token over its own short context: latency
        {"name": "attn8_decode_1", "op": "attn", "bits": 8, "batch": 1, "mode": "decode", "q_len": 1, "kv_len": 287, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 16},
        # a full decode batch with contexts of different lengths: bandwidth
        {"name": "attn8_decode_32", "op": "attn", "bits": 8, "batch": 32, "mode": "decode", "q_len": 1, "kv_len": 4099, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 64},
        # grouped heads, longer contexts, 4 bits
        {"name": "attn4_decode_48", "op": "attn", "bits": 4, "batch": 48, "mode": "decode", "q_len": 1, "kv_len": 9001, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 64},
        # the 280-token prompts of four requests
        {"name": "attn8_prompt_280", "op": "attn", "bits": 8, "batch": 4, "mode": "uniform", "q_len": 280, "kv_len": 280, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 16},
        # continuous batching: one request's chunk of 512 new tokens next to 15 single tokens, grouped heads, 4 bits
        {"name": "attn4_mixed_gqa", "op": "attn", "bits": 4, "batch": 16, "mode": "mixed", "q_len": 512, "kv_len": 6001, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 64},
        # a long prompt taken in chunks: the second 4096 tokens over a cache of 8192
        {"name": "attn8_chunk_4096", "op": "attn", "bits": 8, "batch": 1, "mode": "uniform", "q_len": 4096, "kv_len": 8192, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 64},
        # the next token of one request: temperature, top-k and top-p
        {"name": "sample_1", "op": "sample", "batch": 1, "vocab": 32000, "type": "bf16", "mode": "all"},
        # the tokens of a full batch over a large vocabulary of odd size, every request with settings of its own
        {"name": "sample_64", "op": "sample", "batch": 64, "vocab": 128003, "type": "fp32", "mode": "mixed"},
    ]


def _log_int(rng, lo, hi):
    """A whole number spread over the logarithm of its range; no multiple of 1024, as lengths in service hardly ever are."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n - (n % 1024 == 0)


def draw(rng):
    op = rng.choice(["append", "read", "attn", "attn", "attn", "sample"])
    if op == "sample":
        vocab = _log_int(rng, 256, 128003)
        return {"op": op, "batch": _log_int(rng, 1, min(64, 8_000_000 // vocab)), "vocab": vocab, "type": rng.choice(["bf16", "fp32"]),
                "mode": rng.choice(["all", "top_p", "min_p", "temperature", "greedy", "mixed", "mixed"])}
    heads, kv_heads, dim = rng.choice([(32, 32, 128), (32, 8, 128), (28, 4, 128), (16, 16, 64), (32, 4, 64), (12, 4, 64)])
    case = {"op": op, "bits": rng.choice([8, 4]), "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": rng.choice([16, 32, 64, 128])}
    if op == "append":
        mode = rng.choice(["decode", "prompt"])
        q_len = 1 if mode == "decode" else _log_int(rng, 3, 1000)
        return dict(case, batch=_log_int(rng, 1, 48) if mode == "decode" else rng.randint(1, 8), mode=mode, q_len=q_len,
                    kv_len=rng.randint(q_len, 400) if mode == "decode" else q_len)
    if op == "read":
        return dict(case, batch=_log_int(rng, 1, 24), mode="decode", q_len=1, kv_len=_log_int(rng, 16, 2111))
    mode = rng.choice(["decode", "decode", "prompt", "uniform", "mixed", "ragged"])
    batch = {"decode": _log_int(rng, 1, 48), "mixed": rng.randint(2, 24)}.get(mode, rng.randint(1, 6))
    if mode == "decode":
        q_len, kv_len = 1, _log_int(rng, 16, 9001)
    else:
        q_len = _log_int(rng, 5, 1500)
        kv_len = q_len if mode == "prompt" else q_len + _log_int(rng, 1, 4000)
        kv_len -= kv_len > q_len and kv_len % 1024 == 0
    while batch > 1 and (batch * heads * q_len * kv_len > 1_000_000_000 or batch * kv_len * kv_heads > 2_500_000):
        batch -= 1
    return dict(case, batch=batch, mode=mode, q_len=q_len, kv_len=kv_len)


def _lengths(case):
    """(new tokens, cached tokens with them) of each request: the case's own numbers decide, not the seed."""
    r = random.Random("%d %s %d %d" % (case["batch"], case["mode"], case["q_len"], case["kv_len"]))
    q_len, kv_len, rest = case["q_len"], case["kv_len"], case["batch"] - 1
    if case["mode"] == "decode":
        kv = [kv_len] + [r.randint(max(1, kv_len // 4), kv_len) for _ in range(rest)]
        return list(kv) if case["op"] == "read" else [1] * (rest + 1), kv
    if case["mode"] == "uniform":
        return [q_len] * (rest + 1), [kv_len] * (rest + 1)
    if case["mode"] == "mixed":
        return [q_len] + [1] * rest, [kv_len] + [r.randint(1, kv_len) for _ in range(rest)]
    q = [q_len] + [r.randint(max(1, q_len // 5), q_len) for _ in range(rest)]
    if case["mode"] == "prompt":
        return q, list(q)
    return q, [kv_len] + [n + r.randint(0, kv_len - q_len) for n in q[1:]]


# ------------------------------------------------------------------------------------------------------------------
# the quantised cache in plain operations
#   8 bits: codes int8 [...][D], scales bf16 [...]            value q s
#   4 bits: codes int32 [...][D / 8], scales bf16 [...][2]    value (q - z) s; code d of a head in word d / 8, bits 4 (d % 8)
# ------------------------------------------------------------------------------------------------------------------
def _quantise(x, bits):
    """fp32 heads [...][D] as (codes, scales); fp32 operations one by one, as the format says."""
    if bits == 8:
        s = (x.abs().amax(dim=-1) / 127.0).to(torch.bfloat16)
        none = s < 2.0 ** -126
        s = torch.where(none, 1.0, s)
        q = torch.round(torch.where(none[..., None], 0.0, x) / s.float()[..., None]).clamp(-128, 127)
        return q.to(torch.int8), s
    lo, hi = x.amin(dim=-1).clamp(max=0.0), x.amax(dim=-1).clamp(min=0.0)
    s = ((hi - lo) / 15.0).to(torch.bfloat16)
    none = s < 2.0 ** -126
    s = torch.where(none, 1.0, s)
    z = torch.round(torch.where(none, 0.0, -lo) / s.float()).clamp(0, 15)
    q = (torch.round(torch.where(none[..., None], 0.0, x) / s.float()[..., None]) + z[..., None]).clamp(0, 15).to(torch.int32)
    return _pack(q), torch.stack([s, z.to(torch.bfloat16)], dim=-1)


def _pack(q):
    q = q.view(*q.shape[:-1], -1, 8)
    word = q[..., 0].clone()
    for i in range(1, 8):
        word |= q[..., i] << (4 * i)
    return word


def _unpack(words):
    shift = torch.arange(0, 32, 4, device=words.device, dtype=torch.int32)
    return ((words[..., None] >> shift) & 15).flatten(-2)


def _values(codes, scales, bits):
    """fp32 values that codes and scales stand for."""
    if bits == 8:
        return codes.float() * scales.float()[..., None]
    return (_unpack(codes).float() - scales[..., 1].float()[..., None]) * scales[..., 0].float()[..., None]


# ------------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------------
def _normal(g, *shape, std=1.0, dtype=torch.bfloat16):
    out = torch.empty(shape, dtype=dtype, device=DEV)
    return out.normal_(0.0, std, generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _starts(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def _paged(case, g):
    """Lengths, block table (pages in no order) and the quantised cache."""
    q_lens, kv_lens = _lengths(case)
    page = case["page"]
    per_seq = [-(-n // page) for n in kv_lens]
    width, total = max(per_seq), sum(per_seq)
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    first = _ints(_starts(per_seq)[:-1].tolist())
    column = torch.arange(width, device=DEV, dtype=torch.int32)
    used = column[None, :] < _ints(per_seq)[:, None]
    table = torch.where(used, order[(first[:, None] + column).clamp(max=total - 1).long()], 0).to(torch.int32).contiguous()
    sides = []
    for _ in range(2):
        parts = [_quantise(_normal(g, n, case["kv_heads"], page, case["dim"], dtype=torch.float32), case["bits"])
                 for n in [256] * (total // 256) + [total % 256] * (total % 256 > 0)]
        sides.append([torch.cat([p[i] for p in parts]) for i in range(2)])
    (k, ks), (v, vs) = sides
    return {"cu_q": _ints(_starts(q_lens).tolist()), "kv_len": _ints(kv_lens), "table": table, "cache": [k, v, ks, vs], "max_q": max(q_lens),
            "max_kv": max(kv_lens), "tokens": sum(q_lens)}


# (temperature, top_k, top_p, min_p) of the requests in turn; 0, 1 and 0 switch the last three off
_SETTINGS = {"all": [(0.8, 50, 0.95, 0.0)], "top_p": [(1.0, 0, 0.9, 0.0)], "min_p": [(1.2, 0, 1.0, 0.05)], "temperature": [(0.7, 0, 1.0, 0.0)],
             "greedy": [(0.0, 0, 1.0, 0.0)],
             "mixed": [(0.8, 50, 0.95, 0.0), (1.0, 0, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.02), (0.6, 0, 0.99, 0.0), (1.0, 1000, 1.0, 0.0),
                       (1.5, 200, 0.8, 0.1)]}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": case, "op": case["op"]}
    if case["op"] == "sample":
        B, V = case["batch"], case["vocab"]
        # most of a vocabulary lies in a wide bell, a few candidates well above it
        x = _normal(g, B, V, std=2.0, dtype=torch.float32)
        ahead = torch.randint(0, V, (B, 12), generator=g, device=DEV)
        x.scatter_add_(1, ahead, 4.0 + 5.0 * torch.rand(B, 12, generator=g, device=DEV))
        s["logits"] = x.to(torch.bfloat16) if case["type"] == "bf16" else x
        s["u"] = torch.rand(B, generator=g, device=DEV)
        rows = [_SETTINGS[case["mode"]][b % len(_SETTINGS[case["mode"]])] for b in range(B)]
        for i, name in enumerate(("temperature", "top_k", "top_p", "min_p")):
            s[name] = torch.tensor([r[i] for r in rows], dtype=torch.int32 if name == "top_k" else torch.float32, device=DEV)
        return s
    s.update(_paged(case, g))
    if case["op"] == "append":
        s["qkv"] = _normal(g, s["tokens"], (case["heads"] + 2 * case["kv_heads"]) * case["dim"])
        half = case["dim"] // 2
        angle = np.outer(np.arange(s["max_kv"], dtype=np.float64), THETA ** (-np.arange(half, dtype=np.float64) / half))
        s["cos_sin"] = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], axis=1)).to(torch.float32).to(DEV)
    elif case["op"] == "attn":
        s["q"] = _normal(g, s["tokens"], case["heads"], case["dim"])
        s["scale"] = case["dim"] ** -0.5
        s["workspace"] = None
    return s


# ------------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------------
def run(state):
    return _OWN[state["op"]](state) if own else _PLAIN[state["op"]](state)


def _own_append(s):
    from paper_2412_01034_b200 import api
    cache = api.QuantCache(*s["cache"])
    q = api.rope_append_q(s["qkv"], s["cos_sin"], cache, s["cu_q"], s["kv_len"], s["table"], s["case"]["heads"])
    # the values that the new tokens' codes stand for
    return [q, *api.kv_read_q(cache, s["cu_q"], s["kv_len"], s["table"], s["tokens"])]


def _own_read(s):
    from paper_2412_01034_b200 import api
    return list(api.kv_read_q(api.QuantCache(*s["cache"]), s["cu_q"], s["kv_len"], s["table"], s["tokens"]))


def _own_attn(s):
    from paper_2412_01034_b200 import api
    c = s["case"]
    cache = api.QuantCache(*s["cache"])
    if s["workspace"] is None:
        s["workspace"] = api.new_workspace(api.attn_paged_q_workspace_size(s["tokens"], c["batch"], c["heads"], c["kv_heads"], c["dim"],
                                                                           c["bits"], s["max_q"], s["max_kv"]))
    return api.attn_paged_q(s["q"], cache, s["cu_q"], s["kv_len"], s["table"], s["max_q"], s["max_kv"], scale=s["scale"],
                            workspace=s["workspace"])


def _own_sample(s):
    from paper_2412_01034_b200 import api
    return api.sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])


def _positions(s):
    """Request and cache position of every row."""
    t = torch.arange(s["tokens"], device=DEV)
    cu = s["cu_q"].long()
    seq = torch.bucketize(t, cu[1:], right=True)
    return seq, s["kv_len"].long()[seq] - (cu[1:] - cu[:-1])[seq] + t - cu[:-1][seq]


def _places(s):
    seq, pos = _positions(s)
    page = s["case"]["page"]
    return s["table"][seq, pos // page].long(), pos % page, pos


def _plain_read(s):
    page, slot, _ = _places(s)
    k, v, ks, vs = s["cache"]
    bits = s["case"]["bits"]
    return [_values(codes[page, :, slot], scales[page, :, slot], bits).to(torch.bfloat16) for codes, scales in ((k, ks), (v, vs))]


def _plain_append(s):
    c = s["case"]
    page, slot, pos = _places(s)
    H, Hk, half = c["heads"], c["kv_heads"], c["dim"] // 2
    x = s["qkv"].view(s["tokens"], -1, c["dim"])
    cos, sin = s["cos_sin"][pos, None, :half], s["cos_sin"][pos, None, half:]
    first, second = x[:, : H + Hk, :half].float(), x[:, : H + Hk, half:].float()
    turned = torch.cat([first * cos - second * sin, second * cos + first * sin], dim=2)
    k, v, ks, vs = s["cache"]
    k[page, :, slot], ks[page, :, slot] = _quantise(turned[:, H:], c["bits"])
    v[page, :, slot], vs[page, :, slot] = _quantise(x[:, H + Hk:].float(), c["bits"])
    return [turned[:, :H].to(torch.bfloat16), *_plain_read(s)]


def _plain_attn(s):
    c = s["case"]
    B, D, H, G = c["batch"], c["dim"], c["kv_heads"], c["heads"] // c["kv_heads"]
    seq, pos = _positions(s)
    col = torch.arange(s["tokens"], device=DEV) - s["cu_q"].long()[seq]
    q = torch.zeros(B, s["max_q"], H, G, D, device=DEV)
    q[seq, col] = s["q"].view(s["tokens"], H, G, D).float() * s["scale"]
    at = torch.full((B, s["max_q"]), -1, device=DEV, dtype=torch.long)
    at[seq, col] = pos
    k, v, ks, vs = s["cache"]
    pages = s["table"].long()
    keys, values = (_values(a[pages], b[pages], c["bits"]).transpose(2, 3).reshape(B, -1, H, D) for a, b in ((k, ks), (v, vs)))
    j = torch.arange(keys.shape[1], device=DEV)
    values = values.masked_fill_((j[None, :] >= s["kv_len"][:, None])[:, :, None, None], 0.0)
    score = q.permute(0, 2, 1, 3, 4).reshape(B, H, s["max_q"] * G, D) @ keys.permute(0, 2, 3, 1)
    score = score.view(B, H, s["max_q"], G, -1).masked_fill_((j[None, None, :] > at[:, :, None])[:, None, :, None, :], float("-inf"))
    top = score.amax(dim=-1, keepdim=True)
    p = torch.exp_(score.sub_(torch.where(torch.isinf(top), 0.0, top)))
    total = p.sum(dim=-1, keepdim=True)
    out = p.view(B, H, s["max_q"] * G, -1) @ values.permute(0, 2, 1, 3)
    out = out.view(B, H, s["max_q"], G, D) / torch.where(total == 0, 1.0, total)
    return out.permute(0, 2, 1, 3, 4)[seq, col].reshape(s["tokens"], c["heads"], D).to(torch.bfloat16)


def _plain_sample(s):
    # (in 64 bits: which token a running sum passes must not hang on the order in which it was added up)
    x, V = s["logits"].double(), s["case"]["vocab"]
    t = s["temperature"].double()[:, None]
    x, index = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp((x - x[:, :1]) / torch.where(t > 0, t, 1.0))
    rank = torch.arange(V, device=DEV)[None, :]
    k = s["top_k"][:, None]
    keep = (rank < k) | (k <= 0)
    w = w * keep
    before = torch.cumsum(w, dim=1) - w
    p = s["top_p"].double()[:, None]
    keep &= (before < p * w.sum(dim=1, keepdim=True)) | (p >= 1)
    keep &= w >= s["min_p"].double()[:, None]
    keep = torch.where(t > 0, keep, rank == 0) | (rank == 0)
    kept = torch.zeros_like(w).scatter_(1, index, w * keep)
    run = torch.cumsum(kept, dim=1)
    passed = (run <= s["u"].double()[:, None] * run[:, -1:]).sum(dim=1)
    last = (kept > 0).mul(rank).amax(dim=1)
    return torch.minimum(passed, last).to(torch.int32)


_OWN = {"append": _own_append, "read": _own_read, "attn": _own_attn, "sample": _own_sample}
_PLAIN = {"append": _plain_append, "read": _plain_read, "attn": _plain_attn, "sample": _plain_sample}


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "sample":
        n = case["batch"] * case["vocab"]
        return {"bytes": n * (2 if case["type"] == "bf16" else 4) + 24 * case["batch"], "flops": 4 * n}
    q_lens, kv_lens = _lengths(case)
    T, H, Hk, D = sum(q_lens), case["heads"], case["kv_heads"], case["dim"]
    held = 2 * Hk * (D * case["bits"] // 8 + (2 if case["bits"] == 8 else 4))   # of a cached token
    if case["op"] == "read":
        return {"bytes": T * (held + 4 * Hk * D), "flops": 2 * T * Hk * D}
    if case["op"] == "append":   # the projection in, queries and codes out; the codes in again, their values out
        return {"bytes": T * (2 * (H + 2 * Hk) * D + 4 * D + 2 * H * D + 2 * held + 4 * Hk * D), "flops": T * D * (3 * (H + Hk) + 8 * Hk)}
    pairs = sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(q_lens, kv_lens))
    return {"bytes": 4 * T * H * D + held * sum(kv_lens), "flops": 4 * pairs * H * D}


# ------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    with torch.no_grad():
        return _EXACT[case["op"]](case, prepare(case, seed))


def _spans(s):
    cu, kv = s["cu_q"].tolist(), s["kv_len"].tolist()
    return [(b, cu[b], cu[b + 1], kv[b] - (cu[b + 1] - cu[b]), kv[b]) for b in range(len(kv))]


def _decoded(case, s, side, b, end):
    """Request b's first `end` cached tokens of one side, [Hk][end][D] in 64 bits."""
    pages = s["table"][b, : -(-end // case["page"])].long()
    codes = torch.cat(list(s["cache"][side][pages].unbind(0)), dim=1)[:, :end]
    scales = torch.cat(list(s["cache"][2 + side][pages].unbind(0)), dim=1)[:, :end].double()
    if case["bits"] == 8:
        return torch.einsum("htd,ht->htd", codes.double(), scales)
    nibbles = torch.stack([codes.bitwise_right_shift(4 * i).bitwise_and(15) for i in range(8)], dim=-1).reshape(*codes.shape[:2], -1)
    return torch.einsum("htd,ht->htd", nibbles.double() - scales[..., 1:], scales[..., 0])


def _exact_read(case, s):
    outs = []
    for side in range(2):
        outs.append(torch.cat([_decoded(case, s, side, b, end)[:, before:].transpose(0, 1) for b, _, _, before, end in _spans(s)]))
    return outs


def _levels(x, bits):
    """64-bit heads as the values of their nearest levels (the scale itself is held in bf16)."""
    if bits == 8:
        step = (x.abs().max(-1, keepdim=True).values / 127).to(torch.bfloat16).double()
        return torch.round(x / step).clamp(-128, 127) * step
    low, high = x.min(-1, keepdim=True).values.clamp(max=0), x.max(-1, keepdim=True).values.clamp(min=0)
    step = ((high - low) / 15).to(torch.bfloat16).double()
    zero = torch.round(-low / step).clamp(0, 15)
    return ((torch.round(x / step) + zero).clamp(0, 15) - zero) * step


def _exact_append(case, s):
    H, Hk, half = case["heads"], case["kv_heads"], case["dim"] // 2
    x = torch.view_as_complex(s["qkv"].double().view(-1, H + 2 * Hk, 2, half).transpose(2, 3).contiguous())
    wave = torch.complex(s["cos_sin"][:, :half].double(), s["cos_sin"][:, half:].double())
    join = lambda z: torch.cat([z.real, z.imag], dim=-1)  # noqa: E731
    turned = torch.cat([join(x[lo:hi, : H + Hk] * wave[before:end, None]) for _, lo, hi, before, end in _spans(s)])
    return [turned[:, :H], _levels(turned[:, H:], case["bits"]), _levels(join(x[:, H + Hk:]), case["bits"])]


def _exact_attn(case, s):
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    out = torch.zeros(s["tokens"], H, D, dtype=torch.float64, device=DEV)
    for b, lo, hi, before, end in _spans(s):
        k, v = (_decoded(case, s, side, b, end) for side in range(2))
        seen = torch.arange(end, device=DEV)[None, :] <= torch.arange(before, end, device=DEV)[:, None]
        for h in range(H):
            w = torch.einsum("id,jd->ij", s["q"][lo:hi, h].double(), k[h * Hk // H]) * s["scale"]
            w = torch.softmax(torch.where(seen, w, torch.full_like(w, -math.inf)), dim=1)
            out[lo:hi, h] = w @ v[h * Hk // H]
    return out


def _exact_sample(case, s):
    """Row by row on the host, with sums of the lowest rounding error (math.fsum) where they decide."""
    tokens = []
    for b in range(case["batch"]):
        x = s["logits"][b].double().cpu().numpy()
        t, k, p, least, u = (float(s[n][b]) for n in ("temperature", "top_k", "top_p", "min_p", "u"))
        if not t > 0:
            tokens.append(int(np.argmax(x)))
            continue
        order = np.lexsort((np.arange(len(x)), -x))
        order = order[: int(k)] if k > 0 else order
        w = np.exp((x[order] - x[order[0]]) / t)
        if p < 1:
            goal = p * math.fsum(w)
            order = order[: max(1, int(np.searchsorted(np.concatenate([[0.0], np.cumsum(w)[:-1]]), goal, side="left")))]
            w = w[: len(order)]
        order, w = order[w >= least], w[w >= least]
        index = np.sort(order)
        w = np.exp((x[index] - x.max()) / t)
        tokens.append(int(index[min(len(index) - 1, int(np.searchsorted(np.cumsum(w), u * math.fsum(w), side="right")))]))
    return torch.tensor(tokens, dtype=torch.int32)


_EXACT = {"append": _exact_append, "read": _exact_read, "attn": _exact_attn, "sample": _exact_sample}
