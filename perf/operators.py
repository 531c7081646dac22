"""Operators of a serving step around the quantised linears, as cases that can be timed and compared.

The decoder layer of the Llama-2-7B backbone (hidden size 4096, 32 heads of 128, a gated MLP of 11008) needs, next to its
low-bit linears: the residual addition with the root-mean-square norm (bf16, or the int8 codes the W8A8 linear reads), the
rotary embedding that appends keys and values to a paged cache, the attention of each request's new tokens over that
cache, and the low-rank adapters of many requests beside a shared projection.

A case is a dict of plain values; ``prepare`` makes what a serving program has in hand, ``run`` is one call of the
operator, ``exact`` the same result from the definition in 64 bits.  With ``own`` false ``run`` computes the plain form
in elementary torch operations (fp32, rounded once at the end); with ``own`` true it calls this library.
"""
import math
import random

import numpy as np
import torch

own = False

EPS = 1e-5
THETA = 10000.0
DEV = "cuda"


# ------------------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decode step of one robot: a single token's residual row, norm and int8 codes for a W8A8 projection
        {"name": "norm_a8_decode_1", "op": "norm", "M": 1, "K": 4096, "a8": True, "residual": True},
        # the prompt of the policy (256 vision patches and 24 text tokens), bf16 output for a weight-only projection
        {"name": "norm_prompt_280", "op": "norm", "M": 280, "K": 4096, "a8": False, "residual": True},
        # many prompts stacked for throughput, int8 output
        {"name": "norm_a8_batch_8192", "op": "norm", "M": 8192, "K": 4096, "a8": True, "residual": True},
        # 32 requests in their decode phase, right after the 280-token prompt, one new token each
        {"name": "rope_decode_32", "op": "rope", "batch": 32, "mode": "decode", "q_len": 1, "kv_len": 287, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 16},
        # seven prompts of different lengths, packed one after another
        {"name": "rope_prompts_7", "op": "rope", "batch": 7, "mode": "prompt", "q_len": 1111, "kv_len": 1111, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 64},
        # one robot's action token over its own short context: latency
        {"name": "attn_decode_1", "op": "attn", "batch": 1, "mode": "decode", "q_len": 1, "kv_len": 287, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 16},
        # a full decode batch with contexts of different lengths: bandwidth
        {"name": "attn_decode_32", "op": "attn", "batch": 32, "mode": "decode", "q_len": 1, "kv_len": 4099, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 64},
        # the 280-token prompts of four requests
        {"name": "attn_prompt_280", "op": "attn", "batch": 4, "mode": "uniform", "q_len": 280, "kv_len": 280, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 16},
        # continuous batching: one request's chunk of 512 new tokens next to 15 single tokens, grouped heads
        {"name": "attn_mixed_gqa", "op": "attn", "batch": 16, "mode": "mixed", "q_len": 512, "kv_len": 6001, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 64},
        # a long prompt taken in chunks: the second 4096 tokens over a cache of 8192
        {"name": "attn_chunk_4096", "op": "attn", "batch": 1, "mode": "uniform", "q_len": 4096, "kv_len": 8192, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 64},
        # 32 decoding requests that share 12 task adapters of rank 16 on a square projection (some have none)
        {"name": "lora_decode_32", "op": "lora", "batch": 32, "mode": "decode", "q_len": 1, "K": 4096, "N": 4096, "rank": 16,
         "adapters": 12},
        # nine prompts of different lengths, adapters of rank 32 beside the gate projection
        {"name": "lora_prompts_9", "op": "lora", "batch": 9, "mode": "prompt", "q_len": 700, "K": 4096, "N": 11008, "rank": 32,
         "adapters": 6},
    ]


def _log_int(rng, lo, hi):
    """A whole number spread over the logarithm of its range; no multiple of 1024, as lengths in service hardly ever are."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n - (n % 1024 == 0)


def _odd_width(rng, lo, hi):
    """An odd multiple of 8: a width that no tile divides."""
    return 8 * (2 * rng.randint(lo // 16, hi // 16) + 1)


def draw(rng):
    op = rng.choice(["norm", "rope", "attn", "attn", "lora"])
    if op == "norm":
        K = rng.choice([4096, 11008, 2176, _odd_width(rng, 512, 5120)])
        return {"op": op, "M": _log_int(rng, 1, 8192 * 4096 // max(K, 4096)), "K": K, "a8": rng.random() < 0.5,
                "residual": rng.random() < 0.8}
    if op == "lora":
        mode = rng.choice(["decode", "prompt"])
        return {"op": op, "batch": _log_int(rng, 1, 64) if mode == "decode" else rng.randint(1, 12), "mode": mode,
                "q_len": 1 if mode == "decode" else _log_int(rng, 5, 500), "K": rng.choice([4096, 11008, _odd_width(rng, 512, 5120)]),
                "N": rng.choice([4096, 12288, _odd_width(rng, 512, 8000)]), "rank": rng.choice([8, 16, 32, 64]),
                "adapters": rng.randint(1, 16)}
    heads, kv_heads, dim = rng.choice([(32, 32, 128), (32, 8, 128), (28, 4, 128), (16, 16, 64), (32, 4, 64), (12, 4, 64)])
    page = rng.choice([16, 32, 64, 128])
    if op == "rope":
        mode = rng.choice(["decode", "prompt"])
        q_len = 1 if mode == "decode" else _log_int(rng, 3, 1000)
        return {"op": op, "batch": _log_int(rng, 1, 48) if mode == "decode" else rng.randint(1, 8), "mode": mode, "q_len": q_len,
                "kv_len": rng.randint(q_len, 400) if mode == "decode" else q_len, "heads": heads, "kv_heads": kv_heads, "dim": dim,
                "page": page}
    mode = rng.choice(["decode", "prompt", "uniform", "mixed", "ragged"])
    batch = {"decode": _log_int(rng, 1, 48), "mixed": rng.randint(2, 24)}.get(mode, rng.randint(1, 6))
    if mode == "decode":
        q_len, kv_len = 1, _log_int(rng, 16, 4096)
    else:
        q_len = _log_int(rng, 5, 1500)
        kv_len = q_len if mode == "prompt" else q_len + _log_int(rng, 1, 4000)
        kv_len -= kv_len > q_len and kv_len % 1024 == 0
    while batch > 1 and (batch * heads * q_len * kv_len > 1_000_000_000 or batch * kv_len > 80_000):
        batch -= 1
    return {"op": op, "batch": batch, "mode": mode, "q_len": q_len, "kv_len": kv_len, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "page": page}


def _lengths(case):
    """(new tokens, cached tokens with them) of each request: the case's own numbers decide, not the seed."""
    r = random.Random("%d %s %d %d" % (case["batch"], case["mode"], case["q_len"], case.get("kv_len", 0)))
    q_len, kv_len, rest = case["q_len"], case.get("kv_len", case["q_len"]), case["batch"] - 1
    if case["mode"] == "decode":
        return [1] * (rest + 1), [kv_len] + [r.randint(max(1, kv_len // 4), kv_len) for _ in range(rest)]
    if case["mode"] == "uniform":
        return [q_len] * (rest + 1), [kv_len] * (rest + 1)
    if case["mode"] == "mixed":
        return [q_len] + [1] * rest, [kv_len] + [r.randint(1, kv_len) for _ in range(rest)]
    q = [q_len] + [r.randint(max(1, q_len // 5), q_len) for _ in range(rest)]
    if case["mode"] == "prompt":
        return q, list(q)
    return q, [kv_len] + [n + r.randint(0, kv_len - q_len) for n in q[1:]]


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
    """Lengths, block table (pages in no order) and the two caches."""
    q_lens, kv_lens = _lengths(case)
    page = case["page"]
    per_seq = [-(-n // page) for n in kv_lens]
    width, total = max(per_seq), sum(per_seq)
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    first = _ints(_starts(per_seq)[:-1].tolist())
    column = torch.arange(width, device=DEV, dtype=torch.int32)
    used = column[None, :] < _ints(per_seq)[:, None]
    table = torch.where(used, order[(first[:, None] + column).clamp(max=total - 1).long()], 0).to(torch.int32).contiguous()
    shape = (total, case["kv_heads"], page, case["dim"])
    return {"cu_q": _ints(_starts(q_lens).tolist()), "kv_len": _ints(kv_lens), "table": table, "k_cache": _normal(g, *shape),
            "v_cache": _normal(g, *shape), "max_q": max(q_lens), "max_kv": max(kv_lens), "tokens": sum(q_lens)}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": case, "op": case["op"]}
    if case["op"] == "norm":
        M, K = case["M"], case["K"]
        s["x"] = _normal(g, M, K)
        s["residual"] = _normal(g, M, K, std=2.0) if case["residual"] else None
        s["weight"] = (1.0 + 0.2 * _normal(g, K, dtype=torch.float32)).to(torch.bfloat16)
        if case["a8"]:
            s["values"] = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    elif case["op"] == "rope":
        s.update(_paged(case, g))
        s["qkv"] = _normal(g, s["tokens"], (case["heads"] + 2 * case["kv_heads"]) * case["dim"])
        half = case["dim"] // 2
        angle = np.outer(np.arange(s["max_kv"], dtype=np.float64), THETA ** (-np.arange(half, dtype=np.float64) / half))
        s["cos_sin"] = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], axis=1)).to(torch.float32).to(DEV)
    elif case["op"] == "attn":
        s.update(_paged(case, g))
        s["q"] = _normal(g, s["tokens"], case["heads"], case["dim"])
        s["scale"] = case["dim"] ** -0.5
        s["workspace"] = None
    else:
        q_lens, _ = _lengths(case)
        K, N, r, n = case["K"], case["N"], case["rank"], case["adapters"]
        M = sum(q_lens)
        s["cu_q"] = _ints(_starts(q_lens).tolist())
        s["x"] = _normal(g, M, K)
        s["a"] = _normal(g, n, r, K, std=K ** -0.5)
        s["b"] = _normal(g, n, N, r, std=r ** -0.5)
        s["y"] = _normal(g, M, N)
        s["out"] = torch.empty_like(s["y"])
        s["scales"] = 0.5 + torch.rand(n, generator=g, device=DEV)
        # one request in eight or so has no adapter (-1)
        pick = torch.randint(0, 8 * n, (case["batch"],), generator=g, device=DEV)
        s["adapter"] = torch.where(pick < n, -1, pick % n).to(torch.int32)
        s["workspace"] = None
    return s


# ------------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------------
def run(state):
    return _OWN[state["op"]](state) if own else _PLAIN[state["op"]](state)


def _own_norm(s):
    from paper_2412_01034_b200 import api
    if s["case"]["a8"]:
        codes, scales, *h = api.rmsnorm_a8(s["x"], s["weight"], EPS, residual=s["residual"])
        # the values that the codes stand for
        return [torch.mul(codes, scales[:, None], out=s["values"]), *h]
    y = api.rmsnorm(s["x"], s["weight"], EPS, residual=s["residual"])
    return list(y) if isinstance(y, tuple) else [y]


def _own_rope(s):
    from paper_2412_01034_b200 import api
    q = api.rope_append(s["qkv"], s["cos_sin"], s["k_cache"], s["v_cache"], s["cu_q"], s["kv_len"], s["table"], s["case"]["heads"])
    return [q, s["k_cache"], s["v_cache"]]


def _own_attn(s):
    from paper_2412_01034_b200 import api
    if s["workspace"] is None:
        s["workspace"] = api.new_workspace(api.attn_paged_workspace_size(s["tokens"], s["case"]["batch"], s["case"]["heads"],
                                                                         s["case"]["kv_heads"], s["case"]["dim"], s["max_q"], s["max_kv"]))
    return api.attn_paged(s["q"], s["k_cache"], s["v_cache"], s["cu_q"], s["kv_len"], s["table"], s["max_q"], s["max_kv"],
                          scale=s["scale"], workspace=s["workspace"])


def _own_lora(s):
    from paper_2412_01034_b200 import api
    if s["workspace"] is None:
        s["workspace"] = api.new_workspace(api.lora_batch_workspace_size(s["x"].shape[0], s["case"]["batch"], s["case"]["rank"]))
    return api.lora_batch_add(s["x"], s["a"], s["b"], s["y"], s["cu_q"], s["adapter"], s["scales"], out=s["out"],
                              workspace=s["workspace"])


def _plain_norm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS) * s["weight"].float()
    out = [] if s["residual"] is None else [h.to(torch.bfloat16)]
    if not s["case"]["a8"]:
        return [y.to(torch.bfloat16)] + out
    scale = y.abs().amax(dim=1, keepdim=True) / 127.0
    scale = torch.where(scale == 0, 1.0, scale)
    return [(torch.round(y / scale).clamp(-128, 127) * scale).to(torch.bfloat16)] + out


def _positions(s):
    """Request and cache position of every new token."""
    t = torch.arange(s["tokens"], device=DEV)
    seq = (t[:, None] >= s["cu_q"][1:][None, :]).sum(dim=1)
    cu = s["cu_q"].long()
    return seq, s["kv_len"].long()[seq] - (cu[1:] - cu[:-1])[seq] + t - cu[:-1][seq]


def _plain_rope(s):
    c = s["case"]
    seq, pos = _positions(s)
    half = c["dim"] // 2
    x = s["qkv"].view(s["tokens"], -1, c["dim"])
    cos, sin = s["cos_sin"][pos, None, :half], s["cos_sin"][pos, None, half:]
    first, second = x[:, : c["heads"] + c["kv_heads"], :half].float(), x[:, : c["heads"] + c["kv_heads"], half:].float()
    turned = torch.cat([first * cos - second * sin, second * cos + first * sin], dim=2).to(torch.bfloat16)
    page, slot = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    s["k_cache"][page, :, slot] = turned[:, c["heads"]:]
    s["v_cache"][page, :, slot] = x[:, c["heads"] + c["kv_heads"]:]
    return [turned[:, : c["heads"]].contiguous(), s["k_cache"], s["v_cache"]]


def _plain_attn(s):
    c = s["case"]
    B, D, H, G = c["batch"], c["dim"], c["kv_heads"], c["heads"] // c["kv_heads"]
    seq, pos = _positions(s)
    col = torch.arange(s["tokens"], device=DEV) - s["cu_q"].long()[seq]
    q = torch.zeros(B, s["max_q"], H, G, D, device=DEV)
    q[seq, col] = s["q"].view(s["tokens"], H, G, D).float() * s["scale"]
    at = torch.full((B, s["max_q"]), -1, device=DEV, dtype=torch.long)
    at[seq, col] = pos
    keys, values = (s[n][s["table"].long()].transpose(2, 3).reshape(B, -1, H, D).float() for n in ("k_cache", "v_cache"))
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


def _plain_lora(s):
    M, n = s["x"].shape[0], s["a"].shape[0]
    t = torch.arange(M, device=DEV)
    mine = s["adapter"].long()[(t[:, None] >= s["cu_q"][1:][None, :]).sum(dim=1)]
    # every token against every adapter's down projection, its own kept: [M][adapters * rank]
    down = s["x"].float() @ s["a"].float().view(-1, s["a"].shape[2]).t()
    kept = (mine[:, None] == torch.arange(n, device=DEV)[None, :]).float() * s["scales"][None, :]
    down = (down.view(M, n, -1) * kept[:, :, None]).view(M, -1)
    up = s["b"].float().permute(0, 2, 1).reshape(-1, s["b"].shape[1])
    return (s["y"].float() + down @ up).to(torch.bfloat16)


_OWN = {"norm": _own_norm, "rope": _own_rope, "attn": _own_attn, "lora": _own_lora}
_PLAIN = {"norm": _plain_norm, "rope": _plain_rope, "attn": _plain_attn, "lora": _plain_lora}


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "norm":
        M, K = case["M"], case["K"]
        moved = 2 * M * K * (3 if case["residual"] else 1) + 2 * K + (M * K + 4 * M if case["a8"] else 2 * M * K)
        return {"bytes": moved, "flops": 6 * M * K}
    q_lens, kv_lens = _lengths(case)
    T = sum(q_lens)
    if case["op"] == "lora":
        K, N, r = case["K"], case["N"], case["rank"]
        held = min(case["adapters"], case["batch"])
        return {"bytes": 2 * T * K + 4 * T * N + 2 * held * r * (K + N), "flops": 2 * T * r * (K + N)}
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rope":
        return {"bytes": 4 * T * (H + 2 * Hk) * D + 4 * T * D, "flops": 3 * T * (H + Hk) * D}
    pairs = sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(q_lens, kv_lens))
    return {"bytes": 4 * T * H * D + 4 * sum(kv_lens) * Hk * D, "flops": 4 * pairs * H * D}


# ------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    with torch.no_grad():
        return _EXACT[case["op"]](case, prepare(case, seed))


def _exact_norm(case, s):
    outs, sums = [], []
    for lo in range(0, case["M"], 1024):
        h = s["x"][lo:lo + 1024].double()
        if case["residual"]:
            h = torch.add(h, s["residual"][lo:lo + 1024].double())
            sums.append(h)
        y = torch.einsum("mk,m,k->mk", h, (h.pow(2).sum(1) / case["K"] + EPS).pow(-0.5), s["weight"].double())
        if case["a8"]:
            step = y.abs().max(1, keepdim=True).values / 127
            y = torch.where(step > 0, torch.round(y / step).clamp(-128, 127) * step, torch.zeros_like(y))
        outs.append(y)
    return [torch.cat(outs)] + ([torch.cat(sums)] if sums else [])


def _spans(s):
    cu, kv = s["cu_q"].tolist(), s["kv_len"].tolist()
    return [(b, cu[b], cu[b + 1], kv[b] - (cu[b + 1] - cu[b]), kv[b]) for b in range(len(kv))]


def _exact_rope(case, s):
    H, Hk, D, half = case["heads"], case["kv_heads"], case["dim"], case["dim"] // 2
    x = torch.view_as_complex(s["qkv"].double().view(-1, H + 2 * Hk, 2, half).transpose(2, 3).contiguous())
    wave = torch.complex(s["cos_sin"][:, :half].double(), s["cos_sin"][:, half:].double())
    q = torch.empty(x.shape[0], H, D, dtype=torch.float64, device=DEV)
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    join = lambda z: torch.cat([z.real, z.imag], dim=-1)  # noqa: E731
    for b, lo, hi, before, end in _spans(s):
        turned = x[lo:hi, : H + Hk] * wave[before:end, None]
        q[lo:hi] = join(turned[:, :H])
        where = torch.arange(before, end, device=DEV)
        pages, slots = s["table"][b].long()[where.div(case["page"], rounding_mode="floor")], where.remainder(case["page"])
        k_cache[pages, :, slots] = join(turned[:, H:])
        v_cache[pages, :, slots] = join(x[lo:hi, H + Hk:])
    return [q, k_cache, v_cache]


def _exact_attn(case, s):
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    out = torch.zeros(s["tokens"], H, D, dtype=torch.float64, device=DEV)
    for b, lo, hi, before, end in _spans(s):
        if hi == lo:
            continue
        pages = s["table"][b, : -(-end // case["page"])].long()
        k, v = (torch.cat(list(s[n][pages].unbind(0)), dim=1)[:, :end].double() for n in ("k_cache", "v_cache"))
        seen = torch.arange(end, device=DEV)[None, :] <= torch.arange(before, end, device=DEV)[:, None]
        for h in range(H):
            w = torch.einsum("id,jd->ij", s["q"][lo:hi, h].double(), k[h * Hk // H]) * s["scale"]
            w = torch.where(seen, w, torch.full_like(w, -math.inf))
            w = torch.softmax(w, dim=1)
            out[lo:hi, h] = w @ v[h * Hk // H]
    return out


def _exact_lora(case, s):
    out = s["y"].double()
    cu, mine = s["cu_q"].tolist(), s["adapter"].tolist()
    for b, a in enumerate(mine):
        if a >= 0:
            lo, hi = cu[b], cu[b + 1]
            out[lo:hi] += s["scales"][a].double() * ((s["x"][lo:hi].double() @ s["a"][a].double().t()) @ s["b"][a].double().t())
    return out


_EXACT = {"norm": _exact_norm, "rope": _exact_rope, "attn": _exact_attn, "lora": _exact_lora}
