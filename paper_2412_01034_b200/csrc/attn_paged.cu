// Attention of the new tokens of many requests over a paged cache, causal, grouped heads: which kernel takes which
// requests, and how the work is split.
//   request b: q_len new tokens (rows cu_q[b] ... cu_q[b+1] of q), kv_len cached tokens with the new ones among them
//   new token i of a request has position p = kv_len - q_len + i and sees the cached tokens j <= p
//   o = sum_j softmax_j(scale q . k_j) v_j;  a token that sees nothing (p < 0) gets zeros
// The lengths are on the device; the host knows their bounds.  Requests of at most 16 query rows per key head go to
// attn_few.cu, the others to attn_many.cu; a launch is left out where the bounds show that it would find nothing.
#include "attn_paged.cuh"

namespace qil {

namespace {

// The counters lie in the same place whatever the call's sizes are: they have to be zero between launches, and the parts of
// one call must not lie where another call that shares the workspace has its counters.
constexpr long long kCounters = 16384;

struct AttnPlan {
    bool few, many, together;
    int chunk, slots, few_rows, splits;
    size_t few_floats, many_floats;
};

AttnPlan plan_attn(int total_q, int num_seqs, int H, int Hk, int D, int max_q, int max_kv) {
    AttnPlan pl = {};
    const int G = H / Hk;
    const long long sms = num_sms();
    if (max_q > total_q) max_q = total_q;
    pl.many = (long long)max_q * G > kFewRows;
    // Every request has more than kFewRows rows if the others at their longest leave more for it.  (More than max_q left says
    // that the bound is wrong, and nothing about any one request.)
    const long long least = (long long)total_q - (long long)(num_seqs - 1) * max_q;
    pl.few = least * G <= kFewRows || least > max_q;
    if (pl.few) {
        // Two blocks fit an SM, and one round of blocks is best: each of 2048 tokens at most (the requests' lengths differ).
        // Where it gives a row of the cache (a request and key head) at least two blocks, up to eight of 128 tokens or more
        // are a cluster and join their results on the chip; one token over 500, 32 heads: 5.3 us (7.8 with blocks of 384),
        // over 1500: 7.6, over 4000: 10.9 (14.4 with parts in the workspace).  Eight blocks that would take more than 1024
        // tokens each give way to more, of 384 at least (a part's way through the workspace costs as much as 300 tokens).
        const long long items = (long long)num_seqs * Hk, room = 2 * sms, per_row = room / items;
        const auto round64 = [](long long n) { return (n + 63) / 64 * 64; };
        long long chunk = round64((max_kv * items + room - 1) / room);
        chunk = chunk < 384 ? 384 : chunk > 2048 ? 2048 : chunk;
        if (per_row >= 2) {
            const long long most = per_row < kMostTogether ? per_row : kMostTogether;
            const long long of = round64((max_kv + most - 1) / most), mine = of < 128 ? 128 : of;
            if (mine <= (per_row > kMostTogether ? 1024 : 2048)) {
                chunk = mine;
                pl.together = max_kv > chunk;
            }
        }
        if (items > kCounters) chunk = max_kv;   // (rows enough to fill the GPU many times over: one block each)
        pl.chunk = (int)chunk;
        pl.slots = (int)((max_kv + chunk - 1) / chunk);
        const long long rows = (long long)max_q * G;
        pl.few_rows = (int)(rows < kFewRows ? rows : kFewRows);
        if (pl.slots > 1 && !pl.together) pl.few_floats = ((size_t)items * pl.slots * pl.few_rows * (D + 2) + 3) & ~(size_t)3;   // (16-byte stores behind them)
    }
    if (pl.many) {
        // The cache is split where the row tiles alone leave SMs idle, into parts of at least four tiles of 128 tokens.  The
        // bounds give the least number of row tiles: all rows packed, or one tile for every request that has to be here.
        const long long few = kFewRows / G, here = max_q > few ? (total_q - num_seqs * few + max_q - few - 1) / (max_q - few) : 0;
        long long tiles = ((long long)total_q * G + 255) / 256;
        if (tiles < here) tiles = here;
        long long s = sms / (tiles * Hk);
        if (s > (max_kv + 511LL) / 512) s = (max_kv + 511LL) / 512;
        pl.splits = s < 1 ? 1 : (int)s;
        if (pl.splits > 1) pl.many_floats = (size_t)pl.splits * total_q * H * (D + 2);
    }
    return pl;
}

constexpr size_t kHeader = 256;   // status word
static_assert(kHeader + kCounters * sizeof(int) == QIL_ATTN_PAGED_ZEROED_BYTES, "what has to be zero before the first call");

}  // namespace

size_t attn_paged_workspace(int total_q, int num_seqs, int num_heads, int num_kv_heads, int head_dim, int max_q_len, int max_kv_len) {
    const AttnPlan pl = plan_attn(total_q, num_seqs, num_heads, num_kv_heads, head_dim, max_q_len, max_kv_len);
    return kHeader + kCounters * sizeof(int) + (pl.few_floats + pl.many_floats) * sizeof(float);
}

qil_status launch_attn_paged(const void* q, const void* k_cache, const void* v_cache, void* out, const PagedCache& c, int max_q_len,
                             int max_kv_len, float scale, void* ws, cudaStream_t st) {
    const AttnPlan pl = plan_attn(c.total_q, c.num_seqs, c.num_heads, c.num_kv_heads, c.head_dim, max_q_len, max_kv_len);
    AttnParams p;
    p.q = reinterpret_cast<const __nv_bfloat16*>(q);
    p.k = reinterpret_cast<const __nv_bfloat16*>(k_cache);
    p.v = reinterpret_cast<const __nv_bfloat16*>(v_cache);
    p.out = reinterpret_cast<__nv_bfloat16*>(out);
    p.c = c;
    p.G = c.num_heads / c.num_kv_heads;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.page_shift = c.page_size == 16 ? 4 : c.page_size == 32 ? 5 : c.page_size == 64 ? 6 : 7;
    p.chunk = pl.chunk;
    p.slots = pl.slots;
    p.together = pl.together;
    p.few_rows = pl.few_rows;
    p.splits = pl.splits;
    p.tile_tokens = kTileRows / p.G;
    char* base = static_cast<char*>(ws);
    p.status = reinterpret_cast<int*>(base);
    p.counters = reinterpret_cast<int*>(base + kHeader);
    p.few_parts = reinterpret_cast<float*>(base + kHeader + kCounters * sizeof(int));
    p.many_parts = p.few_parts + pl.few_floats;   // (the two kernels may run at the same time)
    p.both = pl.few && pl.many;
    qil_status s = QIL_OK;
    if (pl.many) s = launch_attn_many(p, st);
    if (s == QIL_OK && pl.few) s = launch_attn_few(p, st);
    if (s == QIL_OK && pl.many && pl.splits > 1) s = launch_attn_many_join(p, st);
    return s;
}

}  // namespace qil
