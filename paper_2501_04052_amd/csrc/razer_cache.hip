// The bookkeeping of a serving step and the encoder of the 8-bit paged key/value cache (include/razer_cache.h),
// and the argument checks of the cache's entry points.
#include "razer_cache.hpp"

namespace razer {

// ---- razer_cache_plan -------------------------------------------------------------------------------------------
//
// Two exclusive sums over the requests (new tokens, new pages) and then one independent result per token.  Bound by
// latency: a step has tens to thousands of requests and the answer is 16 bytes per token.  So it is one launch: every
// workgroup sums all requests again, 1024 at a time (a few microseconds even for thousands of them, less than a
// second launch), up to the one that holds its last token, and then writes its own 1024 tokens.  The first workgroup
// also writes what there is per request.  A table entry is written by the token that begins the page.
constexpr int kPlanThreads = 1024;

__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(
    const int32_t* __restrict__ lens, const int32_t* __restrict__ fresh, int requests, int32_t* __restrict__ table, int width,
    int64_t ld_table, const int32_t* __restrict__ free_pages, int free_count, int lp, int64_t tokens, int32_t* __restrict__ cu,
    int32_t* __restrict__ total, int64_t* __restrict__ slots, int32_t* __restrict__ positions, int32_t* __restrict__ request_of,
    int32_t* __restrict__ used)
{
    __shared__ int s_cu[kPlanThreads], s_len[kPlanThreads], s_take[kPlanThreads];
    __shared__ int s_sum[2][kPlanThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool first = blockIdx.x == 0;
    const int64_t t0 = (int64_t)blockIdx.x * kPlanThreads, t = t0 + tid;
    const int page = 1 << lp;
    int base_new = 0, base_pages = 0;
    bool found = t >= tokens;
    for (int c = 0; c < requests; c += kPlanThreads) {
        const int r = c + tid;
        const int len = r < requests ? max(lens[r], 0) : 0, n = r < requests ? max(fresh[r], 0) : 0;
        const int had = (int)(((int64_t)len + page - 1) >> lp), want = (int)(((int64_t)len + n + page - 1) >> lp);
        int sn = n, sp = want - had;                                     // inclusive sums within the wave
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int a = __shfl_up(sn, d), b = __shfl_up(sp, d);
            if (lane >= d) { sn += a; sp += b; }
        }
        if (lane == 63) { s_sum[0][wave] = sn; s_sum[1][wave] = sp; }
        __syncthreads();
        int on = base_new, op = base_pages;
#pragma unroll
        for (int w = 0; w < kPlanThreads / 64; ++w) {
            const int a = s_sum[0][w], b = s_sum[1][w];
            if (w < wave) { on += a; op += b; }
            base_new += a;
            base_pages += b;
        }
        s_cu[tid] = on + sn - n;
        s_len[tid] = len;
        s_take[tid] = op + sp - (want - had) - had;                      // + page index = place in the list
        if (first && r < requests) {
            cu[r] = on + sn - n;
            total[r] = len + n;
        }
        __syncthreads();
        if (!found && t < base_new) {                                    // the last request of the chunk with cu <= t
            int lo = 0, hi = min(kPlanThreads, requests - c);
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_cu[mid] <= t) lo = mid; else hi = mid;
            }
            const int pos = s_len[lo] + (int)(t - s_cu[lo]), col = pos >> lp;
            const int64_t row = (int64_t)(c + lo) * ld_table;
            int pg = -1;
            if (col >= 0 && col < width) {
                if (col < ((s_len[lo] + page - 1) >> lp)) {
                    pg = table[row + col];
                } else {
                    const int i = s_take[lo] + col;
                    if (i >= 0 && i < free_count) pg = free_pages[i];
                    if ((pos & (page - 1)) == 0) table[row + col] = pg;
                }
            }
            slots[t] = pg < 0 ? -1 : ((int64_t)pg << lp) + (pos & (page - 1));
            if (positions) positions[t] = pos;
            if (request_of) request_of[t] = c + lo;
            found = true;
        }
        if (!first && base_new >= t0 + kPlanThreads) return;             // (uniform: every thread has the same sums)
        __syncthreads();                                                 // the chunk's arrays are written again
    }
    if (!found) {
        slots[t] = -1;
        if (positions) positions[t] = 0;
        if (request_of) request_of[t] = -1;
    }
    if (first && tid == 0) {
        cu[requests] = base_new;
        *used = base_pages;
    }
}

hipError_t launch_cache_plan(const int32_t* lens, const int32_t* fresh, int requests, int32_t* table, int width, int64_t ld_table,
                             const int32_t* free_pages, int free_count, int lp, int64_t tokens, int32_t* cu, int32_t* total,
                             int64_t* slots, int32_t* positions, int32_t* request_of, int32_t* used, hipStream_t st)
{
    const unsigned grid = tokens <= kPlanThreads ? 1u : (unsigned)((tokens + kPlanThreads - 1) / kPlanThreads);
    launch(cache_plan_kernel, grid, kPlanThreads, 0, st, lens, fresh, requests, table, width, ld_table, free_pages, free_count, lp,
           tokens, cu, total, slots, positions, request_of, used);
    return hipGetLastError();
}

// ---- razer_cache_append -----------------------------------------------------------------------------------------
//
// One workgroup per run of new tokens that share a page, per head, for the keys or for the values: absolute maximum,
// exponent byte, the page's earlier codes moved if the byte grew, new codes.  The inputs are read twice (the second
// time from the caches).  Values go through LDS, since their page has the tokens of one element side by side.
constexpr int kAppendThreads = 256;

__device__ __forceinline__ float load_elt(const float* p) { return *p; }
__device__ __forceinline__ float load_elt(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

// smallest b with a <= 448 * 2^(b-127) (448 = 1.75 * 2^8)
__device__ __forceinline__ int exponent_of(float a)
{
    const uint32_t u = __float_as_uint(a);
    return min(max((int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u), RAZER_CACHE_MIN_EXPONENT), RAZER_CACHE_MAX_EXPONENT);
}

// two E4M3 codes, nearest even; NaN -> 0, beyond 448 -> 448
__device__ __forceinline__ uint32_t encode2(float a, float b)
{
    a = a == a ? fminf(fmaxf(a, -448.0f), 448.0f) : 0.0f;
    b = b == b ? fminf(fmaxf(b, -448.0f), 448.0f) : 0.0f;
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
}

// four codes times 2^-shift (mul = that power), nearest even; a NaN code (append writes none) becomes 0x7F
__device__ __forceinline__ uint32_t move4(uint32_t x, float mul)
{
    const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
    uint32_t y = encode2(a.x * mul, a.y * mul) | (encode2(b.x * mul, b.y * mul) << 16);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (((x >> (8 * i)) & 0x7fu) == 0x7fu) y = (y & ~(0xffu << (8 * i))) | (0x7fu << (8 * i));
    return y;
}

template <typename T>
__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(CacheView c, const T* __restrict__ k, int64_t ld_k,
                                                                      const T* __restrict__ v, int64_t ld_v, int64_t tokens,
                                                                      const int64_t* __restrict__ slots)
{
    extern __shared__ __align__(16) uint8_t tile[];                      // values: [page][dim + 4] codes
    __shared__ int s_run;
    __shared__ float s_max[kAppendThreads / 64];
    const int tid = threadIdx.x, page = 1 << c.lp, dim = c.dim;
    const int64_t t0 = blockIdx.x;
    const int head = blockIdx.y >> 1;
    const bool values = blockIdx.y & 1;
    const int64_t slot = slots[t0], pg = slot >> c.lp;
    if (slot < 0 || pg >= c.pages) return;
    const int off = (int)(slot & (page - 1));
    if (t0 > 0 && off > 0 && slots[t0 - 1] == slot - 1) return;          // not the first of its run
    if (tid == 0) s_run = page - off;
    __syncthreads();
    if (tid < page - off && !(t0 + tid < tokens && slots[t0 + tid] == slot + tid)) atomicMin(&s_run, tid);
    __syncthreads();
    const int run = s_run, count = run * dim;
    const T* x = (values ? v + t0 * ld_v : k + t0 * ld_k) + (int64_t)head * dim;
    const int64_t ld = values ? ld_v : ld_k;

    float amax = 0.0f;
    for (int i = tid; i < count; i += kAppendThreads) {
        const float a = fabsf(load_elt(x + (int64_t)(i / dim) * ld + i % dim));
        if (a < INFINITY) amax = fmaxf(amax, a);                         // (NaN compares false)
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) amax = fmaxf(amax, __shfl_xor(amax, d));
    if ((tid & 63) == 0) s_max[tid >> 6] = amax;
    __syncthreads();
    amax = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));

    uint8_t* scale = (values ? c.v_scales : c.k_scales) + pg * c.heads + head;
    uint8_t* codes = (values ? c.v_codes : c.k_codes) + (pg * c.heads + head) * (int64_t)page * dim;
    const int before = off > 0 ? min(max((int)*scale, RAZER_CACHE_MIN_EXPONENT), RAZER_CACHE_MAX_EXPONENT) : RAZER_CACHE_MIN_EXPONENT;
    const int b = max(before, exponent_of(amax));
    __syncthreads();                                                     // everybody has read the old byte
    if (tid == 0) *scale = (uint8_t)b;
    if (off > 0 && b > before) {
        const float mul = exponent_value(max(127 + before - b, 1));
        if (!values) {
            for (int i = tid; i < off * dim / 4; i += kAppendThreads) {
                uint32_t* p = reinterpret_cast<uint32_t*>(codes) + i;
                *p = move4(*p, mul);
            }
        } else {
            for (int i = tid; i < off * dim; i += kAppendThreads) {
                uint8_t* p = codes + (i / off) * page + i % off;
                *p = (uint8_t)move4(*p, mul);
            }
        }
    }
    const float inv = exponent_value(254 - b);
    if (!values) {
        for (int i = tid; i < count / 2; i += kAppendThreads) {
            const T* p = x + (int64_t)(i * 2 / dim) * ld + i * 2 % dim;
            reinterpret_cast<uint16_t*>(codes + off * dim)[i] = (uint16_t)encode2(load_elt(p) * inv, load_elt(p + 1) * inv);
        }
        return;
    }
    const int ldt = dim + 4;
    for (int i = tid; i < count / 2; i += kAppendThreads) {
        const int tok = i * 2 / dim, d = i * 2 % dim;
        const T* p = x + (int64_t)tok * ld + d;
        *reinterpret_cast<uint16_t*>(tile + tok * ldt + d) = (uint16_t)encode2(load_elt(p) * inv, load_elt(p + 1) * inv);
    }
    __syncthreads();
    for (int i = tid; i < count; i += kAppendThreads) {
        const int d = i / run, tok = i % run;
        codes[d * page + off + tok] = tile[tok * ldt + d];
    }
}

hipError_t launch_cache_append(const CacheView& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v, int bf16,
                               int64_t tokens, const int64_t* slots, hipStream_t st)
{
    if (tokens == 0) return hipSuccess;
    const dim3 grid((unsigned)tokens, (unsigned)(2 * c.heads));
    const size_t smem = (size_t)(c.dim + 4) << c.lp;
    if (bf16)
        launch(cache_append_kernel<uint16_t>, grid, kAppendThreads, smem, st, c, reinterpret_cast<const uint16_t*>(k), ld_k,
               reinterpret_cast<const uint16_t*>(v), ld_v, tokens, slots);
    else
        launch(cache_append_kernel<float>, grid, kAppendThreads, smem, st, c, reinterpret_cast<const float*>(k), ld_k,
               reinterpret_cast<const float*>(v), ld_v, tokens, slots);
    return hipGetLastError();
}

// ---- checks -----------------------------------------------------------------------------------------------------

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static bool page_log(int page, int& lp)
{
    switch (page) {
        case 16: lp = 4; return true;
        case 32: lp = 5; return true;
        case 64: lp = 6; return true;
        case 128: lp = 7; return true;
        default: return false;
    }
}

razer_status check_cache(const razer_cache* c, CacheView& o)
{
    if (!c) return RAZER_ERR_NULL;
    if (!page_log(c->page, o.lp)) return RAZER_ERR_CONFIG;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 192 && c->head_dim != 256) return RAZER_ERR_CONFIG;
    if (c->pages < 1 || c->pages > ((int64_t)1 << 31) - 1 || c->kv_heads < 1 || c->kv_heads > 16384) return RAZER_ERR_SHAPE;
    if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return RAZER_ERR_NULL;
    if (!aligned16(c->k_codes) || !aligned16(c->v_codes)) return RAZER_ERR_ALIGN;
    o.k_codes = c->k_codes;
    o.v_codes = c->v_codes;
    o.k_scales = c->k_scales;
    o.v_scales = c->v_scales;
    o.pages = c->pages;
    o.heads = c->kv_heads;
    o.dim = c->head_dim;
    return RAZER_OK;
}

static razer_status check_attention(const razer_cache* cache, const razer_attention* g, CacheView& c, AttentionArgs& a)
{
    const razer_status s = check_cache(cache, c);
    if (s != RAZER_OK) return s;
    if (!g) return RAZER_ERR_NULL;
    const int64_t row = (int64_t)g->q_heads * c.dim;
    if (g->tokens < 0 || g->requests < 0 || g->q_heads < 1 || g->q_heads % c.heads != 0 || g->table_width < 0) return RAZER_ERR_SHAPE;
    // (the grid of the smallest tiles stays below 2^24 workgroups)
    if (g->tokens > ((int64_t)1 << 27) / g->q_heads || g->requests > ((int64_t)1 << 22) / c.heads) return RAZER_ERR_SHAPE;
    if (g->ld_q < row || g->ld_out < row || g->ld_table < g->table_width) return RAZER_ERR_SHAPE;
    if (g->window < 0 || !(g->cap >= 0.0f) || !(g->cap < INFINITY) || !(g->scale == g->scale) || g->scale - g->scale != 0.0f)
        return RAZER_ERR_CONFIG;
    if (g->tokens > 0 && g->requests > 0) {
        if (!g->q || !g->out || !g->cu || !g->total || (!g->table && g->table_width > 0)) return RAZER_ERR_NULL;
        if (!aligned16(g->q) || !aligned16(g->out) || g->ld_q % 8 != 0 || g->ld_out % 8 != 0) return RAZER_ERR_ALIGN;
    }
    a.q = static_cast<const uint16_t*>(g->q);
    a.out = static_cast<uint16_t*>(g->out);
    a.ld_q = g->ld_q;
    a.ld_out = g->ld_out;
    a.tokens = (int)g->tokens;
    a.requests = g->requests;
    a.q_heads = g->q_heads;
    a.group = g->q_heads / c.heads;
    a.cu = g->cu;
    a.total = g->total;
    a.table = g->table;
    a.ld_table = g->ld_table;
    a.width = g->table_width;
    a.scale = g->scale;
    a.cap = g->cap;
    a.window = g->window;
    a.slopes = g->slopes;
    a.prefix = g->prefix;
    return RAZER_OK;
}

}  // namespace razer

using namespace razer;

extern "C" {

razer_status razer_cache_plan(const int32_t* lens, const int32_t* fresh, int32_t requests, int32_t* table, int32_t table_width,
                              int64_t ld_table, const int32_t* free_pages, int32_t free_count, int32_t page, int64_t tokens,
                              int32_t* cu, int32_t* total, int64_t* slots, int32_t* positions, int32_t* request_of,
                              int32_t* used, void* hip_stream)
{
    int lp = 0;
    if (!page_log(page, lp)) return RAZER_ERR_CONFIG;
    if (requests < 0 || table_width < 0 || ld_table < table_width || free_count < 0 || tokens < 0 || tokens >= ((int64_t)1 << 31))
        return RAZER_ERR_SHAPE;
    if (!cu || !used || (tokens > 0 && !slots)) return RAZER_ERR_NULL;
    if (requests > 0 && (!lens || !fresh || !total || (table_width > 0 && !table))) return RAZER_ERR_NULL;
    if (free_count > 0 && !free_pages) return RAZER_ERR_NULL;
    const hipError_t e = launch_cache_plan(lens, fresh, requests, table, table_width, ld_table, free_pages, free_count, lp, tokens,
                                           cu, total, slots, positions, request_of, used, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? RAZER_OK : RAZER_ERR_HIP;
}

razer_status razer_cache_append(const razer_cache* cache, const void* k, int64_t ld_k, const void* v, int64_t ld_v, int32_t dtype,
                                int64_t tokens, const int64_t* slots, void* hip_stream)
{
    CacheView c;
    const razer_status s = check_cache(cache, c);
    if (s != RAZER_OK) return s;
    if (dtype != RAZER_F32 && dtype != RAZER_BF16) return RAZER_ERR_CONFIG;
    if (tokens < 0 || tokens >= ((int64_t)1 << 24)) return RAZER_ERR_SHAPE;
    if (tokens == 0) return RAZER_OK;
    const int64_t row = (int64_t)c.heads * c.dim, per16 = dtype == RAZER_BF16 ? 8 : 4;
    if (ld_k < row || ld_v < row) return RAZER_ERR_SHAPE;
    if (!k || !v || !slots) return RAZER_ERR_NULL;
    if (!aligned16(k) || !aligned16(v) || ld_k % per16 != 0 || ld_v % per16 != 0) return RAZER_ERR_ALIGN;
    const hipError_t e = launch_cache_append(c, k, ld_k, v, ld_v, dtype == RAZER_BF16, tokens, slots, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? RAZER_OK : RAZER_ERR_HIP;
}

size_t razer_attention_workspace_bytes(const razer_cache* cache, const razer_attention* args)
{
    CacheView c;
    AttentionArgs a;
    if (check_attention(cache, args, c, a) != RAZER_OK || a.tokens == 0 || a.requests == 0) return 0;
    return attention_workspace_bytes(c, a, args->max_new, args->max_len);
}

razer_status razer_cache_attention(const razer_cache* cache, const razer_attention* args, void* workspace, size_t workspace_bytes,
                                   void* hip_stream)
{
    CacheView c;
    AttentionArgs a;
    const razer_status s = check_attention(cache, args, c, a);
    if (s != RAZER_OK) return s;
    if (a.tokens == 0 || a.requests == 0) return RAZER_OK;
    const size_t need = attention_workspace_bytes(c, a, args->max_new, args->max_len);
    if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return RAZER_ERR_WORKSPACE;
    const hipError_t e = launch_attention(c, a, args->max_new, args->max_len, static_cast<float*>(workspace),
                                          static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? RAZER_OK : RAZER_ERR_HIP;
}

}  // extern "C"
