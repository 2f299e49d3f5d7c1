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
// A run is a stretch of new tokens in consecutive slots of a page.  One workgroup takes a run and a head: waves 0 and 1 the keys,
// 2 and 3 the values; absolute maximum, exponent byte, the page's earlier codes moved if the byte grew, new codes.  Where
// tokens are skipped or slots left out, a page has several runs: the workgroup of the first takes them one after the other, so
// that a page and head have one writer.  A thread holds its first kHold pieces of 8 elements (a page of up to 2048 elements) and
// reads what is beyond them twice.
// Values pass through LDS, since their page has the tokens of one element side by side.
//
// Bound by memory with long prompts and by latency in decode steps.  Where runs begin only the slots say, so a workgroup
// looks at a window of 16 tokens and takes every `share`-th page whose first run begins there: share = 16 gives each run of a decode
// batch a workgroup of its own, but launches 16 of which one or two find work where prompts fill pages; with more than
// kAppendFew tokens, or more than kAppendFewRows tokens times heads, it is 2 (D = 128, bf16, share 16 against 2, us: single tokens, 8 heads,
// pages of 16, 64 tokens 4.8 / 14.2, 256 10.4 / 14.7, 384 14.2 / 15.6, 512 18.3 / 16.4, 1024 33.1 / 20.0; 32 heads, 64 tokens 12.1 / 16.1, 128
// 20.6 / 18.7; a prompt, 8 heads, 128 tokens 7.0 / 3.9, 512 9.4 / 3.9).  Runs of up to kFewTokens put their values byte by byte,
// without LDS and its barrier (512 requests, 8 heads, pages of 64, with against without, us: 2 tokens each 27.5 / 28.6, 4 18.6 / 19.9;
// 8 26.2 / 25.9, 16 50.3 / 43.8).
constexpr int kAppendThreads = 256, kAppendWindow = 16, kHold = 2, kAppendFew = 1024, kAppendFewRows = 3500, kFewTokens = 4;

// 8 consecutive elements of an input row
struct Eight {
    float x[8];
};
__device__ __forceinline__ Eight widen(uint4 a)
{
    Eight r;
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.x[2 * i] = __uint_as_float(w[i] << 16);
        r.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    return r;
}
struct Raw16 {
    uint4 a;
    __device__ __forceinline__ void load(const uint16_t* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ Eight get() const { return widen(a); }
};
struct Raw32 {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p)
    {
        a = reinterpret_cast<const float4*>(p)[0];
        b = reinterpret_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ Eight get() const { return Eight{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}}; }
};
template <typename T> struct RawOf;
template <> struct RawOf<uint16_t> { typedef Raw16 type; };
template <> struct RawOf<float> { typedef Raw32 type; };

// smallest b in range with a <= 448 * 2^(b-127) (448 = 1.75 * 2^8)
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
__device__ __forceinline__ uint2 encode8(const Eight& e, float inv)
{
    return make_uint2(encode2(e.x[0] * inv, e.x[1] * inv) | (encode2(e.x[2] * inv, e.x[3] * inv) << 16),
                      encode2(e.x[4] * inv, e.x[5] * inv) | (encode2(e.x[6] * inv, e.x[7] * inv) << 16));
}
__device__ __forceinline__ float absmax8(const Eight& e, float m)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = fabsf(e.x[i]);
        m = fmaxf(m, a < INFINITY ? a : 0.0f);                           // (NaN compares false)
    }
    return m;
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

__device__ __forceinline__ int64_t wave_lane(int64_t x, int i)          // of lane i (uniform)
{
    return (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, i) | (int64_t)__builtin_amdgcn_readlane((int)(x >> 32), i) << 32;
}

// the lowest bit of 3 x 64 that is set, from bit `from` on; 192: none
__device__ __forceinline__ int next_set(const uint64_t (&m)[3], int from)
{
#pragma unroll
    for (int n = 0; n < 3; ++n) {
        const int lo = max(from - 64 * n, 0);
        const uint64_t x = lo < 64 ? m[n] & (~0ull << lo) : 0;
        if (x) return 64 * n + __ffsll((unsigned long long)x) - 1;
    }
    return 192;
}

template <typename T, int D>
__global__ __launch_bounds__(kAppendThreads, 4) void cache_append_kernel(CacheView c, const T* __restrict__ k, int64_t ld_k,
                                                                      const T* __restrict__ v, int64_t ld_v, int64_t tokens,
                                                                      const int64_t* __restrict__ slots, int share)
{
    typedef typename RawOf<T>::type Raw;
    constexpr int PR = D / 8;                                            // pieces per token
    extern __shared__ __align__(16) uint8_t tile[];                      // the run's values: [tokens][D + 4]
    __shared__ float s_max[kAppendThreads / 64];
    const int tid = threadIdx.x, page = 1 << c.lp, lane = tid & 63;
    constexpr int LDT = D + 4;
    const bool values = tid >= 128;                                      // (uniform over each wave)
    const int i0 = tid & 127, head = blockIdx.x % c.heads, wi = blockIdx.x / c.heads;   // heads side by side: whole rows are read at a time
    const int64_t w0 = (int64_t)(wi / share) * kAppendWindow;
    const int64_t end = c.pages << c.lp;

    // Where runs begin in the window, and where they cannot go on: in the slots of the tokens up to a page beyond it, a lane
    // each, so that one trip to memory tells both.  Every wave sees the same.
    int64_t slot_at[3], before_at[3];
    uint64_t begins[3], stops[3], inside[3], follows[3] = {0, 0, 0};     // (inside: begins behind the place 0 of a page)
#pragma unroll
    for (int n = 0; n < 3; ++n) {
        slot_at[n] = before_at[n] = -1;
        begins[n] = inside[n] = 0;
        stops[n] = ~0ull;
        if (n > 0 && n * 64 >= kAppendWindow + page) continue;
        const int64_t t = w0 + n * 64 + lane;
        const bool in = t < tokens;
        const int64_t s = in ? slots[t] : -1, before = in && t > 0 ? slots[t - 1] : -2;
        const bool ok = s >= 0 && s < end, zero = (s & (page - 1)) == 0, first = zero || before != s - 1;
        slot_at[n] = s;
        before_at[n] = before;
        begins[n] = __ballot(ok && first);
        stops[n] = __ballot(!ok || first);
        inside[n] = __ballot(ok && first && !zero);
    }
    // A page's first run is one whose page is not that of the last token before it that is not skipped.
    if (inside[0] | inside[1] | inside[2]) {
        uint64_t apart[3];                                               // behind a skipped token
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            follows[n] = inside[n] & __ballot(((before_at[n] ^ slot_at[n]) >> c.lp) == 0);
            apart[n] = inside[n] & __ballot((before_at[n] < 0 || before_at[n] >= end) && w0 + n * 64 + lane > 0);
        }
        if (apart[0] | apart[1] | apart[2]) {
            int page_before = -1;                                        // of the chunks before
            uint64_t valid[3];
#pragma unroll
            for (int n = 0; n < 3; ++n) valid[n] = __ballot(slot_at[n] >= 0 && slot_at[n] < end);
            const int lead = __ffsll((unsigned long long)valid[0]) - 1;
            if (valid[0] && ((apart[0] >> lead) & 1))
                for (int n = 1; 64 * (n - 1) < page && w0 - 64 * (n - 1) > 0; ++n) {
                    const int64_t t = w0 - 64 * n + lane, s = t >= 0 ? slots[t] : -1;
                    const uint64_t there = __ballot(s >= 0 && s < end);
                    if (!there) continue;
                    const int last = 63 - __clzll((long long)there);
                    if (lead + 64 * n - last < page) page_before = (int)(wave_lane(s, last) >> c.lp);
                    break;
                }
#pragma unroll
            for (int n = 0; n < 3; ++n) {
                const uint64_t behind = valid[n] & ((1ull << lane) - 1);
                const int mine = (int)(slot_at[n] >> c.lp), other = __shfl(mine, behind ? 63 - __clzll((long long)behind) : 0);
                follows[n] |= apart[n] & __ballot(mine == (behind ? other : page_before));
                if (valid[n]) page_before = __builtin_amdgcn_readlane(mine, 63 - __clzll((long long)valid[n]));
            }
        }
    }
    const bool several = (follows[0] | follows[1] | follows[2]) != 0;    // runs of a page
    uint32_t mask = (uint32_t)(begins[0] & ~follows[0]) & 0xffffu;
    for (int skip = wi % share; skip > 0; --skip) mask &= mask - 1;
    if (!mask) return;
    int first = 192, reach = 0;
    for (bool again = false;; again = true) {
        if (!several || first >= reach || next_set(follows, first) != first) {   // not another run of the page at hand
            if (!mask) break;
            first = __ffs(mask) - 1;                                     // token w0 + first begins the run
            reach = first + page;
            for (int n = 0; n < share; ++n) mask &= mask - 1;
        }
        if (again) __syncthreads();                                      // the maxima and the tile are written again, the page's bytes read
        const int64_t t0 = w0 + first;
        const int64_t slot = first < 64 ? wave_lane(slot_at[0], first) : slots[t0];
        const int64_t pg = slot >> c.lp;
        const int off = (int)(slot & (page - 1));
        const int next = next_set(stops, first + 1);
        const int run = min(next - first, page - off), pieces = run * PR;
        if (several) first = next_set(begins, next);
        const T* x = (values ? v + t0 * ld_v : k + t0 * ld_k) + (int64_t)head * D;
        const int64_t ld = values ? ld_v : ld_k;
        uint8_t* scale = (values ? c.v_scales : c.k_scales) + pg * c.heads + head;
        uint8_t* codes = (values ? c.v_codes : c.k_codes) + (pg * c.heads + head) * (int64_t)page * D;
        const int before = off > 0 ? min(max((int)*scale, RAZER_CACHE_MIN_EXPONENT), RAZER_CACHE_MAX_EXPONENT) : RAZER_CACHE_MIN_EXPONENT;

        Raw held[kHold];
        float amax = 0.0f;
#pragma unroll
        for (int n = 0; n < kHold; ++n) {
            const int i = i0 + n * 128;
            if (i < pieces) held[n].load(x + (int64_t)(i / PR) * ld + i % PR * 8);
        }
#pragma unroll
        for (int n = 0; n < kHold; ++n)
            if (i0 + n * 128 < pieces) amax = absmax8(held[n].get(), amax);
#pragma unroll 2
        for (int i = i0 + kHold * 128; i < pieces; i += 128) {
            Raw r;
            r.load(x + (int64_t)(i / PR) * ld + i % PR * 8);
            amax = absmax8(r.get(), amax);
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) amax = fmaxf(amax, __shfl_xor(amax, d));
        if ((tid & 63) == 0) s_max[tid >> 6] = amax;
        __syncthreads();
        amax = values ? fmaxf(s_max[2], s_max[3]) : fmaxf(s_max[0], s_max[1]);
        const int b = max(before, exponent_of(amax));
        const bool few = run <= kFewTokens;                              // values byte by byte, without LDS
        if (i0 == 0) *scale = (uint8_t)b;                                // (all have read it: the barrier above)
        if (off > 0 && b > before) {
            const float mul = exponent_value(max(127 + before - b, 1));
            if (!values) {
#pragma unroll 1
                for (int i = i0; i < off * D / 4; i += 128) {
                    uint32_t* p = reinterpret_cast<uint32_t*>(codes) + i;
                    *p = move4(*p, mul);
                }
            } else {                                                     // the last word of a row may hold new places too: byte by byte
                const int words = off >> 2, rest = off & 3;
#pragma unroll 1
                for (int i = i0; i < words * D; i += 128) {
                    uint32_t* p = reinterpret_cast<uint32_t*>(codes + i / words * page) + i % words;
                    *p = move4(*p, mul);
                }
#pragma unroll 1
                for (int i = i0; i < rest * D; i += 128) {
                    uint8_t* p = codes + i / rest * page + words * 4 + i % rest;
                    *p = (uint8_t)move4(*p, mul);
                }
            }
        }
        const float inv = exponent_value(254 - b);
        auto put = [&](int i, const Eight& e) {
            const uint2 w = encode8(e, inv);
            const int tok = i / PR, d = i % PR * 8;
            if (!values) {
                *reinterpret_cast<uint2*>(codes + (off + tok) * D + d) = w;
            } else if (few) {
#pragma unroll
                for (int j = 0; j < 8; ++j) codes[(d + j) * page + off + tok] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
            } else {
                uint32_t* to = reinterpret_cast<uint32_t*>(tile + tok * LDT + d);
                to[0] = w.x;
                to[1] = w.y;
            }
        };
#pragma unroll
        for (int n = 0; n < kHold; ++n)
            if (i0 + n * 128 < pieces) put(i0 + n * 128, held[n].get());
#pragma unroll 2
        for (int i = i0 + kHold * 128; i < pieces; i += 128) {
            Raw r;
            r.load(x + (int64_t)(i / PR) * ld + i % PR * 8);
            put(i, r.get());
        }
        if (few) continue;
        __syncthreads();
        // the values' page, 16 tokens of an element at a time; all threads
        uint8_t* vp = c.v_codes + (pg * c.heads + head) * (int64_t)page * D;
        const int g0 = off >> 4, groups = ((off + run + 15) >> 4) - g0;
#pragma unroll 1
        for (int i = tid; i < D * groups; i += kAppendThreads) {
            const int d = i % D, at = (g0 + i / D) * 16;
            const uint8_t* from = tile + (at - off) * LDT + d;           // (of the group's first token, which may lie before the run)
            if (at >= off && at + 16 <= off + run) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = from[4 * j * LDT] | from[(4 * j + 1) * LDT] << 8 | from[(4 * j + 2) * LDT] << 16 | (uint32_t)from[(4 * j + 3) * LDT] << 24;
                *reinterpret_cast<uint4*>(vp + d * page + at) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll 1
                for (int j = max(off - at, 0); j < min(off + run - at, 16); ++j) vp[d * page + at + j] = from[j * LDT];
            }
        }
    }
}

template <typename T>
static void append_dim(const CacheView& c, const T* k, int64_t ld_k, const T* v, int64_t ld_v, int64_t tokens, const int64_t* slots, hipStream_t st)
{
    const int share = tokens <= kAppendFew && tokens * c.heads <= kAppendFewRows ? kAppendWindow : 2;
    const dim3 grid((unsigned)((tokens + kAppendWindow - 1) / kAppendWindow * share * c.heads));
    const size_t smem = (size_t)(c.dim + 4) << c.lp;
    switch (c.dim) {
        case 64: launch(cache_append_kernel<T, 64>, grid, kAppendThreads, smem, st, c, k, ld_k, v, ld_v, tokens, slots, share); break;
        case 128: launch(cache_append_kernel<T, 128>, grid, kAppendThreads, smem, st, c, k, ld_k, v, ld_v, tokens, slots, share); break;
        case 192: launch(cache_append_kernel<T, 192>, grid, kAppendThreads, smem, st, c, k, ld_k, v, ld_v, tokens, slots, share); break;
        default: launch(cache_append_kernel<T, 256>, grid, kAppendThreads, smem, st, c, k, ld_k, v, ld_v, tokens, slots, share); break;
    }
}

hipError_t launch_cache_append(const CacheView& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v, int bf16,
                               int64_t tokens, const int64_t* slots, hipStream_t st)
{
    if (tokens == 0) return hipSuccess;
    if (bf16) append_dim(c, reinterpret_cast<const uint16_t*>(k), ld_k, reinterpret_cast<const uint16_t*>(v), ld_v, tokens, slots, st);
    else append_dim(c, reinterpret_cast<const float*>(k), ld_k, reinterpret_cast<const float*>(v), ld_v, tokens, slots, st);
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
    if (c->pages < 1 || c->pages > ((int64_t)1 << 31) - 1 || c->kv_heads < 1 || c->kv_heads > 8192) return RAZER_ERR_SHAPE;
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
    if (tokens * c.heads >= ((int64_t)1 << 26)) return RAZER_ERR_SHAPE;  // (fewer than 2^24 workgroups)
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
    const size_t need = attention_workspace_used(c, a, args->max_new, args->max_len);
    if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return RAZER_ERR_WORKSPACE;
    const hipError_t e = launch_attention(c, a, args->max_new, args->max_len, static_cast<float*>(workspace),
                                          static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? RAZER_OK : RAZER_ERR_HIP;
}

}  // extern "C"
