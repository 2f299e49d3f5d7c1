// Sampling from logits (include/razer_step.h) for gfx950.
//
// The tokens of a row, ordered by logit and index, need no sort: top-k, top-p, min-p and the draw itself each ask for one
// place in that order, and a place is found digit by digit of the logits' ordered bit patterns ("keys"), from a histogram
// of counts and one of weights per digit.  Weights are exp((l - max) / T) formed in 64 bits and summed as multiples of
// 2^-shift in 64-bit integers, so the histograms' atomics give the same sums in any order.
#include "razer_step.hpp"

namespace razer {

namespace {

struct SampleArgs {
    const void* logits;
    const float* uniform;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    int32_t* tokens;
    float* logprobs;
    int64_t ld;
    uint32_t vocab;
    int shift;
};

constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;

// Bit pattern whose unsigned order is the logit's; 0: no token (NaN, -infinity)
template <bool B16>
__device__ __forceinline__ uint32_t key_of(float l)
{
    if (!(l > -__builtin_inff())) return 0u;
    l = fminf(l, B16 ? 3.3895313892515355e38f : 3.4028234663852886e38f) + 0.0f;   // (-0 becomes +0)
    const uint32_t u = f2u(l);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return u2f((key >> 31) ? key ^ 0x80000000u : ~key); }

template <bool B16>
__device__ __forceinline__ uint32_t load_key(const void* row, uint32_t i)
{
    return key_of<B16>(B16 ? bf16_bits_to_f32(static_cast<const uint16_t*>(row)[i]) : static_cast<const float*>(row)[i]);
}

struct Weight {                                                            // of a row: exp((l - max) / T) 2^shift
    double max, inv;                                                       // inv: 0 where T is infinite
    double unit;
    __device__ __forceinline__ double real(uint32_t key) const { return exp(((double)logit_of(key) - max) * inv); }
    __device__ __forceinline__ uint64_t whole(uint32_t key) const { return (uint64_t)__builtin_rint(real(key) * unit); }
};

struct Shared {
    uint32_t count[kBins];
    unsigned long long weight[kBins];
    uint64_t wave_sum[kWaves];
    uint64_t answer[4];
};

__device__ __forceinline__ uint64_t shfl_up64(uint64_t v, int d) { return (uint64_t)__shfl_up((unsigned long long)v, d); }

// Sum of v over the threads before this one; total in `total`.
__device__ __forceinline__ uint64_t block_before(uint64_t v, Shared& sh, uint64_t& total)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint64_t run = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = shfl_up64(run, d);
        if (lane >= (uint32_t)d) run += o;
    }
    __syncthreads();
    if (lane == 63) sh.wave_sum[wave] = run;
    __syncthreads();
    uint64_t before = 0;
    total = 0;
    for (uint32_t w = 0; w < kWaves; ++w) {
        const uint64_t s = sh.wave_sum[w];
        if (w < wave) before += s;
        total += s;
    }
    return before + run - v;
}

// A beginning of the order: all tokens above `key` and the first `ties` of the `equal` ones at it; `above`: count or
// weight of the former.
struct Place {
    uint32_t key;
    uint64_t ties, equal, above;
};

// The shortest beginning inside `within` whose count (BY_WEIGHT: weight) reaches target; what is there reaches it.
template <bool B16, bool BY_WEIGHT>
__device__ Place find_place(const void* row, uint32_t vocab, const Weight& wt, Shared& sh, const Place& within, uint64_t target)
{
    constexpr int LEVELS = B16 ? 2 : 3;
    uint32_t prefix = 0, mask = 0;
    uint64_t above = 0;
#pragma unroll 1
    for (int level = 0; level < LEVELS; ++level) {
        const int lo = level == 0 ? 21 : level == 1 ? 10 : 0;
        __syncthreads();
        for (uint32_t b = threadIdx.x; b < kBins; b += kThreads) {
            sh.count[b] = 0;
            sh.weight[b] = 0;
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < vocab; i += kThreads) {
            const uint32_t key = load_key<B16>(row, i);
            if (key != 0 && key >= within.key && (key & mask) == prefix) {
                const uint32_t b = (key >> lo) & (kBins - 1);
                if (BY_WEIGHT) atomicAdd(&sh.weight[b], (unsigned long long)wt.whole(key));
                atomicAdd(&sh.count[b], 1u);
            }
        }
        __syncthreads();
        // two bins per thread, from the top
        const uint32_t b0 = kBins - 1 - 2 * threadIdx.x;
        uint64_t v[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t b = b0 - j;
            v[j] = BY_WEIGHT ? sh.weight[b] : sh.count[b];
            if (within.equal > within.ties && (within.key & mask) == prefix && b == ((within.key >> lo) & (kBins - 1)))   // equal ones that are not inside
                v[j] -= (within.equal - within.ties) * (BY_WEIGHT ? wt.whole(within.key) : 1u);
        }
        uint64_t total;
        uint64_t run = above + block_before(v[0] + v[1], sh, total);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (run < target && run + v[j] >= target) {
                sh.answer[0] = b0 - j;
                sh.answer[1] = run;
                sh.answer[2] = sh.count[b0 - j];
            }
            run += v[j];
        }
        __syncthreads();
        prefix |= (uint32_t)sh.answer[0] << lo;
        mask |= (kBins - 1u) << lo;
        if (lo == 0) mask = 0xFFFFFFFFu;
        above = sh.answer[1];
    }
    Place p;
    p.key = prefix;
    if (B16 && !(prefix >> 31)) p.key |= 0x3FFu;                           // (the low bits of a negative number's key)
    p.above = above;
    p.equal = sh.answer[2];
    const uint64_t each = BY_WEIGHT ? wt.whole(p.key) : 1u;
    p.ties = (target - above + each - 1) / each;
    return p;
}

template <bool B16>
__global__ __launch_bounds__(kThreads) void sample_kernel(const SampleArgs a)
{
    __shared__ Shared sh;
    const uint32_t r = blockIdx.x, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const void* row = static_cast<const uint8_t*>(a.logits) + (int64_t)r * a.ld * (B16 ? 2 : 4);
    // the largest, and how many tokens there are
    uint32_t most = 0;
    uint64_t n = 0;
    for (uint32_t i = tid; i < a.vocab; i += kThreads) {
        const uint32_t key = load_key<B16>(row, i);
        most = max(most, key);
        n += key != 0;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off));
    if (lane == 0) sh.count[wave] = most;
    uint64_t tokens;
    block_before(n, sh, tokens);
    for (uint32_t w = 0; w < kWaves; ++w) most = max(most, sh.count[w]);
    if (tokens == 0) {
        if (tid == 0) {
            a.tokens[r] = -1;
            if (a.logprobs) a.logprobs[r] = -__builtin_inff();
        }
        return;
    }
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    const int32_t top_k = a.top_k ? a.top_k[r] : 0;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p && a.min_p[r] > 0.0f ? fminf(a.min_p[r], 1.0f) : 0.0f;
    const float u = a.uniform[r];
    const bool greedy = !(t > 0.0f);
    Weight wt;
    wt.max = (double)logit_of(most);
    wt.inv = greedy ? 1.0 : 1.0 / (double)t;
    wt.unit = (double)((uint64_t)1 << a.shift);
    Place at;
    double share = 0.0;
    if (greedy) {
        at = Place{most, 1, 1, 0};
    } else {
        Place kept{0u, 0, 0, 0};                                           // everything
        if (top_k > 0 && (uint64_t)top_k < tokens) kept = find_place<B16, false>(row, a.vocab, wt, sh, kept, (uint64_t)top_k);
        auto weight_of = [&](const Place& p) {                             // of a beginning
            uint64_t s = 0, sum;
            for (uint32_t i = tid; i < a.vocab; i += kThreads) {
                const uint32_t key = load_key<B16>(row, i);
                if (key != 0 && key >= p.key) s += wt.whole(key);
            }
            block_before(s, sh, sum);
            return p.equal > p.ties ? sum - (p.equal - p.ties) * wt.whole(p.key) : sum;
        };
        uint64_t sum = weight_of(kept);
        if (top_p < 1.0f) {
            const double want = __builtin_ceil((double)fmaxf(top_p, 0.0f) * (double)sum);
            uint64_t target = want < 1.0 ? 1u : (uint64_t)want;
            target = target > sum ? sum : target;
            kept = find_place<B16, true>(row, a.vocab, wt, sh, kept, target);
            sum = kept.above + kept.ties * wt.whole(kept.key);
        }
        if (min_p > 0.0f && !(kept.key != 0 && wt.real(kept.key) >= (double)min_p)) {
            // the keys whose weights reach min_p lie from a key on that is found by halving
            uint32_t low = kept.key, high = most;                          // high reaches it (or is the largest), low does not
            while (high - low > 1) {
                const uint32_t mid = low + (high - low) / 2;
                if (wt.real(mid) >= (double)min_p) high = mid;
                else low = mid;
            }
            kept = Place{high, 0, 0, 0};
            sum = weight_of(kept);
        }
        const double want = __builtin_floor((double)fmaxf(u, 0.0f) * (double)sum);
        uint64_t target = want >= (double)sum ? sum : (uint64_t)want + 1u;
        target = target > sum ? sum : target;
        at = find_place<B16, true>(row, a.vocab, wt, sh, kept, target);
        share = log((double)wt.whole(at.key) / (double)sum);
    }
    // the at.ties-th token with that key: a wave counts in a stretch of the row
    const uint32_t stretch = ((a.vocab + kWaves - 1) / kWaves + 63u) & ~63u;
    const uint32_t begin = min(wave * stretch, a.vocab), end = min(begin + stretch, a.vocab);
    uint64_t mine = 0;
    for (uint32_t i = begin; i < end; i += 64) mine += __popcll(__ballot(i + lane < end && load_key<B16>(row, i + lane) == at.key));
    uint64_t all;
    uint64_t before = block_before(lane == 0 ? mine : 0, sh, all);
    before = (uint64_t)__shfl((unsigned long long)before, 0);
    if (before < at.ties && before + mine >= at.ties) {
        uint32_t rank = (uint32_t)(at.ties - before);
        for (uint32_t i = begin; i < end; i += 64) {
            const bool hit = i + lane < end && load_key<B16>(row, i + lane) == at.key;
            const uint64_t b = __ballot(hit);
            const uint32_t c = __popcll(b);
            if (rank <= c) {
                if (hit && (uint32_t)__popcll(b & (((uint64_t)1 << lane) - 1)) + 1 == rank) {
                    a.tokens[r] = (int32_t)(i + lane);
                    if (a.logprobs) a.logprobs[r] = (float)share;
                }
                break;
            }
            rank -= c;
        }
    }
}

}  // namespace

}  // namespace razer

using namespace razer;

static razer_status check_sample(const razer_sample_args* g)
{
    if (!g) return RAZER_ERR_NULL;
    if (g->dtype != RAZER_F32 && g->dtype != RAZER_BF16) return RAZER_ERR_CONFIG;
    if (g->rows < 0 || g->rows >= ((int64_t)1 << 24) || g->vocab < 1 || g->vocab > ((int64_t)1 << 24) || g->ld < g->vocab) return RAZER_ERR_SHAPE;
    if (g->rows == 0) return RAZER_OK;
    if (!g->logits || !g->uniform || !g->tokens) return RAZER_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(g->logits) % (g->dtype == RAZER_BF16 ? 2 : 4) != 0 || !aligned4(g->uniform) || !aligned4(g->temperature) || !aligned4(g->top_k) ||
        !aligned4(g->top_p) || !aligned4(g->min_p) || !aligned4(g->tokens) || !aligned4(g->logprobs))
        return RAZER_ERR_ALIGN;
    return RAZER_OK;
}

extern "C" {

size_t razer_sample_workspace_bytes(const razer_sample_args* args)
{
    return 0;
}

razer_status razer_sample(const razer_sample_args* g, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const razer_status s = check_sample(g);
    if (s != RAZER_OK || g->rows == 0) return s;
    int lv = 0;
    while (((int64_t)1 << lv) < g->vocab) ++lv;
    const SampleArgs a{g->logits, g->uniform, g->temperature, g->top_k, g->top_p, g->min_p, g->tokens, g->logprobs, g->ld, (uint32_t)g->vocab, 62 - lv};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->dtype == RAZER_BF16) launch(sample_kernel<true>, (uint32_t)g->rows, kThreads, 0, st, a);
    else launch(sample_kernel<false>, (uint32_t)g->rows, kThreads, 0, st, a);
    return hipGetLastError() == hipSuccess ? RAZER_OK : RAZER_ERR_HIP;
}

}  // extern "C"
