// Sampling from logits (include/razer_step.h) for gfx950.
//
// The tokens of a row, ordered by logit and index, need no sort: top-k, top-p, min-p and the draw itself each ask for one
// place in that order.  With z = (max - l) / T in octaves, weight 2^-z, a histogram of kBinsPerOctave bins per octave of z
// says which bin each place lies in; only those bins' tokens are gathered, sorted and weighed one by one.
//   A bin's entry is one 64-bit integer: the count above, below it how much its tokens weigh less than the bin's
// upper end together (in multiples of 2^-31 of it), so that one LDS atomic per token gives count and weight, in any
// order the same, the weight to a relative 2^-27 (bin_deficit).  What lies beyond 32 octaves shares one bin, in which weights are
// summed in multiples of 2^-57; its tokens are listed and weighed one by one like any other bin's.
//   Bound by the vector unit, not by the logits' bytes: three looks at each logit (the largest, the histogram, the gathering), the
// second of which costs an exponent, a polynomial and an atomic per token, and then one workgroup's sort of up to 4096 tokens.
// A few long rows are cut into pieces over the GPU for those three looks (five launches, pieces_of); many rows, or short ones,
// take one workgroup each from beginning to end.  One row of 32000 19 us, 251 rows of 100003 (50 MB) 54 us, 64 rows of
// 128000 fp32 logits in pieces (33 MB) 50 us: 7 the largest, 14 the bins, 7 the bounds, 11 the gathering, then the sort and
// the draw.
//   Rows whose places lie in too full bins (all logits alike, temperatures of 20 and more) and vocabularies beyond 2^18 are
// resolved digit by digit of the logits' ordered bit patterns instead (find_place), at several looks per place.
#include <type_traits>

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
    uint32_t pieces, piece;                      // of a row: how many, of how many tokens (a multiple of 8)
    uint32_t* piece_max;                         // [rows][pieces] keys
    struct RowState* rows;                       // [rows]
};

constexpr uint32_t kWholeThreads = 1024, kRowThreads = 1024, kPieceThreads = 512, kBins = 2048;
constexpr int kBinsPerOctave = 64;
constexpr uint32_t kRest = kBins - 1;            // the bin of everything beyond 32 octaves
constexpr uint32_t kIdle = 64;                   // idle places behind the bins (fill_bins)
constexpr uint32_t kList = 4096;                 // tokens that can be weighed one by one
constexpr int kCountShift = 44;                  // 2^18 tokens of at most (1 - 2^(-1/64)) 2^31, or of 2^25, stay below it
constexpr int64_t kBinnedVocab = (int64_t)1 << 18;

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

struct Weight {                                                            // of a row: exp((l - max) / T)
    double max, inv;
    __device__ __forceinline__ double real(uint32_t key) const { return exp(((double)logit_of(key) - max) * inv); }
    __device__ __forceinline__ uint64_t whole(uint32_t key) const { return (uint64_t)__builtin_rint(real(key) * 0x1p57); }
};

// A count, or a sum of weights in multiples of 2^-57: high 2^29 + low.  2^24 weights of up to 2^57 need 81 bits; halves of a weight
// are summed each for itself (below 2^53) and the carry settled afterwards.
struct Wide {
    uint64_t high, low;
    static constexpr int kBits = 29;
    static constexpr uint64_t kLow = ((uint64_t)1 << kBits) - 1;
    static __device__ __forceinline__ Wide settled(uint64_t high, uint64_t low) { return Wide{high + (low >> kBits), low & kLow}; }
    static __device__ __forceinline__ Wide of(uint64_t n) { return Wide{n >> kBits, n & kLow}; }
    // n times w, n at most 2^24
    static __device__ __forceinline__ Wide times(uint64_t w, uint64_t n) { return settled((w >> kBits) * n, (w & kLow) * n); }
    // a whole number of at most 2^82
    static __device__ __forceinline__ Wide from(double d)
    {
        const uint64_t high = (uint64_t)(d * 0x1p-29);
        return Wide{high, (uint64_t)(d - (double)high * 0x1p29)};
    }
    __device__ __forceinline__ double real() const { return (double)high * 0x1p29 + (double)low; }
    __device__ __forceinline__ Wide operator+(const Wide& o) const { return settled(high + o.high, low + o.low); }
    __device__ __forceinline__ Wide operator-(const Wide& o) const { return low < o.low ? Wide{high - o.high - 1, low + kLow + 1 - o.low} : Wide{high - o.high, low - o.low}; }
    __device__ __forceinline__ bool operator<(const Wide& o) const { return high != o.high ? high < o.high : low < o.low; }
};

struct Digits {
    uint32_t count[kBins];
    unsigned long long high[kBins], low[kBins];
};
struct Binned {
    unsigned long long bins[kBins + kIdle];      // then the weight ahead of each bin, as doubles
    uint32_t before[kBins];                      // tokens ahead of each bin
    uint32_t start[kBins];                       // of them, the ones that are listed
    uint32_t wanted[kBins / 32];                 // the bins that are listed
    __device__ __forceinline__ double ahead(uint32_t bin) const { return __builtin_bit_cast(double, (uint64_t)bins[bin]); }
};
struct Listed {
    uint64_t list[kList];
    double run[kList];                           // weight of the order up to each one
};
struct Sums {
    uint64_t wave_u[kWholeThreads / 64], wave_v[kWholeThreads / 64];
    uint64_t answer[4];
    uint32_t found[8];
    double octave[kBinsPerOctave];               // 2^(-i / kBinsPerOctave)
    __device__ __forceinline__ void fill_octave()
    {
        if (threadIdx.x < kBinsPerOctave) octave[threadIdx.x] = exp2(-(double)threadIdx.x / kBinsPerOctave);
    }
    // weight of a bin's upper end
    __device__ __forceinline__ double unit(uint32_t bin) const
    {
        return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, octave[bin % kBinsPerOctave]) - ((uint64_t)(bin / kBinsPerOctave) << 52));
    }
};
struct Shared : Sums {
    union {
        Digits d;
        struct {
            Binned b;
            Listed l;
        };
    };
};

// v of another lane of the wave as DPP control CTRL has it; 0 where there is none
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T from_lane(T v)
{
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)__builtin_bit_cast(uint32_t, v), CTRL, ROWS, 0xF, true));
    } else {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xF, true);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xF, true);
        return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
    }
}
// inclusive sums over the 16 lanes of a row, and over the wave's (0.0 and 0 are the same bits)
template <typename T, int CTRL, int ROWS>
__device__ __forceinline__ T plus_lane(T v) { return v + from_lane<CTRL, ROWS>(v); }
template <typename T>
__device__ __forceinline__ T row_scan(T v)
{
    v = plus_lane<T, 0x111, 0xF>(v);                                       // row_shr 1, 2, 4, 8
    v = plus_lane<T, 0x112, 0xF>(v);
    v = plus_lane<T, 0x114, 0xF>(v);
    return plus_lane<T, 0x118, 0xF>(v);
}
template <typename T>
__device__ __forceinline__ T wave_scan(T v)
{
    v = plus_lane<T, 0x142, 0xA>(row_scan(v));                             // row_bcast 15, 31
    return plus_lane<T, 0x143, 0xC>(v);
}
template <typename T>
__device__ __forceinline__ T lane_value(T v, uint32_t lane)                // (lane: uniform)
{
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, (uint32_t)__builtin_amdgcn_readlane((int)__builtin_bit_cast(uint32_t, v), (int)lane));
    } else {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, (int)lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), (int)lane);
        return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
    }
}

// Sum of v over the threads before this one (of WAVES waves), and of all.  Doubles are added in a fixed order.  The sums of
// the waves are scanned by every wave alike, one in a lane: with a loop over them in each thread this took twice as long.
template <typename T>
__device__ __forceinline__ T waves_before(T run, T v, const uint64_t* sums, uint32_t waves, T& all)
{
    const uint32_t lane = threadIdx.x & 63u, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const T own = *reinterpret_cast<const T*>(sums + (lane < waves ? lane : 0u));
    const T up = row_scan(lane < waves ? own : T(0));
    all = lane_value(up, waves - 1);
    return (w ? lane_value(up, w - 1) : T(0)) + (run - v);
}
template <uint32_t WAVES, typename U, typename V>
__device__ __forceinline__ void block_before(U& u, V& v, Sums& sh, U& all_u, V& all_v)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const U ru = wave_scan(u);
    const V rv = wave_scan(v);
    __syncthreads();
    if (lane == 63) {
        *reinterpret_cast<U*>(sh.wave_u + wave) = ru;
        *reinterpret_cast<V*>(sh.wave_v + wave) = rv;
    }
    __syncthreads();
    u = waves_before(ru, u, sh.wave_u, WAVES, all_u);
    v = waves_before(rv, v, sh.wave_v, WAVES, all_v);
}
template <uint32_t WAVES, typename T>
__device__ __forceinline__ T block_before(T v, Sums& sh, T& all)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const T run = wave_scan(v);
    __syncthreads();
    if (lane == 63) *reinterpret_cast<T*>(sh.wave_u + wave) = run;
    __syncthreads();
    return waves_before(run, v, sh.wave_u, WAVES, all);
}

// A beginning of the order: all tokens above `key` and the first `ties` of the `equal` ones at it; `above`: count or
// weight of the former.
struct Place {
    uint32_t key;
    uint64_t ties, equal;
    Wide above;
};

// The shortest beginning inside `within` whose count (BY_WEIGHT: weight) reaches target; what is there reaches it.
template <uint32_t THREADS, bool B16, bool BY_WEIGHT>
__device__ Place find_place(const void* row, uint32_t vocab, const Weight& wt, Shared& sh, Place within, Wide target)
{
    constexpr int LEVELS = B16 ? 2 : 3;
    uint32_t prefix = 0, mask = 0;
    Wide above{0, 0};
#pragma unroll 1
    for (int level = 0; level < LEVELS; ++level) {
        const int lo = level == 0 ? 21 : level == 1 ? 10 : 0;
        __syncthreads();
        for (uint32_t b = threadIdx.x; b < kBins; b += THREADS) {
            sh.d.count[b] = 0;
            sh.d.high[b] = 0;
            sh.d.low[b] = 0;
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < vocab; i += THREADS) {
            const uint32_t key = load_key<B16>(row, i);
            if (key != 0 && key >= within.key && (key & mask) == prefix) {
                const uint32_t b = (key >> lo) & (kBins - 1);
                if (BY_WEIGHT) {
                    const Wide w = Wide::of(wt.whole(key));
                    atomicAdd(&sh.d.high[b], (unsigned long long)w.high);
                    atomicAdd(&sh.d.low[b], (unsigned long long)w.low);
                }
                atomicAdd(&sh.d.count[b], 1u);
            }
        }
        __syncthreads();
        // PER bins per thread, from the top
        constexpr uint32_t PER = kBins / THREADS;
        const uint32_t b0 = kBins - 1 - PER * threadIdx.x;
        Wide v[PER], sum{0, 0};
#pragma unroll
        for (uint32_t j = 0; j < PER; ++j) {
            const uint32_t b = b0 - j;
            v[j] = BY_WEIGHT ? Wide::settled(sh.d.high[b], sh.d.low[b]) : Wide::of(sh.d.count[b]);
            if (within.equal > within.ties && (within.key & mask) == prefix && b == ((within.key >> lo) & (kBins - 1)))   // equal ones that are not inside
                v[j] = v[j] - Wide::times(BY_WEIGHT ? wt.whole(within.key) : 1u, within.equal - within.ties);
            sum = sum + v[j];
        }
        Wide total;
        block_before<THREADS / 64>(sum.high, sum.low, sh, total.high, total.low);
        Wide run = above + Wide::settled(sum.high, sum.low);
#pragma unroll
        for (uint32_t j = 0; j < PER; ++j) {
            const Wide next = run + v[j];
            if (run < target && !(next < target)) {
                sh.answer[0] = b0 - j;
                sh.answer[1] = run.high;
                sh.answer[2] = run.low;
                sh.answer[3] = sh.d.count[b0 - j];
            }
            run = next;
        }
        __syncthreads();
        prefix |= (uint32_t)sh.answer[0] << lo;
        mask |= (kBins - 1u) << lo;
        if (lo == 0) mask = 0xFFFFFFFFu;
        above = Wide{sh.answer[1], sh.answer[2]};
    }
    Place p;
    p.key = prefix;
    if (B16 && !(prefix >> 31)) p.key |= 0x3FFu;                           // (the low bits of a negative number's key)
    p.above = above;
    p.equal = sh.answer[3];
    // the fewest of the equal ones that reach the target: a quotient of at most 2^24, of which doubles may miss 2^-28, so that what they
    // leave before the point is up to two short.  (No loop that ends by what the logits are: they may change under a caller's mistake)
    const uint64_t each = BY_WEIGHT ? wt.whole(p.key) : 1u;
    const Wide rest = target - above;
    p.ties = (uint64_t)(rest.real() / (double)each);
    if (Wide::times(each, p.ties) < rest) ++p.ties;
    if (Wide::times(each, p.ties) < rest) ++p.ties;
    return p;
}

// f(index of the first, 16 bytes of logits) for the logits begin .. end-1 of a row; those at the ends that share their 16 bytes
// with others come alone, -infinity beside them.  There is one copy of f in the code, in a loop that loads four pieces
// ahead: what these kernels wait for on short rows are their instructions (with copies of f for the ends and for four
// pieces at a time the whole-row kernel was 65 KB long).
template <bool B16, typename F>
__device__ __forceinline__ void each_piece(const void* row, uint32_t begin, uint32_t end, F f)
{
    constexpr uint32_t E = B16 ? 8 : 4, SZ = B16 ? 2 : 4, NONE = B16 ? 0xFF80FF80u : 0xFF800000u;
    const uint32_t tid = threadIdx.x, threads = blockDim.x;
    const uint8_t* base = static_cast<const uint8_t*>(row);
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(base + (size_t)begin * SZ) & 15u) / SZ;
    const uint32_t first = min(begin + (off ? E - off : 0u), end), vecs = (end - first) / E, last = first + vecs * E;
    const uint4* p = reinterpret_cast<const uint4*>(base + (size_t)first * SZ);
    uint4 q[4];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
        if (tid + j * threads < vecs) q[j] = p[tid + j * threads];
    // the first wave begins with the ends, a logit in a lane
    const uint32_t head = first - begin, alone = head + end - last;
    uint32_t v = tid;
    bool ends = __builtin_amdgcn_readfirstlane(tid >> 6) == 0 && alone != 0;
    while (ends || v < vecs) {
        uint4 cur;
        uint32_t at;
        if (ends) {
            at = tid < head ? begin + tid : last + tid - head;
            cur = make_uint4(NONE, NONE, NONE, NONE);
            if (tid < alone) cur.x = B16 ? 0xFF800000u | static_cast<const uint16_t*>(row)[at] : static_cast<const uint32_t*>(row)[at];
            ends = false;
        } else {
            at = first + v * E;
            cur = q[0];
            q[0] = q[1]; q[1] = q[2]; q[2] = q[3];
            if (v + 4 * threads < vecs) q[3] = p[v + 4 * threads];
            v += threads;
        }
        f(at, cur);
    }
}
// logit j of 16 bytes
template <bool B16>
__device__ __forceinline__ float logit_at(const uint4& v, int j)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (B16) return u2f(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    else return u2f(w[j]);
}
// f(index, logit) for the few logits that pick(16 bytes) has a bit for
template <bool B16, typename P, typename F>
__device__ __forceinline__ void few_logits(const void* row, uint32_t begin, uint32_t end, P pick, F f)
{
    each_piece<B16>(row, begin, end, [&](uint32_t at, const uint4& v) {
        const uint32_t hits = pick(v);
        if (hits == 0) return;
#pragma unroll
        for (int j = 0; j < (B16 ? 8 : 4); ++j)
            if ((hits >> j) & 1u) f(at + j, logit_at<B16>(v, j));
    });
}
// The lowest index of the row's largest logit, into *token (a maximum of indexes before)
template <bool B16>
__device__ __forceinline__ void first_largest(const void* row, uint32_t begin, uint32_t end, float largest, uint32_t* token)
{
    auto pick = [&](const uint4& v) {
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < (B16 ? 8 : 4); ++j) hits |= logit_at<B16>(v, j) >= largest ? 1u << j : 0u;
        return hits;
    };
    few_logits<B16>(row, begin, end, pick, [&](uint32_t i, float) { atomicMin(token, i); });
}

// Largest key of begin .. end-1, in every lane of the wave (0: no token)
template <bool B16>
__device__ __forceinline__ uint32_t largest_key(const void* row, uint32_t begin, uint32_t end)
{
    float most = -__builtin_inff();
    each_piece<B16>(row, begin, end, [&](uint32_t, const uint4& v) {
#pragma unroll
        for (int j = 0; j < (B16 ? 8 : 4); ++j) most = fmaxf(most, logit_at<B16>(v, j));   // (a NaN never is the larger)
    });
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor(most, off));
    return key_of<B16>(most);
}

// How far a logit lies below the largest, in bins as a number of 11 bits before the point and 21 behind it; it never falls
// as the logit falls.  0 for infinity (the largest counts as finite); all of kRest's are one number.
struct Scale {
    double max, per, most;                                                 // most: of the difference, half a bin into kRest
    __device__ __forceinline__ uint32_t below(float l) const
    {
        const double v = __builtin_fma(fmin(max - (double)l, most), per, 0x1p31);   // (2^31: the unit in the last place is 2^-21)
        return (uint32_t)__builtin_bit_cast(uint64_t, v);
    }
};
__device__ __forceinline__ Scale scale_of(uint32_t largest, float t)
{
    const double per = 1.4426950408889634 * kBinsPerOctave / (double)t;
    return Scale{(double)logit_of(largest), per, ((double)kRest + 0.5) / per};
}
__device__ __forceinline__ uint32_t bin_of(uint32_t below) { return below >> 21; }

// How much less a token weighs than its bin's upper end, 1 - e^-x in multiples of 2^-31, x = frac ln 2 / kBinsPerOctave at most
// 0.0109: x - x^2/2 + x^3/6 in fp32; a token as large as the largest has 0, so that equal ones are counted.
//   What a weight is off by, relative to it: 2.6e-9 because `below` is rounded to 2^-21 of a bin (half of it times ln 2 / 64),
// 2.0e-9 from two roundings and a constant of fp32 (3 2^-24 of 0.0109), 0.6e-9 from x^4/24 and 0.5e-9 from cutting to multiples of
// 2^-31, together below 5.7e-9.  Sums over kRest add 1.1e-9 of the whole at most: up to 256 fp32 additions a thread and an
// exponent in fp32, of 2^-14 together.  So a sum of weights is right to 6.8e-9 < 2^-27 of itself.
__device__ __forceinline__ uint32_t bin_deficit(uint32_t below)
{
    constexpr double kX = 0.6931471805599453 / kBinsPerOctave * 0x1p-21;
    const float f = (float)(below & 0x1FFFFFu);
    const float e = __builtin_fmaf(f, (float)(kX * kX * kX / 6 * 0x1p31), (float)(-kX * kX / 2 * 0x1p31));
    return (uint32_t)(f * __builtin_fmaf(f, e, (float)(kX * 0x1p31)));
}

// kRest's tokens are counted in registers: a temperature below 1 puts most of a row there, and atomics of a whole wave on one
// address take turns.  (In bins[] the wave writes to an idle place of each lane's own instead: no branch parts the others.)
template <bool B16>
__device__ __forceinline__ void fill_bins(const void* row, uint32_t begin, uint32_t end, const Scale& sc, unsigned long long* bins)
{
    constexpr int E = B16 ? 8 : 4;
    uint32_t rest = 0;
    float rest_weight = 0.0f;
    const uint32_t idle = kBins + (threadIdx.x & 63u);
    const float max32 = (float)sc.max, octaves32 = (float)(-sc.per / kBinsPerOctave);
    each_piece<B16>(row, begin, end, [&](uint32_t, const uint4& v) {
        uint32_t below[E];
        bool any = false;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float l = logit_at<B16>(v, j);
            below[j] = sc.below(l);
            any |= (bin_of(below[j]) == kRest) & (l > -__builtin_inff());  // (masked tokens are not in the rest)
        }
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const uint32_t bin = bin_of(below[j]);
            atomicAdd(&bins[bin == kRest ? idle : bin], (unsigned long long)((uint64_t)1 << kCountShift | bin_deficit(below[j])));
        }
        if (any) {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                // its weight (below 2^-31) in multiples of 2^-57: fp32 is enough beside the whole
                const float l = logit_at<B16>(v, j), w = __builtin_amdgcn_exp2f(__builtin_fmaf(max32 - l, octaves32, 57.0f));
                const bool in = bin_of(below[j]) == kRest && l > -__builtin_inff();
                rest += in;
                rest_weight += in ? w : 0.0f;
            }
        }
    });
    if (rest != 0) atomicAdd(&bins[kRest], (unsigned long long)((uint64_t)rest << kCountShift | (uint64_t)rest_weight));
}

struct Settings {
    float t, top_p, min_p, u;
    int32_t top_k;
    bool greedy;
};
__device__ __forceinline__ Settings settings_of(const SampleArgs& a, uint32_t r)
{
    Settings s;
    s.t = fminf(a.temperature ? a.temperature[r] : 1.0f, 3.4028234663852886e38f);   // 
    s.greedy = a.temperature && !(a.temperature[r] > 0.0f);
    s.top_k = a.top_k ? a.top_k[r] : 0;
    s.top_p = a.top_p ? a.top_p[r] : 1.0f;
    s.min_p = a.min_p && a.min_p[r] > 0.0f ? fminf(a.min_p[r], 1.0f) : 0.0f;
    s.u = fminf(fmaxf(a.uniform[r], 0.0f), 1.0f);                          // (a NaN: 0)
    return s;
}

// Where a row's places lie: bins that contain them for certain, and what is listed because of that.
struct Bounds {
    bool k_on, p_on, m_on;
    uint32_t bk, bm, p0, p1, s0, s1;     // top-k, min-p, top-p (first, last bin), the drawn token (first, last)
    uint32_t listed;                     // tokens in these bins
    double top;                          // weight of everything
    float floor;                         // no listed token lies below
};

// A row's state in the workspace, where it is cut into pieces
struct RowState {
    Binned b;
    Bounds o;
    uint32_t cursor;                             // of list; a greedy row's token
    uint64_t list[kList];
};

__device__ __forceinline__ void set_token(const SampleArgs& a, uint32_t r, int32_t token, float logprob)
{
    a.tokens[r] = token;
    if (a.logprobs) a.logprobs[r] = logprob;
}

// From the filled bins (in LDS); b then holds what the Binned fields say.
template <uint32_t THREADS>
__device__ __forceinline__ Bounds bounds_of(const Settings& s, const Scale& sc, Binned& b, Sums& sh)
{
    constexpr uint32_t PER = kBins / THREADS, WAVES = THREADS / 64;
    const uint32_t tid = threadIdx.x;
    uint32_t count[PER], n = 0, tokens;
    double weight[PER], sum = 0.0;
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) {
        const uint32_t bin = tid * PER + i;
        const uint64_t e = b.bins[bin];
        count[i] = (uint32_t)(e >> kCountShift);
        // (44 bits as a double: behind the point of 2^52)
        const double low = __builtin_bit_cast(double, (e & (((uint64_t)1 << kCountShift) - 1)) | 0x4330000000000000u) - 0x1p52;
        weight[i] = bin == kRest ? low * 0x1p-57 : sh.unit(bin) * ((double)count[i] - low * 0x1p-31);
        n += count[i];
        sum += weight[i];
    }
    if (tid < kBins / 32) b.wanted[tid] = 0;
    if (tid < 8) sh.found[tid] = kBins;
    Bounds o;
    block_before<WAVES>(n, sum, sh, tokens, o.top);
    uint32_t nb = n;
    double wb = sum;
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) {
        const uint32_t bin = tid * PER + i;
        b.before[bin] = nb;
        b.bins[bin] = __builtin_bit_cast(uint64_t, wb);                    // (every entry is in registers)
        nb += count[i];
        wb += weight[i];
        if (count[i] != 0 && nb == tokens) sh.found[6] = bin;    // the last one
        if (count[i] != 0 && s.top_k > 0 && nb >= (uint32_t)s.top_k && nb - count[i] < (uint32_t)s.top_k) sh.found[0] = bin;
    }
    __syncthreads();
    const uint32_t last = sh.found[6];
    o.k_on = s.top_k > 0 && (uint32_t)s.top_k < tokens;
    o.m_on = s.min_p > 0.0f;
    o.p_on = s.top_p < 1.0f;
    o.bk = o.k_on ? sh.found[0] : last;
    o.bm = last;
    if (o.m_on) {
        const double below = -log2((double)s.min_p) * kBinsPerOctave;
        // (a bin before kRest, or the last that has tokens; rounded as the logits' places are, or a token of min_p's own weight next
        // to a bin's border would stand in the bin behind)
        o.bm = below < (double)last ? bin_of((uint32_t)__builtin_bit_cast(uint64_t, below + 0x1p31)) : last;
    }
    auto after = [&](uint32_t bin) { return bin + 1 < kBins ? b.ahead(bin + 1) : o.top; };
    // the bin in which the running weight passes a target (STRICT: exceeds it); the first one for targets of 0
    auto pass = [&](int slot, double target, auto strict) {
#pragma unroll
        for (uint32_t i = 0; i < PER; ++i) {
            const double run = b.ahead(tid * PER + i), next = after(tid * PER + i);
            if (decltype(strict)::value ? run <= target && next > target : run < target && next >= target) sh.found[slot] = tid * PER + i;
        }
    };
    // A bin's tokens weighed one by one may come to less or more than its entry, by 6.8e-9 of the sum so far at most (bin_deficit), and
    // so may what stays: with 2e-8 the bounds hold whichever of the two a comparison uses.
    constexpr double kLess = 1.0 - 2e-8, kMore = 1.0 + 2e-8;
    double least = o.k_on ? b.ahead(o.bk) : o.top, largest = after(o.bk);    // of what stays
    o.p0 = o.p1 = last;
    if (o.p_on) {
        const double p = (double)fmaxf(s.top_p, 0.0f), t0 = p * least * kLess, t1 = p * largest * kMore;
        pass(1, t0, std::false_type{});
        pass(2, t1, std::false_type{});
        __syncthreads();
        o.p1 = t1 > 0.0 ? min(sh.found[2], o.bk) : 0u;
        o.p0 = t0 > 0.0 ? min(sh.found[1], o.p1) : 0u;
        least = fmin(least, b.ahead(o.p0));
        largest = fmin(largest, after(o.p1));
    }
    if (o.m_on) {
        least = fmin(least, b.ahead(o.bm));
        largest = fmin(largest, after(o.bm));
    }
    pass(3, (double)s.u * least * kLess, std::true_type{});
    pass(4, (double)s.u * largest * kMore, std::true_type{});
    __syncthreads();
    // (where top-p or min-p leave nothing of their last bin, `least` has led s0 to the one before)
    o.s1 = min(sh.found[4], min(min(o.bk, o.p1), o.bm));
    o.s0 = min(sh.found[3], o.s1);
    uint32_t want[PER], wants = 0;
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) {
        const uint32_t bin = tid * PER + i;
        const bool w = count[i] != 0 && ((o.k_on && bin == o.bk) || (o.m_on && bin == o.bm) || (o.p_on && bin >= o.p0 && bin <= o.p1) || (bin >= o.s0 && bin <= o.s1));
        want[i] = w ? count[i] : 0u;
        wants += want[i];
        if (w) atomicOr(&b.wanted[bin >> 5], 1u << (bin & 31u));
    }
    uint32_t listed, at = block_before<WAVES>(wants, sh, listed);
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) {
        b.start[tid * PER + i] = at;
        at += want[i];
    }
    o.listed = listed;
    const uint32_t lowest = max(max(o.k_on ? o.bk : 0u, o.m_on ? o.bm : 0u), max(o.p_on ? o.p1 : 0u, o.s1));
    o.floor = lowest == kRest ? -__builtin_inff() : (float)(sc.max - ((double)lowest + 1.5) / sc.per);
    __syncthreads();
    return o;
}

// The tokens of the wanted bins go to list[], `cursor` counting them: most logits lie below the floor and cost a comparison.
template <bool B16>
__device__ __forceinline__ void gather(const void* row, uint32_t begin, uint32_t end, const Scale& sc, float floor, const uint32_t* wanted, uint64_t* list, uint32_t* cursor)
{
    auto pick = [&](const uint4& v) {
        constexpr int E = B16 ? 8 : 4;
        float most = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < E; ++j) most = fmaxf(most, logit_at<B16>(v, j));
        if (most < floor) return 0u;
        uint32_t bin[E], word[E], hits = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) bin[j] = bin_of(sc.below(logit_at<B16>(v, j)));
#pragma unroll
        for (int j = 0; j < E; ++j) word[j] = wanted[bin[j] >> 5];
#pragma unroll
        for (int j = 0; j < E; ++j) hits |= (word[j] >> (bin[j] & 31u) & (uint32_t)(logit_at<B16>(v, j) > -__builtin_inff())) << j;
        return hits;
    };
    few_logits<B16>(row, begin, end, pick, [&](uint32_t i, float l) {
        const uint32_t at = atomicAdd(cursor, 1u);
        if (at < kList) list[at] = (uint64_t)~key_of<B16>(l) << 32 | i;
    });
}

// v of the lane J further up or down (lane ^ J)
template <int CTRL>
__device__ __forceinline__ uint64_t exchanged(uint64_t v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, 0xF, 0xF, true);
    return (uint64_t)hi << 32 | lo;
}
template <uint32_t J>
__device__ __forceinline__ uint64_t across(uint64_t v)
{
    if constexpr (J == 1) return exchanged<0xB1>(v);                       // quad_perm 1 0 3 2
    else if constexpr (J == 2) return exchanged<0x4E>(v);                  // quad_perm 2 3 0 1
    else if constexpr (J == 4) return exchanged<0x1B>(exchanged<0x141>(v));     // row_half_mirror, quad_perm 3 2 1 0: 7 ^ 3
    else if constexpr (J == 8) return exchanged<0x128>(v);                 // row_ror 8
    else return (uint64_t)__shfl_xor((unsigned long long)v, (int)J);
}

// Ascending sort of size (a power of two, 64 .. threads) entries, one in each thread: steps inside a wave exchange registers, the
// others go through list and spare in turn, so that one barrier each is enough.  (With every step in LDS 0.2 us each, 11 for
// 903 listed tokens; 64 rows of 128000: the call 57 us, 50 so.)
__device__ __forceinline__ void sort_in_registers(uint64_t* list, uint64_t* spare, uint32_t size)
{
    const uint32_t tid = threadIdx.x;
    const bool in = tid < size;                                            // (of whole waves)
    uint64_t v = in ? list[tid] : 0;
    uint64_t* to = spare;
    uint64_t* next = list;
    auto keep = [&](uint64_t o, uint32_t j, uint32_t k) {
        const bool least = ((tid & j) == 0) == ((tid & k) == 0);
        v = (o < v) == least ? o : v;
    };
#pragma unroll 1
    for (uint32_t k = 2; k <= size; k <<= 1) {
#pragma unroll 1
        for (uint32_t j = k >> 1; j >= 64; j >>= 1) {
            if (in) to[tid] = v;
            __syncthreads();
            if (in) keep(to[tid ^ j], j, k);
            uint64_t* t = to;
            to = next;
            next = t;
        }
        if (k > 32) keep(across<32>(v), 32, k);
        if (k > 16) keep(across<16>(v), 16, k);
        if (k > 8) keep(across<8>(v), 8, k);
        if (k > 4) keep(across<4>(v), 4, k);
        if (k > 2) keep(across<2>(v), 2, k);
        keep(across<1>(v), 1, k);
    }
    __syncthreads();
    if (in) list[tid] = v;
}

// The token from what is listed: o.listed entries of l.list, in any order.
template <uint32_t THREADS>
__device__ __forceinline__ void finish(const SampleArgs& a, uint32_t r, const Settings& s, const Scale& sc, const Bounds& o, const Binned& b, Listed& l, Sums& sh)
{
    const uint32_t tid = threadIdx.x, lane = tid & 63u, have = o.listed;
    uint32_t size = 64;
    while (size < have) size <<= 1;
    for (uint32_t i = have + tid; i < size; i += THREADS) l.list[i] = ~(uint64_t)0;
    if (tid < 8) sh.found[tid] = tid < 4 ? have : 0;
    // sort: by key, the largest first, then by index.  More entries than threads: in LDS, where steps of up to 64 stay inside the
    // 128 entries of one wave's pairs; its LDS operations are in order, the other waves are waited for ahead of the longer steps only.
    __syncthreads();
    if (size <= THREADS) sort_in_registers(l.list, reinterpret_cast<uint64_t*>(l.run), size);
    else for (uint32_t k = 2; k <= size; k <<= 1) {
        for (uint32_t j = k >> 1; j > 0; j >>= 1) {
            if (j > 64) __syncthreads();
            for (uint32_t i = tid; i < size / 2; i += THREADS) {
                const uint32_t x = ((i & ~(j - 1)) << 1) | (i & (j - 1)), y = x | j;
                const uint64_t u = l.list[x], v = l.list[y];
                if ((u > v) == ((x & k) == 0)) { l.list[x] = v; l.list[y] = u; }
            }
            if (j > 64) __syncthreads();
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
    __syncthreads();
    // the running sum of their weights; with it the sum up to each one in the order of all tokens: what is ahead of its bin,
    // and of the bin's own.  (Loops that are not unrolled: see each_piece.)
    Weight wt;
    wt.max = sc.max;
    wt.inv = 1.0 / (double)s.t;
    auto key_at = [&](uint32_t at) { return ~(uint32_t)(l.list[at] >> 32); };
    auto bin_at = [&](uint32_t at) { return bin_of(sc.below(logit_of(key_at(at)))); };
    auto up_to = [&](uint32_t at, uint32_t bin) {
        const uint32_t first = b.start[bin];
        return b.ahead(bin) + (l.run[at] - (first ? l.run[first - 1] : 0.0));
    };
    double carry = 0.0;
#pragma unroll 1
    for (uint32_t i = 0; i < have; i += THREADS) {
        const uint32_t at = i + tid;
        const double w = at < have ? wt.real(key_at(at)) : 0.0;
        double total;
        const double ahead = block_before<THREADS / 64>(w, sh, total);
        l.run[at] = carry + (ahead + w);
        carry += total;
    }
    __syncthreads();
    // first entry that fulfils a condition, one atomic per wave (entries of a wave ascend with the lane)
    auto first_of = [&](int slot, auto cond) {
#pragma unroll 1
        for (uint32_t i = 0; i < have; i += THREADS) {
            const uint32_t at = i + tid;
            const uint64_t hits = __ballot(at < have && cond(at));
            if (hits != 0 && lane == (uint32_t)__builtin_ctzll(hits)) atomicMin(&sh.found[slot], at);
        }
    };
    // what stays ends at a place of the list (or does not: behind any place, kList too is one), and weighs so much
    uint32_t stop = 0xFFFFFFFFu;
    double stays = o.top;
    if (o.k_on) {
        stop = b.start[o.bk] + ((uint32_t)s.top_k - b.before[o.bk]);       // one behind the last that stays
        stays = up_to(stop - 1, o.bk);
    }
    if (o.p_on) {
        const double target = (double)fmaxf(s.top_p, 0.0f) * stays;
        first_of(1, [&](uint32_t at) {
            const uint32_t bin = bin_at(at);
            return bin >= o.p0 && bin <= o.p1 && up_to(at, bin) >= target;
        });
        __syncthreads();
        const uint32_t behind = o.p1 + 1 < kBins ? b.start[o.p1 + 1] : have;   // (rounding may leave the target behind the last)
        const uint32_t at = min(sh.found[1] + 1u, behind);
        if (at < stop) {
            stop = at;
            stays = up_to(at - 1, bin_at(at - 1));
        }
    }
    if (o.m_on) {
        first_of(2, [&](uint32_t at) {
            const uint32_t bin = bin_at(at);
            return bin > o.bm || (bin == o.bm && wt.real(key_at(at)) < (double)s.min_p);
        });
        __syncthreads();
        const uint32_t first = b.start[o.bm], at = sh.found[2];
        if (at < stop) {
            stop = at;
            stays = at > first ? up_to(at - 1, o.bm) : b.ahead(o.bm);
        }
    }
    // (among the entries of the bins s0 .. s1 alone: between a later bin that is listed and these there are tokens that are not.
    // Nothing exceeds the whole, though a rounded running sum may)
    const double target = (double)s.u * stays;
    first_of(3, [&](uint32_t at) {
        const uint32_t bin = bin_at(at);
        return s.u < 1.0f && at < stop && bin >= o.s0 && bin <= o.s1 && up_to(at, bin) > target;
    });
    __syncthreads();
    uint32_t at = sh.found[3];
    if (at >= have) {                                                      // nothing exceeds the target: the last that can be drawn
#pragma unroll 1
        for (uint32_t i = 0; i < have; i += THREADS) {
            const uint64_t hits = __ballot(i + tid < have && i + tid < stop && bin_at(i + tid) <= o.s1 && wt.real(key_at(i + tid)) > 0.0);
            if (hits != 0 && lane == 63u - (uint32_t)__builtin_clzll(hits)) atomicMax(&sh.found[7], i + tid);
        }
        __syncthreads();
        at = sh.found[7];
    }
    if (tid == 0) set_token(a, r, (int32_t)(uint32_t)l.list[at], (float)log(wt.real(key_at(at)) / stays));
}

// The row's token digit by digit of the keys.  A sum is off by 2^24 halves of 2^-57 at most, less than 2^-33 of itself.
template <uint32_t THREADS, bool B16>
__device__ void by_digits(const void* row, const SampleArgs& a, uint32_t r, const Settings& s, uint32_t most, Shared& sh)
{
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    Weight wt;
    wt.max = (double)logit_of(most);
    wt.inv = 1.0 / (double)s.t;
    const float top_p = s.top_p, min_p = s.min_p;
    Place kept{0u, 0, 0, Wide{0, 0}};                                      // everything
    if (s.top_k > 0) {
        uint64_t n = 0, tokens;
        for (uint32_t i = tid; i < a.vocab; i += THREADS) n += load_key<B16>(row, i) != 0;
        (void)block_before<THREADS / 64>(n, sh, tokens);
        if ((uint64_t)s.top_k < tokens) kept = find_place<THREADS, B16, false>(row, a.vocab, wt, sh, kept, Wide::of((uint64_t)s.top_k));
    }
    auto weight_of = [&](const Place& p) {                             // of a beginning
        Wide s{0, 0}, sum;
        for (uint32_t i = tid; i < a.vocab; i += THREADS) {
            const uint32_t key = load_key<B16>(row, i);
            if (key != 0 && key >= p.key) {
                const Wide w = Wide::of(wt.whole(key));
                s.high += w.high;
                s.low += w.low;
            }
        }
        block_before<THREADS / 64>(s.high, s.low, sh, sum.high, sum.low);
        sum = Wide::settled(sum.high, sum.low);
        return p.equal > p.ties ? sum - Wide::times(wt.whole(p.key), p.equal - p.ties) : sum;
    };
    Wide sum = weight_of(kept);
    if (top_p < 1.0f) {
        const double want = __builtin_ceil((double)fmaxf(top_p, 0.0f) * sum.real());
        Wide target = Wide::from(want < 1.0 ? 1.0 : want);
        if (sum < target) target = sum;
        kept = find_place<THREADS, B16, true>(row, a.vocab, wt, sh, kept, target);
        sum = kept.above + Wide::times(wt.whole(kept.key), kept.ties);
    }
    if (min_p > 0.0f && !(kept.key != 0 && wt.real(kept.key) >= (double)min_p)) {
        // the keys whose weights reach min_p lie from a key on that is found by halving
        uint32_t low = kept.key, high = most;                          // high reaches it (or is the largest), low does not
        while (high - low > 1) {
            const uint32_t mid = low + (high - low) / 2;
            if (wt.real(mid) >= (double)min_p) high = mid;
            else low = mid;
        }
        kept = Place{high, 0, 0, Wide{0, 0}};
        sum = weight_of(kept);
    }
    const double want = __builtin_floor((double)s.u * sum.real());
    Wide target = sum;
    if (want < sum.real()) target = Wide::from(want) + Wide::of(1);
    if (sum < target) target = sum;
    const Place at = find_place<THREADS, B16, true>(row, a.vocab, wt, sh, kept, target);
    const double share = log(wt.real(at.key) / (sum.real() * 0x1p-57));      // (its own weight: as a whole number a light one has few digits)
    // the at.ties-th token with that key: a wave counts in a stretch of the row
    const uint32_t stretch = ((a.vocab + (THREADS / 64) - 1) / (THREADS / 64) + 63u) & ~63u;
    const uint32_t begin = min(wave * stretch, a.vocab), end = min(begin + stretch, a.vocab);
    uint64_t mine = 0;
    for (uint32_t i = begin; i < end; i += 64) mine += __popcll(__ballot(i + lane < end && load_key<B16>(row, i + lane) == at.key));
    uint64_t all;
    uint64_t before = block_before<THREADS / 64>((uint64_t)(lane == 0 ? mine : 0), sh, all);
    before = (uint64_t)__shfl((unsigned long long)before, 0);
    if (before < at.ties && before + mine >= at.ties) {
        uint32_t rank = (uint32_t)(at.ties - before);
        for (uint32_t i = begin; i < end; i += 64) {
            const bool hit = i + lane < end && load_key<B16>(row, i + lane) == at.key;
            const uint64_t b = __ballot(hit);
            const uint32_t c = __popcll(b);
            if (rank <= c) {
                if (hit && (uint32_t)__popcll(b & (((uint64_t)1 << lane) - 1)) + 1 == rank) {
                    set_token(a, r, (int32_t)(i + lane), (float)share);
                }
                break;
            }
            rank -= c;
        }
    }
}

// Rows that need no order: without a token, or the largest token alone
template <bool B16>
__device__ __forceinline__ bool plain_row(const void* row, const SampleArgs& a, uint32_t r, const Settings& s, uint32_t most, Sums& sh)
{
    if (most == 0) {
        if (threadIdx.x == 0) set_token(a, r, -1, -__builtin_inff());
        return true;
    }
    if (!s.greedy) return false;
    if (threadIdx.x == 0) sh.found[0] = a.vocab;
    __syncthreads();
    first_largest<B16>(row, 0, a.vocab, logit_of(most), &sh.found[0]);
    __syncthreads();
    if (threadIdx.x == 0) set_token(a, r, (int32_t)sh.found[0], 0.0f);
    return true;
}

template <bool B16>
__device__ __forceinline__ const void* row_of(const SampleArgs& a, uint32_t r) { return static_cast<const uint8_t*>(a.logits) + (int64_t)r * a.ld * (B16 ? 2 : 4); }

// A row per workgroup, from its first look to its token
template <bool B16>
__global__ __launch_bounds__(kWholeThreads) void sample_kernel(const SampleArgs a)
{
    __shared__ Shared sh;
    const uint32_t r = blockIdx.x, tid = threadIdx.x;
    const void* row = row_of<B16>(a, r);
    const Settings s = settings_of(a, r);
    const uint32_t mine = largest_key<B16>(row, 0, a.vocab);
    if ((tid & 63u) == 0) sh.wave_u[tid >> 6] = mine;
    for (uint32_t i = tid; i < kBins; i += kWholeThreads) sh.b.bins[i] = 0;
    sh.fill_octave();
    __syncthreads();
    uint32_t most = 0;
    for (uint32_t w = 0; w < kWholeThreads / 64; ++w) most = max(most, (uint32_t)sh.wave_u[w]);
    if (plain_row<B16>(row, a, r, s, most, sh)) return;
    if (a.vocab <= kBinnedVocab) {
        const Scale sc = scale_of(most, s.t);
        fill_bins<B16>(row, 0, a.vocab, sc, sh.b.bins);
        __syncthreads();
        const Bounds o = bounds_of<kWholeThreads>(s, sc, sh.b, sh);
        if (o.listed <= kList) {
            if (tid == 0) sh.found[7] = 0;
            __syncthreads();
            gather<B16>(row, 0, a.vocab, sc, o.floor, sh.b.wanted, sh.l.list, &sh.found[7]);
            __syncthreads();
            finish<kWholeThreads>(a, r, s, sc, o, sh.b, sh.l, sh);
            return;
        }
    }
    __syncthreads();
    by_digits<kWholeThreads, B16>(row, a, r, s, most, sh);
}

// A row in pieces, five launches: the largest key of each (and the row's bins and cursor cleared); the bins; the bounds; the
// listed tokens; the row's token.
template <bool B16>
__global__ __launch_bounds__(kPieceThreads) void piece_max_kernel(const SampleArgs a)
{
    __shared__ uint32_t waves[kPieceThreads / 64];
    const uint32_t r = blockIdx.y, c = blockIdx.x, begin = min(c * a.piece, a.vocab), end = min(begin + a.piece, a.vocab);
    for (uint32_t i = c * kPieceThreads + threadIdx.x; i < kBins; i += a.pieces * kPieceThreads) a.rows[r].b.bins[i] = 0;
    if (c == 0 && threadIdx.x == 0) a.rows[r].cursor = settings_of(a, r).greedy ? a.vocab : 0u;
    const uint32_t mine = largest_key<B16>(row_of<B16>(a, r), begin, end);
    if ((threadIdx.x & 63u) == 0) waves[threadIdx.x >> 6] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t most = 0;
        for (uint32_t w = 0; w < kPieceThreads / 64; ++w) most = max(most, waves[w]);
        a.piece_max[(uint64_t)r * a.pieces + c] = most;
    }
}

__device__ __forceinline__ uint32_t most_of_pieces(const SampleArgs& a, uint32_t r)
{
    uint32_t most = 0;
    for (uint32_t i = threadIdx.x & 63u; i < a.pieces; i += 64) most = max(most, a.piece_max[(uint64_t)r * a.pieces + i]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off));
    return most;
}

template <bool B16>
__global__ __launch_bounds__(kPieceThreads) void piece_bins_kernel(const SampleArgs a)
{
    __shared__ unsigned long long bins[kBins + kIdle];
    const uint32_t r = blockIdx.y, c = blockIdx.x, begin = min(c * a.piece, a.vocab), end = min(begin + a.piece, a.vocab);
    const uint32_t most = most_of_pieces(a, r);
    const Settings s = settings_of(a, r);
    if (most == 0 || s.greedy) return;
    for (uint32_t i = threadIdx.x; i < kBins; i += kPieceThreads) bins[i] = 0;
    __syncthreads();
    fill_bins<B16>(row_of<B16>(a, r), begin, end, scale_of(most, s.t), bins);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kBins; i += kPieceThreads)
        if (bins[i] != 0) atomicAdd(&a.rows[r].b.bins[i], bins[i]);
}

__global__ __launch_bounds__(kRowThreads) void row_bounds_kernel(const SampleArgs a)
{
    __shared__ Binned b;
    __shared__ Sums sh;
    const uint32_t r = blockIdx.x;
    const uint32_t most = most_of_pieces(a, r);
    const Settings s = settings_of(a, r);
    if (most == 0 || s.greedy) return;
    RowState& g = a.rows[r];
    for (uint32_t i = threadIdx.x; i < kBins; i += kRowThreads) b.bins[i] = g.b.bins[i];
    sh.fill_octave();
    __syncthreads();
    const Bounds o = bounds_of<kRowThreads>(s, scale_of(most, s.t), b, sh);
    for (uint32_t i = threadIdx.x; i < kBins; i += kRowThreads) {
        g.b.bins[i] = b.bins[i];
        g.b.before[i] = b.before[i];
        g.b.start[i] = b.start[i];
        if (i < kBins / 32) g.b.wanted[i] = b.wanted[i];
    }
    if (threadIdx.x == 0) g.o = o;
}

template <bool B16>
__global__ __launch_bounds__(kPieceThreads) void piece_list_kernel(const SampleArgs a)
{
    __shared__ uint64_t list[kList];
    __shared__ uint32_t wanted[kBins / 32], count, base;
    const uint32_t r = blockIdx.y, c = blockIdx.x, begin = min(c * a.piece, a.vocab), end = min(begin + a.piece, a.vocab);
    const void* row = row_of<B16>(a, r);
    const uint32_t most = most_of_pieces(a, r);
    const Settings s = settings_of(a, r);
    RowState& g = a.rows[r];
    if (most == 0) return;
    if (s.greedy) {
        if (a.piece_max[(uint64_t)r * a.pieces + c] == most) first_largest<B16>(row, begin, end, logit_of(most), &g.cursor);
        return;
    }
    if (g.o.listed > kList) return;
    // (atomics on a row's cursor for each token take turns across the whole GPU, for 2500 of them 50 us)
    if (threadIdx.x == 0) count = 0;
    if (threadIdx.x < kBins / 32) wanted[threadIdx.x] = g.b.wanted[threadIdx.x];
    __syncthreads();
    gather<B16>(row, begin, end, scale_of(most, s.t), g.o.floor, wanted, list, &count);
    __syncthreads();
    if (threadIdx.x == 0) base = count != 0 ? atomicAdd(&g.cursor, count) : 0u;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < count && base + i < kList; i += kPieceThreads) g.list[base + i] = list[i];
}

template <bool B16>
__global__ __launch_bounds__(kRowThreads) void row_token_kernel(const SampleArgs a)
{
    __shared__ Shared sh;
    const uint32_t r = blockIdx.x;
    const uint32_t most = most_of_pieces(a, r);
    const Settings s = settings_of(a, r);
    const RowState& g = a.rows[r];
    if (most == 0 || s.greedy) {
        if (threadIdx.x == 0) set_token(a, r, most == 0 ? -1 : (int32_t)g.cursor, most == 0 ? -__builtin_inff() : 0.0f);
        return;
    }
    const Bounds o = g.o;
    if (o.listed <= kList) {
        for (uint32_t i = threadIdx.x; i < o.listed; i += kRowThreads) sh.l.list[i] = g.list[i];
        finish<kRowThreads>(a, r, s, scale_of(most, s.t), o, g.b, sh.l, sh);
        return;
    }
    by_digits<kRowThreads, B16>(row_of<B16>(a, r), a, r, s, most, sh);
}

// Pieces per row; 1: a workgroup per row.  The pieces' five launches take 24 us at least; a workgroup takes 11 us and 0.35 us per
// thousand tokens, side by side with the other rows'.  Measured with pieces / whole (us, bf16, top-p alone):
//   1 row    32000 tokens 26 / 24, 48000 25 / 28, 128000 27 / 52, 200000 30 / 75
//   16 rows  32000 28 / 25, 48000 30 / 31, 64000 31 / 35, 128000 39 / 58;  32 rows  48000 33 / 31, 64000 35 / 36
//   64 rows  64000 38 / 36, 96000 42 / 47, 128000 45 / 58 (fp32 64000 38 / 37, 128000 49 / 63)
//   96 rows  64000 41 / 36, 96000 47 / 47, 128000 53 / 59;  128 rows  96000 51 / 49, 128000 59 / 60, 200000 89 / 99
//   160 rows 128000 68 / 62, 200000 102 / 100;  256 rows  200000 126 / 107
uint32_t pieces_of(int64_t rows, int64_t vocab)
{
    if (rows > 256 || vocab > kBinnedVocab || vocab < 40000 + 6 * rows * rows) return 1;
    const int64_t most = (vocab + 4095) / 4096, want = (512 + rows - 1) / rows;
    return (uint32_t)(want < most ? want : most);
}

}  // namespace

}  // namespace razer

using namespace razer;

static razer_status check_sample(const razer_sample_args* g)
{
    if (!g) return RAZER_ERR_NULL;
    if (g->dtype != RAZER_F32 && g->dtype != RAZER_BF16) return RAZER_ERR_CONFIG;
    if (g->rows < 0 || g->rows >= ((int64_t)1 << 22) || g->vocab < 1 || g->vocab > ((int64_t)1 << 24) || g->ld < g->vocab) return RAZER_ERR_SHAPE;
    if (g->rows == 0) return RAZER_OK;
    if (!g->logits || !g->uniform || !g->tokens) return RAZER_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(g->logits) % (g->dtype == RAZER_BF16 ? 2 : 4) != 0 || !aligned4(g->uniform) || !aligned4(g->temperature) || !aligned4(g->top_k) ||
        !aligned4(g->top_p) || !aligned4(g->min_p) || !aligned4(g->tokens) || !aligned4(g->logprobs))
        return RAZER_ERR_ALIGN;
    return RAZER_OK;
}

extern "C" {

size_t razer_sample_workspace_bytes(const razer_sample_args* g)
{
    if (check_sample(g) != RAZER_OK || g->rows == 0) return 0;
    const uint32_t pieces = pieces_of(g->rows, g->vocab);
    return pieces > 1 ? (size_t)g->rows * (sizeof(RowState) + (size_t)pieces * 4) : 0;
}

razer_status razer_sample(const razer_sample_args* g, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const razer_status s = check_sample(g);
    if (s != RAZER_OK || g->rows == 0) return s;
    const uint32_t pieces = pieces_of(g->rows, g->vocab);
    if (pieces > 1 && (!workspace || !aligned16(workspace) || workspace_bytes < razer_sample_workspace_bytes(g))) return RAZER_ERR_WORKSPACE;
    SampleArgs a{g->logits, g->uniform, g->temperature, g->top_k, g->top_p, g->min_p, g->tokens, g->logprobs, g->ld, (uint32_t)g->vocab, pieces, 0, nullptr, nullptr};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool b16 = g->dtype == RAZER_BF16;
    if (pieces > 1) {
        a.piece = (uint32_t)(((g->vocab + pieces - 1) / pieces + 7) & ~(int64_t)7);
        a.rows = static_cast<RowState*>(workspace);
        a.piece_max = reinterpret_cast<uint32_t*>(a.rows + g->rows);
        const dim3 grid(pieces, (uint32_t)g->rows);
        launch(b16 ? piece_max_kernel<true> : piece_max_kernel<false>, grid, kPieceThreads, 0, st, a);
        launch(b16 ? piece_bins_kernel<true> : piece_bins_kernel<false>, grid, kPieceThreads, 0, st, a);
        launch(row_bounds_kernel, (uint32_t)g->rows, kRowThreads, 0, st, a);
        launch(b16 ? piece_list_kernel<true> : piece_list_kernel<false>, grid, kPieceThreads, 0, st, a);
        launch(b16 ? row_token_kernel<true> : row_token_kernel<false>, (uint32_t)g->rows, kRowThreads, 0, st, a);
    } else {
        launch(b16 ? sample_kernel<true> : sample_kernel<false>, (uint32_t)g->rows, kWholeThreads, 0, st, a);
    }
    return hipGetLastError() == hipSuccess ? RAZER_OK : RAZER_ERR_HIP;
}

}  // extern "C"
