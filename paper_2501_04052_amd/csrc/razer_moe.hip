// Mixture-of-experts layer for a few tokens on stacked RaZeR weights (include/razer_step.h) for gfx950.
//
// Routing.  The router's product goes 32 elements at a time through v_mfma_f32_16x16x32_bf16; those partial sums (products
// of bf16 numbers, exact in fp32) are added up in 64 bits, so that which of two close experts is chosen does not hang on how K is cut.
//
// Bound by latency: one token with 64 experts of 4096 3.4 us, then 3.8 for the choice; 257 tokens with 160 of 5120 10 and 8 us.
//
// Experts.  The tokens' choices are grouped by expert into tiles of up to 4 NA rows, by a launch of its own or, up to 64 choices,
// by each wave for itself (3 us less for 19 tokens); a workgroup multiplies one tile with G
// groups of 16 weight rows, its waves taking the 128-k steps of K in turn, each with copies into LDS of its own as in
// razer_skinny.hip: codes, scale bytes and activations arrive in whole lines, are decoded once through byte tables and meet
// in v_mfma_f32_16x16x32_bf16.  The weights' bytes are what a call has to read: 5 tokens, 8 experts of 4096 -> 11008 -> 4096
// (464 MB) take 93-110 us, 4.2-5.0 TB/s; 64 tokens, 64 experts of 4096 -> 1408 -> 4096 (624 MB) 180 us, 3.5 TB/s, where copies,
// decoding and activations take turns (one of them left out at a time: 146-159 us of 176).
#include "razer_decode.hpp"
#include "razer_step.hpp"

namespace razer {

namespace {

// ------------------------------------------------------------------------------------------------ routing
struct RouteArgs {
    const uint16_t* x;
    const uint16_t* router;
    const void* logits;
    const float* bias;
    int32_t* ids;
    float* weights;
    double* partial;             // [slices][tokens][experts]
    int64_t ld_x, ld_logits, tokens;
    int hidden, experts, top_k, slices, sigmoid, renormalize, logits_bf16;
    float scale;
};

constexpr int kRouteWaves = 4, kRouteAhead = 4;  // waves of a workgroup; steps that a wave requests at once
constexpr int kRouteSlices = 10;

// A workgroup: 16 ET experts x 16 TT tokens over a slice of K, its waves a part of the slice each.  Bound by the loads of both
// operands from the caches: two by two fragments halve them, where there are workgroups enough without (route_fragments).
template <int ET, int TT>
__global__ __launch_bounds__(64 * kRouteWaves) void router_kernel(const RouteArgs a)
{
    __shared__ double part[kRouteWaves][64][4];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, r = lane & 15u, g = lane >> 4;
    const int e0 = blockIdx.x * 16 * ET;
    const int64_t t0 = (int64_t)blockIdx.y * 16 * TT;
    const uint16_t* w[ET];
    const uint16_t* x[TT];
#pragma unroll
    for (int i = 0; i < ET; ++i) w[i] = a.router + (int64_t)min(e0 + 16 * i + (int)r, a.experts - 1) * a.hidden + 8 * g;
#pragma unroll
    for (int i = 0; i < TT; ++i) {
        const int64_t t = t0 + 16 * i + r;
        x[i] = a.x + (t < a.tokens ? t : a.tokens - 1) * a.ld_x + 8 * g;
    }
    const int steps = a.hidden / 32, pieces = a.slices * kRouteWaves, piece = blockIdx.z * kRouteWaves + wave;
    const int begin = (int)((int64_t)steps * piece / pieces), end = (int)((int64_t)steps * (piece + 1) / pieces);
    double sum[ET][TT][4];
#pragma unroll
    for (int i = 0; i < ET * TT * 4; ++i) sum[i / (4 * TT)][i / 4 % TT][i % 4] = 0.0;
    for (int s = begin; s < end; s += kRouteAhead) {
        v8bf wf[kRouteAhead][ET], xf[kRouteAhead][TT];
#pragma unroll
        for (int j = 0; j < kRouteAhead; ++j) {                            // (steps past the end: the last one again, not added)
            const int at = s + j < end ? s + j : end - 1;
#pragma unroll
            for (int i = 0; i < ET; ++i) wf[j][i] = *reinterpret_cast<const v8bf*>(w[i] + 32 * at);
#pragma unroll
            for (int i = 0; i < TT; ++i) xf[j][i] = *reinterpret_cast<const v8bf*>(x[i] + 32 * at);
        }
#pragma unroll
        for (int j = 0; j < kRouteAhead; ++j) {
            // (a branch ahead of the products splits the requests: 3.4 against 3.7 us for one token; two by two fragments would
            // then take 126 registers for 68, and 13.2 us for 10.8)
            if (ET > 1 && s + j >= end) break;
            const bool in = ET > 1 || s + j < end;
#pragma unroll
            for (int ie = 0; ie < ET; ++ie)
#pragma unroll
                for (int it = 0; it < TT; ++it) {
                    const v4f p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[j][ie], xf[j][it], v4f{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[ie][it][i] += in ? (double)p[i] : 0.0;
                }
        }
    }
#pragma unroll
    for (int ie = 0; ie < ET; ++ie)
#pragma unroll
        for (int it = 0; it < TT; ++it) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i) part[wave][lane][i] = sum[ie][it][i];
            __syncthreads();
            // thread: token tid / 16, expert tid % 16 of the fragment
            const uint32_t tt = threadIdx.x >> 4, ee = threadIdx.x & 15u, from = (ee >> 2) * 16u + tt;
            double v = 0.0;
#pragma unroll
            for (int w4 = 0; w4 < kRouteWaves; ++w4) v += part[w4][from][ee & 3u];
            const int64_t t = t0 + 16 * it + tt;
            const int e = e0 + 16 * ie + (int)ee;
            if (t < a.tokens && e < a.experts) a.partial[((int64_t)blockIdx.z * a.tokens + t) * a.experts + e] = v;
        }
}
// Fragments of tokens and of experts per workgroup.  One by one / two by two, us of a call, by fragments in all: 64 experts, hidden 4096: 64
// tokens (16) 9.1 / 10.7, 128 (32) 9.5 / 11.0, 257 (68) 11.3 / 11.4, 512 (128) 13.0 / 12.3, 4096 (1024) 39.6 / 29.5; 160 experts, 5120: 64
// (40) 13.2 / 14.1, 96 (60) 14.3 / 14.3, 128 (80) 15.3 / 14.5, 257 (170) 21.0 / 17.3; 256 experts, 2048: 64 (64) 12.2 / 13.7.  Up to 16 experts leave
// half of the two empty: 8 experts, 8192 tokens (512) 22.3 / 24.7.  (A grid dimension holds 65535 fragments of 16 tokens.)
int route_fragments(int64_t tokens, int experts)
{
    const int64_t fragments = ((tokens + 15) / 16) * ((experts + 15) / 16);
    return (fragments > 64 && experts > 16) || tokens > ((int64_t)1 << 19) ? 2 : 1;
}

// An unsigned number in the order of a double (-0 below 0: sums that come out as one of them are 0 here)
__device__ __forceinline__ uint64_t ordered(double d)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, d + 0.0);
    return u ^ ((int64_t)u < 0 ? ~(uint64_t)0 : (uint64_t)1 << 63);
}
__device__ __forceinline__ double number_of(uint64_t u) { return __builtin_bit_cast(double, u ^ ((int64_t)u < 0 ? (uint64_t)1 << 63 : ~(uint64_t)0)); }
// the largest of the wave's, in every lane
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t larger(uint64_t v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xF, true);
    const uint64_t o = (uint64_t)hi << 32 | lo;
    return o > v ? o : v;
}
__device__ __forceinline__ uint64_t wave_largest(uint64_t v)
{
    v = larger<0x111, 0xF>(v);                                             // row_shr 1, 2, 4, 8, row_bcast 15, 31
    v = larger<0x112, 0xF>(v);
    v = larger<0x114, 0xF>(v);
    v = larger<0x118, 0xF>(v);
    v = larger<0x142, 0xA>(v);
    v = larger<0x143, 0xC>(v);
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
}
__device__ __forceinline__ double wave_total(double v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// One wave per token, expert 64 i + lane in place i of the lane.  The choices come one after the other: the largest key of all,
// then the first place that holds it.  0 is no key (taken, or no expert), 1 that of a NaN: behind -infinity's and all others.
template <int N>
__global__ __launch_bounds__(256) void select_kernel(const RouteArgs a)
{
    const uint32_t lane = threadIdx.x & 63u;
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.tokens) return;
    const double inf = __builtin_inf();
    double l[N];
    uint64_t key[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = 64 * i + (int)lane, from = e < a.experts ? e : a.experts - 1;
        if (a.partial) {
            double p[kRouteSlices];
#pragma unroll
            for (int s = 0; s < kRouteSlices; ++s)                         // (all requested before the first is waited for)
                p[s] = s < a.slices ? a.partial[((int64_t)s * a.tokens + t) * a.experts + from] : 0.0;
            l[i] = p[0];
#pragma unroll
            for (int s = 1; s < kRouteSlices; ++s) l[i] += p[s];
        } else {
            const int64_t at = t * a.ld_logits + from;
            l[i] = (double)(a.logits_bf16 ? bf16_bits_to_f32(static_cast<const uint16_t*>(a.logits)[at]) : static_cast<const float*>(a.logits)[at]);
        }
    }
    uint64_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = 64 * i + (int)lane;
        const bool number = l[i] == l[i];
        l[i] = e < a.experts && number ? fmin(l[i], 3.4028234663852886e38) : -inf;
        double k = a.sigmoid ? 1.0 / (1.0 + exp(-l[i])) : l[i];
        if (a.bias && e < a.experts) k += (double)a.bias[e];
        key[i] = e < a.experts ? (number && k == k ? ordered(k) : 1u) : 0u;
        const uint64_t o = ordered(l[i]);
        top = o > top ? o : top;
    }
    double most = 0.0, total = 1.0;                                        // of the logits: the largest, the sum of exponentials
    if (!a.sigmoid && !a.renormalize) {                                    // (else they cancel)
        most = number_of(wave_largest(top));
        total = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) total += l[i] > -inf ? exp(l[i] - most) : 0.0;
        total = wave_total(total);
    }
    double mine = -inf;                                                    // lane j: the j-th choice
    int id = 0;
    for (int j = 0; j < a.top_k; ++j) {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) best = key[i] > best ? key[i] : best;
        best = wave_largest(best);
        bool found = false;                                                // uniform
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t with = __ballot(key[i] == best);
            if (!found && with != 0) {
                found = true;
                const int from = __builtin_ctzll(with);
                const uint64_t b = __builtin_bit_cast(uint64_t, l[i]);
                const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, from), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), from);
                if ((int)lane == j) { mine = __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); id = 64 * i + from; }
                if ((int)lane == from) key[i] = 0;
            }
        }
    }
    double w;
    if (a.renormalize) {
        // relative to the best of the chosen, which may all be nothing beside others or beside 1.
        // 1 / (1 + exp(-l)) = exp(min(l, 0)) / (1 + exp(-|l|))
        double p = mine, q = 1.0;
        if (a.sigmoid) { p = fmin(mine, 0.0); q = 1.0 + exp(-fabs(mine)); }
        most = number_of(wave_largest(ordered(p)));                        // (lanes without a choice: -infinity)
        w = mine > -inf ? exp(p - most) / q : 0.0;
        const double sum = wave_total(w);
        w = sum > 0.0 ? w / sum : 0.0;
    } else {
        w = !(mine > -inf) ? 0.0 : a.sigmoid ? 1.0 / (1.0 + exp(-mine)) : exp(mine - most) / total;
    }
    if ((int)lane < a.top_k) {
        a.ids[t * a.top_k + lane] = id;
        a.weights[t * a.top_k + lane] = (float)(w * (double)a.scale);
    }
}

int route_slices(int64_t tokens, int experts, int hidden)
{
    const int side = 16 * route_fragments(tokens, experts);
    const int64_t tiles = ((tokens + side - 1) / side) * ((experts + side - 1) / side), steps = hidden / 32;
    // enough waves to cover the way to memory, none with less than it requests at once
    int64_t s = (1024 + tiles - 1) / tiles;
    if (s > kRouteSlices) s = kRouteSlices;
    if (s > steps / (kRouteWaves * kRouteAhead)) s = steps / (kRouteWaves * kRouteAhead);
    return (int)(s < 1 ? 1 : s);
}

// ------------------------------------------------------------------------------------------------ experts
struct Tile {
    int32_t expert, start, count, spare;     // choices list[start .. start + count)
};

// One projection's weights as the kernels take them.
struct Stack {
    const uint8_t* codes;
    const uint8_t* scales;
    const float* ts;
};

struct ExpertArgs {
    Stack w[2];                  // gate and up, or down
    const Tile* tiles;           // NULL: 64 choices at most, and no plan
    const int32_t* tile_count;
    const int32_t* list;         // choices (token top_k + place), grouped by expert
    const int32_t* ids;
    int experts, choices;
    const uint8_t* act;          // x, or what stands between the products [choices][inter]
    void* out;                   // bf16 or fp32 [choices][rows]
    const float* weights;
    int64_t code_stride, scale_stride;      // bytes of one expert
    uint32_t k, rows;
    int64_t act_ld;              // bytes, a multiple of 16
    float sv0, sv1;
    int top_k, lb, act_kind, waves;
};

// Groups the choices by expert.  Which place a choice gets among those of its expert is a matter of chance and leaves no
// trace: a tile's rows do not influence each other.
__global__ __launch_bounds__(1024) void plan_kernel(const int32_t* __restrict__ ids, int count, int experts, int rows, Tile* __restrict__ tiles,
                                                    int32_t* __restrict__ tile_count, int32_t* __restrict__ list)
{
    __shared__ int32_t n[1024], at[1024];
    __shared__ int32_t wave_n[16], wave_t[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    n[tid] = 0;
    __syncthreads();
    for (int i = tid; i < count; i += 1024) {
        const int e = ids[i];
        if (e >= 0 && e < experts) atomicAdd(&n[e], 1);
    }
    __syncthreads();
    const int mine = n[tid], my_tiles = (mine + rows - 1) / rows;
    int rn = mine, rt = my_tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int on = __shfl_up(rn, d), ot = __shfl_up(rt, d);
        if (lane >= d) { rn += on; rt += ot; }
    }
    if (lane == 63) { wave_n[wave] = rn; wave_t[wave] = rt; }
    __syncthreads();
    int start = rn - mine, tile = rt - my_tiles;
    for (int w = 0; w < wave; ++w) { start += wave_n[w]; tile += wave_t[w]; }
    at[tid] = start;
    for (int i = 0; i < my_tiles; ++i) tiles[tile + i] = Tile{tid, start + i * rows, min(rows, mine - i * rows), 0};
    if (tid == 1023) *tile_count = tile + my_tiles;
    __syncthreads();
    for (int i = tid; i < count; i += 1024) {
        const int e = ids[i];
        if (e >= 0 && e < experts) list[atomicAdd(&at[e], 1)] = i;
    }
}

__device__ __forceinline__ float activate(float z, int kind)
{
    if (kind == RAZER_RELU) return z < 0.0f ? 0.0f : z;                    // (a NaN stays one)
    // gelu: 0.5 (1 + tanh(u)) = 1 / (1 + exp(-2 u))
    const float v = kind == RAZER_SILU ? z : 1.5957691216057308f * __builtin_fmaf(0.044715f * z * z, z, z);
    return z / (1.0f + expf(-v));
}

enum { kGated = 0, kPlain = 1, kDown = 2 };

// What stands between the products is kept in two bf16 parts, the second one what the first leaves of 32 bits: the output's own
// rounding to bf16 is then all that is lost, whatever the number of tokens, where one part makes the error sqrt(2) times that, and
// more where few values carry the sum.  Weights are decoded once for both parts (one part, then two: 1 token 15.6 and 16.0 us, 5
// tokens of 16 experts 101 and 105, 64 tokens of 64 experts 168 and 182; with the launch shapes of either: 64 tokens of 8
// experts 4096 -> 1408 -> 4096 39 and 46, 512 of 64 529 and 528, 2048 of 64 1599 and 1676).
template <int MODE>
constexpr int parts() { return MODE == kDown ? 2 : 1; }

template <int NA, int G, int MODE>
constexpr uint32_t wave_bytes()
{
    const uint32_t slot = parts<MODE>() * NA * 1024u + G * 1280u, part = G * ((NA + 3) / 4) * 1024u;
    return slot > part ? slot : part;
}

#define RAZER_COPY(src, off, dst, bytes)                                                                           \
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)((src) + (off)),              \
                                     (__attribute__((address_space(3))) void*)(dst), bytes, 0, 0)
#define RAZER_DS128(dst, addr, imm) asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(imm))
#define RAZER_DS16(dst, addr, imm) asm volatile("ds_read_u16 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(imm))

// Steps that a wave has under way.  One token: few waves, each with few steps, all of which are requested at once.
template <int NA, int MODE>
constexpr int depth() { return NA == 1 && MODE != kDown ? 2 : 1; }

// NA: activation KiB per step (tiles of 4 NA rows), G: groups of 16 weight rows (kGated: half of them gate's, half up's).
template <int NA, int G, bool GB, int MODE>
__global__ __launch_bounds__(512) void expert_kernel(const ExpertArgs arg)
{
    constexpr int NB = (NA + 3) / 4;
    constexpr bool ONE = NA == 1 && MODE != kDown;                        // (launch_expert: one token)
    constexpr int D = depth<NA, MODE>();
    constexpr int NP = parts<MODE>();
    constexpr uint32_t ACT = NP * NA * 1024u, SLOT = wave_bytes<NA, G, MODE>(), WAVE = D * SLOT;
    __shared__ uint4 lut[256];
    extern __shared__ __align__(16) uint8_t dyn_smem[];                   // [waves][D][SLOT]
    const uint32_t lane = threadIdx.x & 63u, nwaves = (uint32_t)arg.waves;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t expert = -1, count = 0, mine_choice = 0;                      // lane j: the tile's j-th choice
    uint8_t* const mine = dyn_smem + wave * WAVE;
    if constexpr (ONE) {
        const int32_t e = arg.ids[blockIdx.y];
        if (e < 0 || e >= arg.experts) return;
        expert = e;
        count = 1;
        mine_choice = (int32_t)blockIdx.y;
    } else if (!arg.tiles) {
        // a choice in each lane: the experts in the order in which they first occur, until the tile's comes
        constexpr int R = 4 * NA;
        const int32_t id = (int)lane < arg.choices ? arg.ids[lane] : -1;
        uint64_t left = __ballot(id >= 0 && id < arg.experts), with = 0;
        int skip = (int)blockIdx.y;
        while (left != 0) {
            expert = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
            with = __ballot(id == expert);
            const int tiles = (__builtin_popcountll(with) + R - 1) / R;
            if (skip < tiles) break;
            skip -= tiles;
            left &= ~with;
        }
        if (left == 0) return;
        const int place = __builtin_popcountll(with & (((uint64_t)1 << lane) - 1)) - skip * R;
        count = __builtin_popcountll(with) - skip * R;
        count = count < R ? count : R;
        int32_t* chosen = reinterpret_cast<int32_t*>(mine);               // (this wave's, before its copies come there)
        if ((with >> lane & 1u) && place >= 0 && place < R) chosen[place] = (int32_t)lane;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        mine_choice = chosen[(int)lane < count ? lane : 0u];
    } else {
        if ((int)blockIdx.y >= *arg.tile_count) return;
        const Tile tile = arg.tiles[blockIdx.y];
        expert = tile.expert;
        count = tile.count;
        mine_choice = arg.list[tile.start + ((int)lane < count ? lane : 0u)];
    }
    const uint32_t r = lane & 15u, g = lane >> 4;
    const uint32_t kk = arg.k, nsteps = (kk + 127u) >> 7, code_ld = kk >> 1, scale_ld = kk >> (GB ? arg.lb : 4);
    const int lb = arg.lb;

    // copy lanes: codes and scale bytes -- row lane / 4, 16-byte chunk / 32-element run; activations -- row 4 i + lane / 16
    const uint32_t wr = lane >> 2, wp = lane & 3u, wc = wp ^ ((wr >> 2) & 3u);
    const uint8_t* cbase[G];
    const uint8_t* sbase[G];
    uint32_t row_of[G];
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
        const int m = MODE == kGated ? gi & 1 : 0;
        const uint32_t q = MODE == kGated ? blockIdx.x * (G / 2) + gi / 2 : blockIdx.x * G + gi;
        row_of[gi] = q * 16u;
        const uint32_t row0 = min(row_of[gi], arg.rows - 16u);            // groups past the last one re-read it, never stored
        cbase[gi] = arg.w[m].codes + (int64_t)expert * arg.code_stride + (int64_t)row0 * code_ld;
        sbase[gi] = arg.w[m].scales + (int64_t)expert * arg.scale_stride + (int64_t)row0 * scale_ld;
    }
    const uint32_t crow = wr * code_ld, srow = wr * scale_ld;
    // (rows in chunks of 16 bytes: at most tokens * ld_x / 8 < 2^28 and choices * inter * 2 parts / 8 < 2^29; in bytes they may
    // pass 2^32)
    const uint32_t act_ld = (uint32_t)(arg.act_ld >> 4);
    uint32_t arow[NA], achk[NA];
#pragma unroll
    for (int i = 0; i < NA; ++i) {
        const uint32_t row = 4u * i + (lane >> 4), choice = (uint32_t)__shfl(mine_choice, (int)min(row, (uint32_t)count - 1u));
        arow[i] = (ONE ? 0u : MODE == kDown ? choice : choice / (uint32_t)arg.top_k) * act_ld;
        achk[i] = (lane & 15u) ^ (row & 15u);                             // logical 16-byte chunk this lane fetches
    }
    auto issue = [&](uint32_t step, uint32_t slot) {
        const bool full = 128u * step + 128u <= kk;                       // uniform
        const uint32_t left = kk - 128u * step;                           // elements of this step inside K (>= 32)
        uint8_t* ring = mine + slot;
        const uint32_t wcc = full || wc * 32u < left ? wc : 0u, wpp = full || wp * 32u < left ? wp : 0u;
#pragma unroll
        for (int gi = 0; gi < G; ++gi) RAZER_COPY(cbase[gi] + (size_t)step * 64u, crow + wcc * 16u, ring + ACT + gi * 1024, 16);
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
            if constexpr (GB) RAZER_COPY(sbase[gi], srow + ((128u * step + 32u * wpp) >> lb), ring + ACT + G * 1024 + gi * 256, 1);
            else RAZER_COPY(sbase[gi] + (size_t)step * 8u, srow + wpp * 2u, ring + ACT + G * 1024 + gi * 256, 2);
        }
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (i == 0 || 4 * i < count)                                  // (rows behind the last one: whatever is there, for columns that nobody reads)
#pragma unroll
                for (int h = 0; h < NP; ++h)
                    RAZER_COPY(arg.act + (size_t)step * 256u, (size_t)(arow[i] + h * (kk / 8u) + (full || achk[i] * 8u < left ? achk[i] : 0u)) << 4,
                               ring + (h * NA + i) * 1024, 16);
    };
    const uint32_t ring_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)mine;
    const uint32_t lut_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4*)lut;
    const uint32_t code_lds = ring_lds + ACT + r * 64u + ((g ^ ((r >> 2) & 3u)) << 4);
    const uint32_t scale_lds = ring_lds + ACT + G * 1024u + (4u * r + g) * 4u;
    const uint32_t ra = NA < 4 ? r & (4u * NA - 1u) : r;
    uint32_t a_lds[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) a_lds[j] = ring_lds + ra * 256u + (((4u * g + j) ^ ra) << 4);

    uint32_t step = wave;                                                 // (the host starts no more waves than there are steps)
    uint32_t slot = 0;
    // (what the end needs is asked for here: its way from memory would be the last thing a workgroup waits for)
    const float my_weight = MODE == kDown ? arg.weights[mine_choice] : 0.0f;
    issue(step, 0u);
    if (D == 2 && step + nwaves < nsteps) issue(step + nwaves, SLOT);
    float s0 = *(const __attribute__((address_space(4))) float*)(uintptr_t)(arg.w[0].ts + expert), s1 = 0.0f;
    if constexpr (MODE == kGated) s1 = *(const __attribute__((address_space(4))) float*)(uintptr_t)(arg.w[1].ts + expert);
    for (uint32_t sb = threadIdx.x; sb < 256u; sb += 64u * nwaves) {
        const v4u e = __builtin_bit_cast(v4u, sk_byte_table(sb, arg.sv0, arg.sv1));
        asm volatile("ds_write_b128 %0, %1" ::"v"(lut_lds + sb * 16u), "v"(e) : "memory");
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    asm volatile("" : "+s"(s0), "+s"(s1));                                // (loaded by here, not at their use)
    v4f acc[G][NB];
#pragma unroll
    for (int gi = 0; gi < G; ++gi)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[gi][b] = v4f{0.f, 0.f, 0.f, 0.f};

    while (step < nsteps) {
        v4u cw[G], le[G][GB ? 1 : 2], af[NP * NB][4];                     // (block h NB + b: part h of columns 16 b ..)
        uint32_t sw[G];
        // what this step reads has landed (D == 2: the next one's 2 G + NA copies may be under way)
        if (D == 2 && step + nwaves < nsteps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * G + NA) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
            RAZER_DS16(sw[gi], scale_lds + slot, gi * 256);
            RAZER_DS128(cw[gi], code_lds + slot, gi * 1024);
        }
#pragma unroll
        for (int b = 0; b < NP * NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) RAZER_DS128(af[b][j], a_lds[j] + slot, (b / NB) * NA * 1024 + (b % NB) * 4096);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int gi = 0; gi < G; ++gi) asm volatile("" : "+v"(cw[gi]), "+v"(sw[gi]));
#pragma unroll
        for (int b = 0; b < NP * NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(af[b][j]));
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
            RAZER_DS128(le[gi][0], lut_lds + (sw[gi] & 255u) * 16u, 0);
            if constexpr (!GB) RAZER_DS128(le[gi][1], lut_lds + (sw[gi] >> 8) * 16u, 0);
        }
        // (everything that the copies overwrite has been read)
        if (step + D * nwaves < nsteps) issue(step + D * nwaves, slot);
        if (D == 2) slot ^= SLOT;
        if (128u * step + 128u > kk) {                                    // ragged last step: activations past K are 0 (0 x Inf is not)
            const uint32_t keep = (128u * step + 32u * g < kk) ? 0xFFFFFFFFu : 0u;
#pragma unroll
            for (int b = 0; b < NP * NB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) af[b][j] &= keep;
        }
#pragma unroll
        for (int b = 0; b < NP * NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) af[b][j] = sk_permute_pairs(af[b][j]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
            asm volatile("" : "+v"(le[gi][0]));
            if constexpr (!GB) asm volatile("" : "+v"(le[gi][1]));
        }
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const v8bf wf = sk_decode_dword_table(cw[gi][j], le[gi][(GB || j < 2) ? 0 : 1]);
#pragma unroll
                for (int b = 0; b < NP * NB; ++b)
                    acc[gi][b % NB] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, __builtin_bit_cast(v8bf, af[b][j]), acc[gi][b % NB], 0, 0, 0);
            }
        }
        step += nwaves;
    }
    // partial sums in the wave's own ring (all its copies have landed and been read)
    float4* part = reinterpret_cast<float4*>(mine);
#pragma unroll
    for (int gi = 0; gi < G; ++gi)
#pragma unroll
        for (int b = 0; b < NB; ++b) part[(gi * NB + b) * 64 + lane] = make_float4(acc[gi][b][0], acc[gi][b][1], acc[gi][b][2], acc[gi][b][3]);
    __syncthreads();
    auto total = [&](uint32_t u) {
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        for (uint32_t w = 0; w < nwaves; ++w) {
            const float4 p = *reinterpret_cast<const float4*>(dyn_smem + w * WAVE + (u * 64u + lane) * 16u);
            t.x += p.x; t.y += p.y; t.z += p.z; t.w += p.w;
        }
        return t;
    };
    // a unit is one fragment of an output group: lane l holds weight rows 4 (l / 16) + 0..3 of it, tile row 16 b + l % 16
    constexpr int UNITS = (MODE == kGated ? G / 2 : G) * NB;
    for (uint32_t u = wave; u < (uint32_t)UNITS; u += nwaves) {
        const uint32_t p = u / NB, b = u % NB, col = 16u * b + r;
        const uint32_t q = MODE == kGated ? blockIdx.x * (G / 2) + p : blockIdx.x * G + p, row = q * 16u + 4u * g;
        const int32_t choice = __shfl(mine_choice, (int)col);
        if constexpr (MODE == kDown) {
            const float4 t = total(u);
            const float w = __shfl(my_weight, (int)col);
            if (col < (uint32_t)count && row < arg.rows) {
                *reinterpret_cast<float4*>(static_cast<float*>(arg.out) + (int64_t)choice * arg.rows + row) =
                    make_float4(s0 * t.x * w, s0 * t.y * w, s0 * t.z * w, s0 * t.w * w);
            }
        } else {
            const float4 t = total(MODE == kGated ? 2 * p * NB + b : u);
            float v[4] = {activate(s0 * t.x, arg.act_kind), activate(s0 * t.y, arg.act_kind), activate(s0 * t.z, arg.act_kind), activate(s0 * t.w, arg.act_kind)};
            if constexpr (MODE == kGated) {
                const float4 o = total((2 * p + 1) * NB + b);
                v[0] *= s1 * o.x; v[1] *= s1 * o.y; v[2] *= s1 * o.z; v[3] *= s1 * o.w;
            }
            if (col < (uint32_t)count && row < arg.rows) {
                const uint32_t lo = (uint32_t)f32_to_bf16_rne(v[0]) | ((uint32_t)f32_to_bf16_rne(v[1]) << 16);
                const uint32_t hi = (uint32_t)f32_to_bf16_rne(v[2]) | ((uint32_t)f32_to_bf16_rne(v[3]) << 16);
                uint16_t* out = static_cast<uint16_t*>(arg.out) + (int64_t)choice * parts<kDown>() * arg.rows + row;
                *reinterpret_cast<uint2*>(out) = make_uint2(lo, hi);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float first = __builtin_bit_cast(float, (uint32_t)f32_to_bf16_rne(v[i]) << 16);
                    v[i] = fabsf(first) < __builtin_inff() ? v[i] - first : 0.0f;           // (Inf and NaN: the first part alone)
                }
                const uint32_t lo2 = (uint32_t)f32_to_bf16_rne(v[0]) | ((uint32_t)f32_to_bf16_rne(v[1]) << 16);
                const uint32_t hi2 = (uint32_t)f32_to_bf16_rne(v[2]) | ((uint32_t)f32_to_bf16_rne(v[3]) << 16);
                *reinterpret_cast<uint2*>(out + arg.rows) = make_uint2(lo2, hi2);
            }
        }
    }
}

// One token's down products, summed over its experts at once: the waves take the steps of all of them in turn, a step's
// product is added with its expert's tensor scale and routing weight.  With one activation row the matrix instruction has
// columns to spare: of its 16 rows eight are weight rows over a step's first 128 k and eight the same weight rows over its second
// 128; columns 0 and 1 hold the two halves' activations, columns 2 and 3 what the bf16 of those left, and all are added at the end.  So a workgroup
// has 8 rows, twice as many compute units have one, and nothing is decoded twice (2048 rows, 8 experts of 1024: 16 rows
// on half of the units 9.4 us).  Bound by the issue of decode instructions, then by the start and end of one round.
constexpr uint32_t kOneDepth = 4, kOneRows = 8, kOneSlot = 1024u + 1024u + 256u;   // a slot: activations, codes, scale entries
template <bool GB>
__global__ __launch_bounds__(1024) void one_down_kernel(const ExpertArgs arg)
{
    constexpr uint32_t D = kOneDepth, ACT = 1024u, SLOT = kOneSlot, WAVE = D * SLOT;
    __shared__ uint4 lut[256];
    extern __shared__ __align__(16) uint8_t dyn_smem[];                   // [waves][D][SLOT]
    const uint32_t lane = threadIdx.x & 63u, nwaves = (uint32_t)arg.waves;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t r = lane & 15u, g = lane >> 4;
    const uint32_t kk = arg.k, nsteps = (kk + 255u) >> 8, code_ld = kk >> 1, scale_ld = kk >> (GB ? arg.lb : 4);
    const uint32_t all = nsteps * (uint32_t)arg.top_k, row0 = blockIdx.x * kOneRows;
    const int lb = arg.lb;
    // copy lanes: codes and scale bytes -- matrix row lane / 4 (weight row (lane / 4) % 8, half lane / 32), 16-byte chunk / run of 32
    // elements; activations -- part lane / 32, half (lane / 16) % 2
    const uint32_t wr = lane >> 2, wp = lane & 3u, wc = wp ^ ((wr >> 2) & 3u), wh = lane >> 5;
    const uint32_t crow = (wr & 7u) * code_ld, srow = (wr & 7u) * scale_ld, achk = (lane & 15u) ^ (lane >> 4);
    uint8_t* const mine = dyn_smem + wave * WAVE;
    const uint32_t ring_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)mine;
    const uint32_t lut_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4*)lut;
    // lane j: the j-th choice's expert and factor
    const int32_t id = (int)lane < arg.top_k ? arg.ids[lane] : -1;
    const bool valid = id >= 0 && id < arg.experts;
    const uint64_t valids = __ballot(valid);
    const int32_t my_expert = valid ? id : 0;
    const float factor = valid ? arg.w[0].ts[my_expert] * arg.weights[lane] : 0.0f;
    // a step's three copies (a choice without an expert: some expert's, for nothing); what lies past K is the step's first
    auto issue = [&](uint32_t choice, uint32_t step, uint32_t slot) {
        const int32_t e = __builtin_amdgcn_readlane(my_expert, (int)choice);
        uint8_t* ring = mine + slot;
        const uint32_t left = kk - 256u * step;                           // elements from the step's first on
        const uint32_t we = 128u * wh + 32u * wc, wq = 128u * wh + 32u * wp, ae = 128u * ((lane >> 4) & 1u) + 8u * achk;
        const uint8_t* codes = arg.w[0].codes + e * arg.code_stride + (int64_t)row0 * code_ld;
        const uint8_t* scales = arg.w[0].scales + e * arg.scale_stride + (int64_t)row0 * scale_ld;
        const uint8_t* act = arg.act + (int64_t)choice * arg.act_ld;
        RAZER_COPY(codes + (size_t)step * 128u, crow + (we < left ? we : 0u) / 2u, ring + ACT, 16);
        if constexpr (GB) RAZER_COPY(scales, srow + ((256u * step + (wq < left ? wq : 0u)) >> lb), ring + ACT + 1024, 1);
        else RAZER_COPY(scales + (size_t)step * 16u, srow + (wq < left ? wq : 0u) / 16u, ring + ACT + 1024, 2);
        RAZER_COPY(act + (size_t)step * 512u, (lane >> 5) * (2u * kk) + (ae < left ? ae : 0u) * 2u, ring, 16);
    };
    const uint32_t code_lds = ring_lds + ACT + r * 64u + ((g ^ ((r >> 2) & 3u)) << 4);
    const uint32_t scale_lds = ring_lds + ACT + 1024u + (4u * r + g) * 4u;
    const uint32_t half = r & 1u, arow = r & 3u;                          // of this lane's column
    uint32_t a_lds[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) a_lds[j] = ring_lds + arow * 256u + (((4u * g + j) ^ arow) << 4);

    // this wave's steps are wave, wave + nwaves, ... of all (the host starts no more waves than there are): choice and step of
    // the next to be requested and of the next to be multiplied
    auto advance = [&](uint32_t& choice, uint32_t& step) {
        step += nwaves;
        while (step >= nsteps) { step -= nsteps; ++choice; }
    };
    uint32_t ic = 0, is = wave, slot = 0;
    while (is >= nsteps) { is -= nsteps; ++ic; }
    uint32_t choice = ic, step = is;
#pragma unroll
    for (uint32_t d = 0; d < D; ++d) {
        if (wave + d * nwaves < all) {
            issue(ic, is, d * SLOT);
            advance(ic, is);
        }
    }
    for (uint32_t sb = threadIdx.x; sb < 256u; sb += 64u * nwaves) {
        const v4u t = __builtin_bit_cast(v4u, sk_byte_table(sb, arg.sv0, arg.sv1));
        asm volatile("ds_write_b128 %0, %1" ::"v"(lut_lds + sb * 16u), "v"(t) : "memory");
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    v4f sum = v4f{0.f, 0.f, 0.f, 0.f};
    for (uint32_t s = wave; s < all; s += nwaves) {
        const float coef = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, factor), (int)choice));
        v4u cw, le[GB ? 1 : 2], af[4];
        uint32_t sw;
        // what this step reads has landed: the steps behind it, three copies each, may be under way
        if (s + 3 * nwaves < all) asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
        else if (s + 2 * nwaves < all) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
        else if (s + nwaves < all) asm volatile("s_waitcnt vmcnt(3)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        static_assert(D == 4, "the waits above");
        RAZER_DS16(sw, scale_lds + slot, 0);
        RAZER_DS128(cw, code_lds + slot, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) RAZER_DS128(af[j], a_lds[j] + slot, 0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        asm volatile("" : "+v"(cw), "+v"(sw));
#pragma unroll
        for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(af[j]));
        RAZER_DS128(le[0], lut_lds + (sw & 255u) * 16u, 0);
        if constexpr (!GB) RAZER_DS128(le[1], lut_lds + (sw >> 8) * 16u, 0);
        if (s + D * nwaves < all) {
            issue(ic, is, slot);
            advance(ic, is);
        }
        slot = slot + SLOT < WAVE ? slot + SLOT : 0u;
        if (256u * step + 256u > kk) {                                    // activations past K are 0 (0 x Inf is not)
            const uint32_t keep = 256u * step + 128u * half + 32u * g < kk ? 0xFFFFFFFFu : 0u;
#pragma unroll
            for (int j = 0; j < 4; ++j) af[j] &= keep;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) af[j] = sk_permute_pairs(af[j]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        asm volatile("" : "+v"(le[0]));
        if constexpr (!GB) asm volatile("" : "+v"(le[1]));
        v4f acc = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sk_decode_dword_table(cw[j], le[(GB || j < 2) ? 0 : 1]), __builtin_bit_cast(v8bf, af[j]), acc, 0, 0, 0);
        if (valids >> choice & 1u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(coef, acc[i], sum[i]);
        }
        advance(choice, step);
    }
    // matrix rows 4 g .. 4 g + 3: the first half's in columns 0 and 2, the second half's (g >= 2) in columns 1 and 3
    float4* part = reinterpret_cast<float4*>(mine);
    if (r < 4u && half == g / 2u) part[(r >> 1) * 4u + g] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    __syncthreads();
    if (threadIdx.x < kOneRows) {
        float t = 0.0f;
        for (uint32_t w = 0; w < nwaves; ++w) {
            const float* p = reinterpret_cast<const float*>(dyn_smem + w * WAVE) + threadIdx.x;
            t += (p[0] + p[kOneRows]) + (p[2 * kOneRows] + p[3 * kOneRows]);
        }
        static_cast<uint16_t*>(arg.out)[row0 + threadIdx.x] = f32_to_bf16_rne(t);
    }
}

#undef RAZER_DS128
#undef RAZER_DS16
#undef RAZER_COPY

// y[t] = sum of the token's experts' outputs, in the order of its choices
__global__ __launch_bounds__(256) void combine_kernel(const float* __restrict__ partial, const int32_t* __restrict__ ids, int experts, int top_k, int64_t rows,
                                                      uint16_t* __restrict__ y, int64_t ld_y)
{
    const int64_t t = blockIdx.x, c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
    if (c >= rows) return;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int j = 0; j < top_k; ++j) {
        const int e = ids[t * top_k + j];
        if (e < 0 || e >= experts) continue;
        const float4 p = *reinterpret_cast<const float4*>(partial + (t * top_k + j) * rows + c);
        s.x += p.x; s.y += p.y; s.z += p.z; s.w += p.w;
    }
    const uint32_t lo = (uint32_t)f32_to_bf16_rne(s.x) | ((uint32_t)f32_to_bf16_rne(s.y) << 16);
    const uint32_t hi = (uint32_t)f32_to_bf16_rne(s.z) | ((uint32_t)f32_to_bf16_rne(s.w) << 16);
    *reinterpret_cast<uint2*>(y + t * ld_y + c) = make_uint2(lo, hi);
}

// ------------------------------------------------------------------------------------------------ host
struct MoePlan {
    int na;                      // activation KiB per step
    int64_t choices, tiles;      // tiles: at most
    size_t list, mid, out, bytes;    // offsets into the workspace; tile count and tiles stand at its front
};

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Tiles of 16 rows up to 12 choices per expert, of 32 beyond that (us with 16, 32 and 64 rows; 4096 -> 1408 -> 4096):
//   12 choices each, 8 experts 38 / 44 / 66, 64 experts 202 / 219 / 391;  16 each 49 / 46 / 67 and 247 / 226 / 400;  64 each 92 / 86 / 95 and
//   620 / 540 / 684;  256 each, 64 experts 2109 / 1713 / 2057.  Two to eight tokens: tiles of 8.
MoePlan plan_of(int64_t tokens, int top_k, int experts, int64_t inter, int64_t rows)
{
    MoePlan p;
    p.choices = tokens * top_k;
    p.na = tokens == 1 ? 1 : tokens <= 8 ? 2 : p.choices / experts <= 12 ? 4 : 8;
    p.tiles = (p.choices < experts ? p.choices : experts) + p.choices / (4 * p.na);
    p.list = up256(16 + (size_t)(p.choices + p.choices / 4) * sizeof(Tile));     // (more than any number of rows per tile gives)
    p.mid = up256(p.list + (size_t)p.choices * 4);
    p.out = up256(p.mid + (size_t)p.choices * inter * 2 * parts<kDown>());
    p.bytes = up256(p.out + (size_t)p.choices * rows * 4);
    return p;
}

template <int NA, int G, bool GB, int MODE>
hipError_t launch_expert_t(ExpertArgs a, int64_t tiles, hipStream_t st)
{
    const uint32_t nsteps = (a.k + 127) / 128;
    // (several tokens: there are workgroups enough, four waves share the steps more evenly.  64 tokens, 64 experts, 4096 -> 1408
    // -> 4096: 8 waves 174 us, 4 waves 168, 2 waves 198; one token: 8 waves 18.9, 4 19.2, 2 21.4.
    //   The down product of four groups keeps two parts in LDS, so that few workgroups fit a compute unit: few waves leave room for more.
    // us with 2 / 3 / 4 waves, 4096 -> inter -> 4096, tiles of 16 rows, 64 tokens of 64 experts: 704 103 / 106 / 111, 1408
    // 188 / 189 / 189, 2816 350 / 346 / 341, 8192 1017 / 974 / 939; tiles of 32, 128 tokens of 64 experts: 704 137 / 143 / 182, 1408
    // 225 / 234 / 271, 2816 430 / 440 / 484, 4096 614 / 610 / 650; 64 tokens of 8: 1408 46 / 43 / 46, 4096 91 / 81 / 83, 14336 311 / 275 / 272)
    const uint32_t most = NA == 1 ? 8 : G < 4 || MODE != kDown ? 4 : NA == 4 ? (nsteps < 11 ? 2 : 4) : nsteps < 16 ? 2 : 3;
    const uint32_t waves = nsteps < most ? nsteps : most;
    a.waves = (int)waves;
    constexpr uint32_t WAVE = depth<NA, MODE>() * wave_bytes<NA, G, MODE>(), smem = (NA == 1 ? 8 : 4) * WAVE;
    RAZER_RAISE_LDS_LIMIT((expert_kernel<NA, G, GB, MODE>), smem);
    const uint32_t groups = a.rows / 16, per = MODE == kGated ? G / 2 : G;
    launch(expert_kernel<NA, G, GB, MODE>, dim3((groups + per - 1) / per, (uint32_t)tiles), 64 * waves, waves * WAVE, st, a);
    return hipGetLastError();
}
template <int NA, int MODE>
hipError_t launch_expert_g(const ExpertArgs& a, int64_t tiles, hipStream_t st)
{
    // four groups of rows per workgroup halve the copies of activations per weight, where that leaves enough workgroups (us with two /
    // four, hidden -> inter -> hidden, workgroups of the down product at two groups in brackets: 64 tokens of 8 experts x 2 512 -> 512 (160) 17 / 20, 64 of 16 x 4
    // 1024 -> 1024 (1024) 30 / 30, 64 of 64 x 8 512 -> 512 (1536) 30 / 28, 4096 -> 1408 (12288) 199 / 187, 64 of 16 x 8 4096 -> 4096 (6144) 251 / 228, 1024 ->
    // 1024 (1536) 42 / 41, 128 of 8 x 2 1024 -> 1024 (512) 26 / 29, 2048 -> 1408 (1024) 45 / 48)
    const bool gb = a.lb != 4, four = NA > 2 && (int64_t)(a.rows / 16) * tiles >= 2048;
    if constexpr (NA > 2)
        if (four) return gb ? launch_expert_t<NA, 4, true, MODE>(a, tiles, st) : launch_expert_t<NA, 4, false, MODE>(a, tiles, st);
    return gb ? launch_expert_t<NA, 2, true, MODE>(a, tiles, st) : launch_expert_t<NA, 2, false, MODE>(a, tiles, st);
}
template <int MODE>
hipError_t launch_expert(const ExpertArgs& a, int na, int64_t tiles, hipStream_t st)
{
    if constexpr (MODE != kDown)
        if (na == 1) return launch_expert_g<1, MODE>(a, tiles, st);        // (one token's down products: one_down_kernel)
    switch (na) {
        case 2: return launch_expert_g<2, MODE>(a, tiles, st);
        case 4: return launch_expert_g<4, MODE>(a, tiles, st);
        default: return launch_expert_g<8, MODE>(a, tiles, st);
    }
}

template <bool GB>
hipError_t launch_one_down(ExpertArgs a, hipStream_t st)
{
    constexpr uint32_t WAVE = kOneDepth * kOneSlot, smem = 16 * WAVE;
    // (more than one workgroup per unit share it.  us with 8 / 16 waves, 8 experts of 1024: 2048 outputs 15.6 / 15.6, 3104 17.8 / 19.9, 4096
    // 18.0 / 20.1, 8192 25.6 / 30.3; 2 of 11008: 2048 outputs 39.3 / 38.9, 4096 43.8 / 47.1)
    const uint32_t groups = a.rows / kOneRows, steps = (uint32_t)a.top_k * ((a.k + 255) / 256), most = groups <= kComputeUnits ? 16 : 8;
    a.waves = (int)(steps < most ? steps : most);
    RAZER_RAISE_LDS_LIMIT((one_down_kernel<GB>), smem);
    launch(one_down_kernel<GB>, groups, 64u * a.waves, a.waves * WAVE, st, a);
    return hipGetLastError();
}

razer_status check_experts(const razer_experts* s, SvConfig& cfg)
{
    if (!s) return RAZER_ERR_NULL;
    if (s->cfg.format != RAZER_FMT_WEIGHT || s->cfg.layout != RAZER_LAYOUT_CANONICAL || check_cfg(s->cfg, cfg) != RAZER_OK) return RAZER_ERR_CONFIG;
    if (s->experts < 1 || s->experts > 1024 || s->rows < 32 || s->rows % 32 != 0 || s->rows > ((int64_t)1 << 20)) return RAZER_ERR_SHAPE;
    if (s->cols < 32 || s->cols % 32 != 0 || s->cols % ((int64_t)1 << cfg.lb) != 0 || s->cols > ((int64_t)1 << 20)) return RAZER_ERR_SHAPE;
    if (!s->codes || !s->scales || !s->tensor_scales) return RAZER_ERR_NULL;
    if (!aligned16(s->codes) || !aligned16(s->scales) || !aligned4(s->tensor_scales)) return RAZER_ERR_ALIGN;
    return RAZER_OK;
}

razer_status check_moe(const razer_moe_args* g, SvConfig& up_cfg, SvConfig& down_cfg)
{
    if (!g) return RAZER_ERR_NULL;
    if (g->act != RAZER_SILU && g->act != RAZER_GELU && g->act != RAZER_RELU) return RAZER_ERR_CONFIG;
    razer_status s = check_experts(g->gate, up_cfg);
    if (s != RAZER_OK) return s;
    s = check_experts(g->down, down_cfg);
    if (s != RAZER_OK) return s;
    if (g->up) {
        SvConfig c;
        s = check_experts(g->up, c);
        if (s != RAZER_OK) return s;
        if (c.lb != up_cfg.lb || c.sv0 != up_cfg.sv0 || c.sv1 != up_cfg.sv1) return RAZER_ERR_CONFIG;
        if (g->up->rows != g->gate->rows || g->up->cols != g->gate->cols || g->up->experts != g->gate->experts) return RAZER_ERR_SHAPE;
    }
    if (g->down->cols != g->gate->rows || g->down->experts != g->gate->experts) return RAZER_ERR_SHAPE;
    if (g->tokens < 0 || g->top_k < 1 || g->top_k > 32 || g->tokens > ((int64_t)1 << 20) / g->top_k) return RAZER_ERR_SHAPE;
    if (g->tokens * g->top_k * g->gate->rows >= ((int64_t)1 << 31)) return RAZER_ERR_SHAPE;
    return RAZER_OK;
}

}  // namespace

}  // namespace razer

using namespace razer;

static razer_status check_route(const razer_moe_route_args* g)
{
    if (!g) return RAZER_ERR_NULL;
    if ((g->score != RAZER_SOFTMAX && g->score != RAZER_SIGMOID) || (!g->x && g->logits_dtype != RAZER_F32 && g->logits_dtype != RAZER_BF16)) return RAZER_ERR_CONFIG;
    if (g->tokens < 0 || g->tokens > ((int64_t)1 << 20) || g->experts < 1 || g->experts > 512 || g->top_k < 1 || g->top_k > 32 || g->top_k > g->experts) return RAZER_ERR_SHAPE;
    if (g->tokens == 0) return RAZER_OK;                                   // (x of no tokens may be NULL too)
    if (g->x ? g->hidden < 32 || g->hidden % 32 != 0 || g->ld_x < g->hidden : g->ld_logits < g->experts) return RAZER_ERR_SHAPE;
    return RAZER_OK;
}

extern "C" {

size_t razer_moe_route_workspace_bytes(const razer_moe_route_args* g)
{
    if (check_route(g) != RAZER_OK || !g->x) return 0;
    return (size_t)route_slices(g->tokens, g->experts, g->hidden) * g->tokens * g->experts * 8;
}

razer_status razer_moe_route(const razer_moe_route_args* g, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const razer_status s = check_route(g);
    if (s != RAZER_OK || g->tokens == 0) return s;
    if (!g->ids || !g->weights || (g->x ? !g->router : !g->logits)) return RAZER_ERR_NULL;
    if (!aligned4(g->ids) || !aligned4(g->weights) || !aligned4(g->bias)) return RAZER_ERR_ALIGN;
    if (g->x ? !aligned16(g->x) || !aligned16(g->router) || g->ld_x % 8 != 0 : reinterpret_cast<uintptr_t>(g->logits) % (g->logits_dtype == RAZER_BF16 ? 2 : 4) != 0) return RAZER_ERR_ALIGN;
    RouteArgs a{static_cast<const uint16_t*>(g->x), static_cast<const uint16_t*>(g->router), g->logits, g->bias, g->ids, g->weights, nullptr, g->ld_x, g->ld_logits,
                g->tokens, g->hidden, g->experts, g->top_k, 1, g->score == RAZER_SIGMOID, g->renormalize != 0, g->logits_dtype == RAZER_BF16, g->scale};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->x) {
        if (!workspace || !aligned16(workspace) || workspace_bytes < razer_moe_route_workspace_bytes(g)) return RAZER_ERR_WORKSPACE;
        a.slices = route_slices(g->tokens, g->experts, g->hidden);
        a.partial = static_cast<double*>(workspace);
        const int side = 16 * route_fragments(g->tokens, g->experts);
        launch(side == 32 ? router_kernel<2, 2> : router_kernel<1, 1>, dim3((g->experts + side - 1) / side, (uint32_t)((g->tokens + side - 1) / side), a.slices),
               64 * kRouteWaves, 0, st, a);
    }
    const uint32_t blocks = (uint32_t)((g->tokens + 3) / 4);
    if (g->experts <= 64) launch(select_kernel<1>, blocks, 256, 0, st, a);
    else if (g->experts <= 128) launch(select_kernel<2>, blocks, 256, 0, st, a);
    else if (g->experts <= 256) launch(select_kernel<4>, blocks, 256, 0, st, a);
    else launch(select_kernel<8>, blocks, 256, 0, st, a);
    return hipGetLastError() == hipSuccess ? RAZER_OK : RAZER_ERR_HIP;
}

size_t razer_moe_workspace_bytes(const razer_moe_args* g)
{
    SvConfig u, d;
    if (check_moe(g, u, d) != RAZER_OK || g->tokens == 0) return 0;
    return plan_of(g->tokens, g->top_k, g->gate->experts, g->gate->rows, g->down->rows).bytes;
}

razer_status razer_moe_experts(const razer_moe_args* g, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    SvConfig u, d;
    const razer_status s = check_moe(g, u, d);
    if (s != RAZER_OK || g->tokens == 0) return s;
    const int64_t hidden = g->gate->cols, inter = g->gate->rows, rows = g->down->rows;
    if (g->ld_x < hidden || g->ld_y < rows || g->tokens * g->ld_x >= ((int64_t)1 << 31)) return RAZER_ERR_SHAPE;
    if (!g->x || !g->ids || !g->weights || !g->y) return RAZER_ERR_NULL;
    if (!aligned16(g->x) || !aligned16(g->y) || g->ld_x % 8 != 0 || g->ld_y % 8 != 0 || !aligned4(g->ids) || !aligned4(g->weights)) return RAZER_ERR_ALIGN;
    const MoePlan p = plan_of(g->tokens, g->top_k, g->gate->experts, inter, rows);
    if (!workspace || !aligned16(workspace) || workspace_bytes < p.bytes) return RAZER_ERR_WORKSPACE;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    int32_t* tile_count = reinterpret_cast<int32_t*>(ws);
    Tile* tiles = reinterpret_cast<Tile*>(ws + 16);
    int32_t* list = reinterpret_cast<int32_t*>(ws + p.list);
    float* out = reinterpret_cast<float*>(ws + p.out);
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool one = g->tokens == 1, few = p.choices <= 64;
    if (!few) launch(plan_kernel, 1, 1024, 0, st, g->ids, (int)p.choices, g->gate->experts, 4 * p.na, tiles, tile_count, list);
    ExpertArgs a{};
    a.ids = g->ids;
    a.experts = g->gate->experts;
    a.choices = (int)p.choices;
    a.tiles = few ? nullptr : tiles;
    a.tile_count = tile_count;
    a.list = list;
    a.top_k = g->top_k;
    a.weights = g->weights;
    a.act_kind = g->act;
    a.w[0] = Stack{g->gate->codes, g->gate->scales, g->gate->tensor_scales};
    if (g->up) a.w[1] = Stack{g->up->codes, g->up->scales, g->up->tensor_scales};
    a.act = static_cast<const uint8_t*>(g->x);
    a.act_ld = g->ld_x * 2;
    a.out = ws + p.mid;
    a.k = (uint32_t)hidden;
    a.rows = (uint32_t)inter;
    a.lb = u.lb;
    a.sv0 = u.sv0;
    a.sv1 = u.sv1;
    a.code_stride = inter * hidden / 2;
    a.scale_stride = inter * (hidden >> u.lb);
    const int64_t up_tiles = one ? p.choices : p.tiles;
    hipError_t e = g->up ? launch_expert<kGated>(a, p.na, up_tiles, st) : launch_expert<kPlain>(a, p.na, up_tiles, st);
    if (e != hipSuccess) return RAZER_ERR_HIP;
    a.w[0] = Stack{g->down->codes, g->down->scales, g->down->tensor_scales};
    a.act = ws + p.mid;
    a.act_ld = inter * 2 * parts<kDown>();
    a.out = out;
    a.k = (uint32_t)inter;
    a.rows = (uint32_t)rows;
    a.lb = d.lb;
    a.sv0 = d.sv0;
    a.sv1 = d.sv1;
    a.code_stride = rows * inter / 2;
    a.scale_stride = rows * (inter >> d.lb);
    if (one) {
        a.out = g->y;
        e = d.lb != 4 ? launch_one_down<true>(a, st) : launch_one_down<false>(a, st);
        if (e != hipSuccess) return RAZER_ERR_HIP;
        return hipGetLastError() == hipSuccess ? RAZER_OK : RAZER_ERR_HIP;
    }
    e = launch_expert<kDown>(a, p.na, p.tiles, st);
    if (e != hipSuccess) return RAZER_ERR_HIP;
    launch(combine_kernel, dim3((uint32_t)g->tokens, (uint32_t)((rows / 4 + 255) / 256)), 256, 0, st, out, g->ids, g->gate->experts, g->top_k, rows,
           static_cast<uint16_t*>(g->y), g->ld_y);
    return hipGetLastError() == hipSuccess ? RAZER_OK : RAZER_ERR_HIP;
}

}  // extern "C"
