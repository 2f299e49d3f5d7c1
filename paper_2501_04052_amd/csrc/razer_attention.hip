// Attention over the 8-bit paged key/value cache (include/razer_cache.h).
//
// Rows.  The query heads that share a key/value head are rows of one product: row rho of request r is token
// rho / group, head rho % group, and a unit is a run of M rows of one request and one key/value head.  The units of
// request r start at index floor(cu[r] * group / M) + r, which leaves room for them whatever the lengths are, so that a
// grid of floor(tokens * group / M) + requests units covers every batch without the host knowing its lengths; a
// workgroup finds its request by a search over cu, 64 entries at a time.
//
// Tiles.  Scores are formed transposed, S^T = K Q^T, so that a lane holds the scores of ONE query row and the softmax
// needs two exchanges between lanes.  O^T = V^T P^T then takes the weights from the very registers that the scores
// were in: the product over keys may run in any order, and key g*16 + 4t + j of a tile of 64 sits in row 4g + j of the
// t-th 16-row key operand, which makes a lane's 16 weights 16 consecutive keys -- 16 bytes of a value page's row.
#include <algorithm>

#include "razer_cache.hpp"

namespace razer {

namespace {

constexpr int kTile = 64;                     // keys per tile
constexpr int kMaxKeys = 1 << 30;             // of a request (tile arithmetic stays within 32 bits)
constexpr float kLog2e = 1.4426950408889634f;

// What a workgroup needs to know of its unit.  Uniform over the workgroup.
struct Unit {
    int request, token0, rows, rho0;          // first token's row of q; rows of the request (new tokens * group); first row here
    int pos0;                                 // position of the request's first new token
    int len;                                  // keys that exist: total, cut to what the table can name
    int prefix;
    int pmin, pmax;                           // positions of the first and last row of this unit
    int n1, start2, tiles;                    // tiles to read: 0 .. n1-1, then from start2 on; how many in all
};

__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ int cu_at(const AttentionArgs& a, int r) { return min(max(a.cu[r], 0), a.tokens); }

// The first key within the window of a query at position pos, which may lie in front of the first key and anywhere below 2^31.
__device__ __forceinline__ int window_begin(const AttentionArgs& a, int pos) { return a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0; }

// The unit of m rows that begins at row rho0 of a request with n new tokens from row token0 of q on.
__device__ __forceinline__ Unit make_unit(const AttentionArgs& a, int lp, int m, int request, int token0, int n, int total, int prefix, int rho0)
{
    Unit o;
    o.request = request;
    o.token0 = token0;
    o.rows = n * a.group;
    o.rho0 = rho0;
    total = max(total, 0);
    o.pos0 = total - n;
    o.len = (int)min((int64_t)min(total, kMaxKeys), (int64_t)a.width << lp);
    o.prefix = min(max(prefix, 0), o.len);
    o.pmin = o.pos0 + rho0 / a.group;
    o.pmax = o.pos0 + min(rho0 + m - 1, o.rows - 1) / a.group;
    const int end = min(max(o.pmax + 1, o.prefix), o.len);                 // >= 0 as len >= 0, prefix >= 0
    const int last = (end + kTile - 1) / kTile;
    o.n1 = 0;
    o.start2 = 0;
    if (a.window > 0) {
        o.n1 = (o.prefix + kTile - 1) / kTile;
        o.start2 = max(o.n1, window_begin(a, o.pmin) / kTile);
    }
    o.tiles = o.n1 + max(last - o.start2, 0);
    return o;
}

// A lane's request.
struct Lengths {
    int token0, n, total, prefix;
};
__device__ __forceinline__ Lengths load_lengths(const AttentionArgs& a, int r)
{
    Lengths o = {0, 0, 0, 0};
    if (r < a.requests) {
        o.token0 = cu_at(a, r);
        o.n = max(cu_at(a, r + 1) - o.token0, 0);
        o.total = a.total[r];
        o.prefix = a.prefix ? a.prefix[r] : 0;
    }
    return o;
}

__device__ __forceinline__ int lane32(int x, int i) { return __builtin_amdgcn_readlane(x, i); }

// false: no such unit.  64 requests at a time, a lane each; with more of them the right 64 are searched for first.
__device__ __forceinline__ bool find_unit(const AttentionArgs& a, int lp, int u, int m, Unit& o)
{
    int lo = 0, count = a.requests;
    const int lane = threadIdx.x & 63;
    while (count > 64) {
        const int stride = (count + 63) >> 6, i = lane * stride;
        const bool le = i < count && cu_at(a, lo + i) * a.group / m + lo + i <= u;
        const int n = max(__popcll(__ballot(le)), 1);
        lo = uni(lo + (n - 1) * stride);
        count = uni(min(stride, count - (n - 1) * stride));
    }
    const Lengths q = load_lengths(a, lo + lane);
    const int first = q.token0 * a.group / m + lo + lane;
    const int i = max(__popcll(__ballot(lane < count && first <= u)), 1) - 1;
    const int n = lane32(q.n, i), rho0 = (u - lane32(first, i)) * m;
    if (rho0 < 0 || rho0 >= n * a.group) return false;
    o = make_unit(a, lp, m, lo + i, lane32(q.token0, i), n, lane32(q.total, i), lane32(q.prefix, i), rho0);
    return true;
}

// Which keys a row sees, for a lane whose first key is j0: key j0 + i if (unsigned)(i - from) < count or i < pre.  Keys past
// the request's are in neither, those of an absent page are cleared with `there`.
struct Sight {
    int from, count, pre;
};
__device__ __forceinline__ Sight sight_of(const AttentionArgs& a, const Unit& un, int pos, int j0)
{
    const int hi = min(pos + 1, un.len), lo = window_begin(a, pos);
    return Sight{lo - j0, max(hi - lo, 0), un.prefix - j0};
}
__device__ __forceinline__ bool sees(const Sight& v, int i) { return ((uint32_t)(i - v.from) < (uint32_t)v.count) | (i < v.pre); }

// of 16 one-byte values, the first n: a mask
__device__ __forceinline__ v4u first_bytes(int n)
{
    v4u keep;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int k = min(max(n - 4 * w, 0), 4);
        keep[w] = (uint32_t)((1ull << (8 * k)) - 1u);
    }
    return keep;
}

__device__ __forceinline__ v8bf decode8(uint32_t lo, uint32_t hi, float scale)
{
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const v2bf c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return v8bf{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

__device__ __forceinline__ v8h decode8h(uint32_t lo, uint32_t hi)
{
    const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return v8h{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// cap * tanh(s / cap) * log2(e) of a score s = x * scale, relative to |s| within 2^-18 whatever the cap is.  From |y| = |s / cap| = 1/4
// on tanh y = 1 - 2 / (e^2y + 1), which cancels for smaller ones; those take the series y - y^3/3 + 2 y^5/15 - 17 y^7/315 +
// 62 y^9/2835 (what is left out is below 2^-26 of it) with s itself in the place of cap * y.
struct Cap {
    float inv, mul, cap2;                     // scale / cap, scale * log2(e), cap * log2(e)
};
__device__ __forceinline__ Cap cap_of(const AttentionArgs& a)
{
    constexpr float most = 3.402823466e38f;   // (a product of 0 stays 0 where scale / cap overflows)
    return Cap{a.cap > 0.0f ? fminf(fmaxf(a.scale / a.cap, -most), most) : 0.0f, a.scale * kLog2e, a.cap * kLog2e};
}
__device__ __forceinline__ float capped(float x, const Cap& c)
{
    const float y = x * c.inv, z = y * y;
    const float series = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
    const float far = c.cap2 * (1.0f - 2.0f * __builtin_amdgcn_rcpf(exp2_fast(2.0f * kLog2e * y) + 1.0f));
    return fabsf(y) < 0.25f ? x * c.mul * series : far;
}

// the larger of this lane's value and that of lane ^ 16 / lane ^ 32: the swap of half rows (halves) of two copies of a
// register leaves the two values in the two copies
__device__ __forceinline__ float max_xor16(float x)
{
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float max_xor32(float x)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// Weights.  In units of log2, a key of score s on a page of value scale 2^e enters O^T with 2^(s + e - m), m being the
// row's running maximum of s + e, and the sum with that times 2^-e: values are multiplied as bare codes, which f16
// holds exactly, and the weights are rounded to f16 (11 bits, where bf16 would have 8 at the same rate) relative to the
// row's largest.  kTop puts that one near f16's upper end, so that subnormals begin 2^-26 below it.  The maximum
// follows lazily: while it grows by less than kSlack, O and the sum keep their scale (2^(kTop + kSlack) < 65504).
constexpr float kTop = 12.0f, kSlack = 3.0f;

}  // namespace

// Few rows.  A piece is a run of tiles of one unit of M = kRows rows and one key/value head; the NW waves of a workgroup
// take every NW-th tile with a running maximum and sum of their own, and meet in LDS at the end.  Bound by memory: a wave
// requests the next tile's keys once the scores are formed and the next values behind the products with the last ones, so that
// 8 to 16 KB a wave (D = 128) are always on their way.  The loads of a step are the same number in every step, wanted or
// not (the last ones go to one address), so that the compiler can wait for the older ones alone; page ids and scales wait in
// LDS.  Where one unit is all that reads a head's keys (ONCE), codes are loaded without being kept in the caches (64 ragged
// requests, 305 MB: 63 -> 56 us; 32 of 16384 keys, 1075 MB: 192 -> 172), but not values in pages of 128 tokens, of whose
// 128-byte rows a tile takes half (three requests of up to 131001: 107 -> 125 with them).  With
// D > 128 keys and values take turns in the same registers, which leaves room for a second wave per SIMD.
constexpr int kIdTiles = 64;                  // tiles whose page ids are in LDS at a time

struct Block {                                // of 16 keys
    int id;                                   // page, or -1
    uint8_t ks, vs, unused[2];                // exponent bytes
};

constexpr int kRows = 16;                     // of a unit

// What a wave has of a piece: row col (col = lane % 16, g = lane / 16): running maximum, sum, and O for the
// elements dt*16 + g*4 + i.  Equal over g but for O.
template <int D>
struct Rows {
    v4f o[D / 16];
    float m, l;
};

// the barrier of the NW waves that work on a piece together
template <int NW>
__device__ __forceinline__ void piece_barrier()
{
    if constexpr (NW == 1) {                  // (a wave's LDS accesses are carried out in order: only the compiler has to keep to it)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}

// tile number -> first key
__device__ __forceinline__ int tile_key(const Unit& un, int t) { return (t < un.n1 ? t : un.start2 + t - un.n1) * kTile; }

// Kept within the format's range: a page that holds nothing yet may have any byte, and its 2^-e must not make a NaN of the
// weights 0 of its keys.
__device__ __forceinline__ uint8_t scale_byte(const uint8_t* scales, int64_t at)
{
    return (uint8_t)min(max((int)scales[at], RAZER_CACHE_MIN_EXPONENT), RAZER_CACHE_MAX_EXPONENT);
}

__device__ __forceinline__ Block load_block(const CacheView& c, const AttentionArgs& a, const Unit& un, int head, int t, int blk)
{
    const int i = (tile_key(un, t) + blk * 16) >> c.lp;
    Block b = {-1, 127, 127, {0, 0}};
    if (i < a.width) {
        const int id = a.table[(int64_t)un.request * a.ld_table + i];
        if (id >= 0 && id < c.pages) {
            b.id = id;
            b.ks = scale_byte(c.k_scales, (int64_t)id * c.heads + head);
            b.vs = scale_byte(c.v_scales, (int64_t)id * c.heads + head);
        }
    }
    return b;
}

template <bool ONCE>
__device__ __forceinline__ v4u load_codes(const uint8_t* p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p));
    else return *reinterpret_cast<const v4u*>(p);
}

template <int D, int NW, int ONCE>
__device__ __forceinline__ Rows<D> rows_piece(const CacheView& c, const AttentionArgs& a, const Unit& un, int head, int tile0, int tile_end,
                                                  Block (&block)[kIdTiles][4])
{
    constexpr int KC = D / 64, DT = D / 16;
    constexpr bool kTurns = D > 128;
    const int tid = NW == 1 ? threadIdx.x & 63 : threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), col = lane & 15, g = lane >> 4;
    const int page = 1 << c.lp;
    const int64_t page_bytes = (int64_t)page * D;

    // queries: row rho0 + col, as the second operand of S^T = K Q^T
    const int rho = un.rho0 + col;
    const bool ok = rho < un.rows;
    const int tok = ok ? rho / a.group : 0, h = head * a.group + (ok ? rho % a.group : 0), pos = un.pos0 + tok;
    const float slope = a.slopes ? a.slopes[h] * kLog2e : 0.0f;
    const uint16_t* query = a.q + (int64_t)(un.token0 + tok) * a.ld_q + (int64_t)h * D + g * 16;
    v8bf q[KC][2];
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint4 w = ok ? *reinterpret_cast<const uint4*>(query + kc * 64 + hf * 8) : make_uint4(0, 0, 0, 0);
            q[kc][hf] = __builtin_bit_cast(v8bf, w);
        }

    Rows<D> x;
    v4f (&o)[DT] = x.o;
    float &m = x.m, &l = x.l;
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const Cap cap = cap_of(a);
    const float mul = cap.mul;
    const bool bent = a.cap > 0.0f || a.slopes != nullptr || !(mul > 0.0f);
    const float by = bent ? 1.0f : mul;

    // a lane reads keys of block col >> 2 of a tile, and values of block g
    v4u kx[4][KC], vx[DT];
    int first = 0;
    auto load_keys = [&](int t, bool want) __attribute__((always_inline)) {
        const int key = tile_key(un, t) + (col >> 2) * 16 + (col & 3);
        const uint8_t* p = c.k_codes + ((int64_t)max(block[t - first][col >> 2].id, 0) * c.heads + head) * page_bytes + (key & (page - 1)) * D + g * 16;
        p = want ? p : c.k_codes;
        const int step = want ? 4 * D : 0;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int kc = 0; kc < KC; ++kc) kx[kt][kc] = load_codes<(ONCE >= 1)>(p + kt * step + kc * 64);
    };
    auto load_values = [&](int t, bool want) __attribute__((always_inline)) {
        const int key = tile_key(un, t) + g * 16;
        const uint8_t* p = c.v_codes + ((int64_t)max(block[t - first][g].id, 0) * c.heads + head) * page_bytes + col * page + (key & (page - 1));
        p = want ? p : c.v_codes;
        const int step = want ? 16 * page : 0;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vx[dt] = load_codes<(ONCE >= 2)>(p + dt * step);
    };

    for (first = tile0; first < tile_end; first += kIdTiles) {
        const int stop = min(tile_end, first + kIdTiles);
        piece_barrier<NW>();                             // (the last tiles' ids have been read)
        for (int i = tid; i < (stop - first) * 4; i += NW * 64) block[i >> 2][i & 3] = load_block(c, a, un, head, first + (i >> 2), i & 3);
        piece_barrier<NW>();
        int t = first + wave;
        if (t >= stop) continue;                         // (uniform over the wave; it meets the others at the next barrier)
        load_keys(t, true);
        if (!kTurns) load_values(t, true);
        for (; t < stop; t += NW) {
            const int kb = tile_key(un, t);
            const bool more = t + NW < stop;
            const int tn = more ? t + NW : t;
            const Block kb_now = block[t - first][col >> 2], vb_now = block[t - first][g];
            v4f s[4];
            const float ks = exponent_value(kb_now.ks);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                s[kt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int kc = 0; kc < KC; ++kc) {
                    const v8bf k0 = decode8(kx[kt][kc].x, kx[kt][kc].y, ks), k1 = decode8(kx[kt][kc].z, kx[kt][kc].w, ks);
                    s[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[kc][0], s[kt], 0, 0, 0);
                    s[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[kc][1], s[kt], 0, 0, 0);
                }
            }
            if (kTurns) load_values(t, true);
            else load_keys(tn, more);
            // scores, in units of log2 once multiplied by `by`: lane has key j0 + kt*4 + i of row col
            const int j0 = kb + g * 16;
            const bool vok = vb_now.id >= 0;
            const bool whole = kb + kTile <= un.len && __all(vok) &&
                               ((kb + kTile - 1 <= un.pmin && kb >= window_begin(a, un.pmax)) || kb + kTile <= un.prefix);
            if (bent) {
                if (a.cap > 0.0f) {
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[kt][i] = capped(s[kt][i], cap);
                        if constexpr (D > 192) __builtin_amdgcn_sched_barrier(0);   // (16 at once would not fit the registers)
                    }
                } else {
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt) s[kt] *= mul;
                }
                if (a.slopes) {
                    const float far = (float)(pos - j0);
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[kt][i] -= slope * fabsf(far - (float)(kt * 4 + i));
                }
            }
            if (!whole) {
                if (a.window == 0 && un.prefix == 0) {               // (a third of the instructions)
                    const int hi = vok ? min(pos + 1, un.len) - j0 : 0;
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[kt][i] = kt * 4 + i < hi ? s[kt][i] : -INFINITY;
                } else {
                    const Sight v = sight_of(a, un, vok ? pos : -1, j0);
                    const int pre = vok ? v.pre : 0;
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[kt][i] = sees(Sight{v.from, v.count, pre}, kt * 4 + i) ? s[kt][i] : -INFINITY;
                }
                // values of keys that are not there: anything may be in their place
                const v4u keep = first_bytes(vok ? un.len - j0 : 0);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) vx[dt] &= keep;
            }
            v8h p[2];
            const float e = (float)(vb_now.vs - 127), unscale = exponent_value(254 - vb_now.vs);
            float top = s[0][0];
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[kt][i]);
            top = max_xor32(max_xor16(top * by + e));
            if (__any(top > m + kSlack)) {
                const float mn = fmaxf(m, top), f = exp2_fast(m - (mn == -INFINITY ? 0.0f : mn));
                m = mn;
                l *= f;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] *= f;
            }
            const float shift = e + kTop - (m == -INFINITY ? 0.0f : m);
            float sum = 0.0f;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = exp2_fast(__builtin_fmaf(s[kt][i], by, shift));
                    sum += w;
                    p[kt >> 1][(kt & 1) * 4 + i] = (_Float16)w;
                }
            l += sum * unscale;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const v8h v0 = decode8h(vx[dt].x, vx[dt].y), v1 = decode8h(vx[dt].z, vx[dt].w);
                o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[0], o[dt], 0, 0, 0);
                o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[1], o[dt], 0, 0, 0);
            }
            if (kTurns) load_keys(tn, more);
            else load_values(tn, more);
        }
    }

    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    return x;
}

__device__ __forceinline__ uint16_t* out_at(const AttentionArgs& a, int token0, int head, int rho, int dim)
{
    return a.out + (int64_t)(token0 + rho / a.group) * a.ld_out + (int64_t)(head * a.group + rho % a.group) * dim;
}
__device__ __forceinline__ v4bf finished(v4f x, float sum)
{
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    return v4bf{(__bf16)(x.x * inv), (__bf16)(x.y * inv), (__bf16)(x.z * inv), (__bf16)(x.w * inv)};
}

// One workgroup of NW waves per unit and key/value head.
template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attention_rows_kernel(CacheView c, AttentionArgs a)
{
    constexpr int M = kRows, DT = D / 16;
    __shared__ Block block[kIdTiles][4];
    __shared__ __align__(16) float s_o[2][M][D + 4];
    __shared__ float s_m[NW][M], s_l[NW][M];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), col = lane & 15, g = lane >> 4, head = blockIdx.x % c.heads;
    Unit un;
    if (!find_unit(a, c.lp, blockIdx.x / c.heads, M, un)) return;
    const Rows<D> x = rows_piece<D, NW, 0>(c, a, un, head, 0, un.tiles, block);
    if (g == 0) {
        s_m[wave][col] = x.m;
        s_l[wave][col] = x.l;
    }
    __syncthreads();
    auto top_of = [&](int r) {
        float t = s_m[0][r];
#pragma unroll
        for (int w = 1; w < NW; ++w) t = fmaxf(t, s_m[w][r]);
        return t == -INFINITY ? 0.0f : t;
    };
    const float f = exp2_fast(x.m - top_of(col));
#pragma unroll
    for (int turn = 0; turn < NW / 2; ++turn) {
        if ((wave >> 1) == turn) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                v4f* at = reinterpret_cast<v4f*>(&s_o[wave & 1][col][dt * 16 + g * 4]);
                const v4f y = x.o[dt] * f;
                *at = turn ? *at + y : y;
            }
        }
        __syncthreads();
    }
    for (int i = tid; i < M * D / 4; i += NW * 64) {
        const int r = i / (D / 4), d = i % (D / 4) * 4, rho = un.rho0 + r;
        if (rho >= un.rows) break;
        const float top = top_of(r);
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += s_l[w][r] * exp2_fast(s_m[w][r] - top);
        const v4f y = *reinterpret_cast<const v4f*>(&s_o[0][r][d]) + *reinterpret_cast<const v4f*>(&s_o[1][r][d]);
        *reinterpret_cast<v4bf*>(out_at(a, un.token0, head, rho, D) + d) = finished(y, sum);
    }
}

// The tiles of all units, laid end to end (request, head, unit, tile; a unit without tiles counts as one), in equal
// shares for a fixed number of waves: requests of any lengths keep the whole card busy to the end. A wave sums up the lengths
// by itself, 64 requests at a time, a lane each, and works alone, so that it seldom begins more than two pieces and meets no
// other before its end (with shares that four waves worked on together, tile by tile, each began all of their pieces: 64
// ragged requests of up to 8192 keys took 83 us, then 66; 58 us + 5 to join with codes that are not kept in the caches, 305 MB at
// 5.2 TB/s). The waves of a workgroup have neighbouring shares. A wave that begins with the
// rest of a unit leaves it in LDS, where the wave that began the unit picks it up; what the workgroup's end cuts is left in the
// workspace for attention_join_shares_kernel: at most two pieces a workgroup.
struct Share {                 // what a workgroup leaves
    int open;                  // 1: piece 1 begins a unit that goes on in the next workgroup
    int request, head, rho0, token0, rows;
    int cont;                  // piece 0 continues a unit of the workgroup before: 1 to its end, 2 and further on
    int cont_rows;             // rows that piece 0 has
};
constexpr int shares_of(int dim) { return (int)kComputeUnits * (dim <= 128 ? 2 : 1); }   // as many as are resident at a time,
constexpr int share_waves(int dim) { return dim <= 128 ? 4 : 8; }                         // with eight waves a compute unit
constexpr int kLeastTiles = 2;                 // of a wave

// tiles of one head of a lane's request
__device__ __forceinline__ int64_t tiles_of(const AttentionArgs& a, int lp, int m, int r, const Lengths& q)
{
    int64_t n = 0;
    for (int rho = 0; rho < q.n * a.group; rho += m) n += max(make_unit(a, lp, m, r, q.token0, q.n, q.total, q.prefix, rho).tiles, 1);
    return n;
}
__device__ __forceinline__ int64_t lane64(int64_t x, int i)
{
    return (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, i) | (int64_t)__builtin_amdgcn_readlane((int)(x >> 32), i) << 32;
}
__device__ __forceinline__ int64_t wave_inclusive(int64_t x)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = __shfl_up(x, d);
        if ((int)(threadIdx.x & 63) >= d) x += y;
    }
    return x;
}

// m and l [M], O [M][D + 4]
template <int D>
__device__ __forceinline__ void put_piece(float* to, const Rows<D>& x, int rows)
{
    constexpr int M = kRows;
    const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    if (col >= rows) return;
    if (g == 0) {
        to[col] = x.m;
        to[M + col] = x.l;
    }
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<v4f*>(to + 2 * M + col * (D + 4) + dt * 16 + g * 4) = x.o[dt];
}
template <int D>
__device__ __forceinline__ void add_piece(Rows<D>& x, const float* from, int rows)
{
    constexpr int M = kRows;
    const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    if (col >= rows) return;
    const float m = from[col], top = fmaxf(x.m, m), ref = top == -INFINITY ? 0.0f : top, f = exp2_fast(x.m - ref), fp = exp2_fast(m - ref);
    x.m = top;
    x.l = x.l * f + from[M + col] * fp;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
        x.o[dt] = x.o[dt] * f + *reinterpret_cast<const v4f*>(from + 2 * M + col * (D + 4) + dt * 16 + g * 4) * fp;
}
template <int D>
__device__ __forceinline__ void put_out(const AttentionArgs& a, const Rows<D>& x, int token0, int head, int rho0, int rows)
{
    const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const int rho = rho0 + col;
    if (rho >= rows) return;
    uint16_t* p = out_at(a, token0, head, rho, D) + g * 4;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<v4bf*>(p + dt * 16) = finished(x.o[dt], x.l);
}

template <int D, int ONCE>
__global__ __launch_bounds__(64 * share_waves(D), 2) void attention_shares_kernel(CacheView c, AttentionArgs a, Share* __restrict__ shares, float* __restrict__ ws)
{
    constexpr int M = kRows, PIECE = 2 * M + M * (D + 4), kShares = shares_of(D), NW = share_waves(D);
    __shared__ Block block[NW][kIdTiles][4];
    __shared__ __align__(16) float s_piece[NW][PIECE];   // the first piece of a wave, if it continues a unit
    __shared__ Share s_share[NW];
    const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
    int rb = 0;
    Lengths q = load_lengths(a, lane);
    int64_t own = tiles_of(a, c.lp, M, lane, q), upto = wave_inclusive(own * c.heads), all = lane64(upto, 63);
    const int64_t first = all;
    for (int r = 64; r < a.requests; r += 64) {
        const Lengths x = load_lengths(a, r + lane);
        all += lane64(wave_inclusive(tiles_of(a, c.lp, M, r + lane, x) * c.heads), 63);
    }
    const int64_t share = max((all + NW * kShares - 1) / (NW * kShares), (int64_t)kLeastTiles);
    // neighbouring shares, which may read the same keys, on one XCD (workgroups go to the 8 XCDs in turn)
    const int per = (int)(((all + NW * share - 1) / (NW * share) + 7) / 8), xcd = (int)(blockIdx.x % 8), nth = (int)(blockIdx.x / 8);
    const int w = nth < per ? xcd * per + nth : 8 * per + (nth - per) * 8 + xcd;   // (the others have nothing to do but say so)
    int64_t pos = (w * NW + wave) * share;
    const int64_t end = min(all, pos + share);
    Share mine = {0, 0, 0, 0, 0, 0, 0, 0};
    Rows<D> x;                                       // the last piece
    if (pos < end) {
        int64_t base = 0, chunk = first;
        while (pos >= base + chunk) {                    // (ends: pos < all)
            base += chunk;
            rb += 64;
            q = load_lengths(a, rb + lane);
            own = tiles_of(a, c.lp, M, rb + lane, q);
            upto = wave_inclusive(own * c.heads);
            chunk = lane64(upto, 63);
        }
        int i = __popcll(__ballot(base + upto <= pos));
        while (pos < end) {
            const int64_t tiles = lane64(own, i), at = pos - (base + lane64(upto, i) - tiles * c.heads);
            const int head = (int)(at / tiles);
            int64_t in = at - head * tiles;
            Unit un;
            int64_t size;
            for (int rho = 0;; rho += M) {
                un = make_unit(a, c.lp, M, rb + i, lane32(q.token0, i), lane32(q.n, i), lane32(q.total, i), lane32(q.prefix, i), rho);
                size = max(un.tiles, 1);
                if (in < size) break;
                in -= size;
            }
            const int64_t take = min(size - in, end - pos);
            const bool begins = in == 0, ends = in + take == size;
            x = rows_piece<D, 1, ONCE>(c, a, un, head, (int)in, (int)min(in + take, (int64_t)un.tiles), block[wave]);
            if (begins && ends) {
                put_out(a, x, un.token0, head, un.rho0, un.rows);
            } else if (begins) {
                mine = Share{1, un.request, head, un.rho0, un.token0, un.rows, mine.cont, mine.cont_rows};
            } else {
                mine.cont = ends ? 1 : 2;
                mine.cont_rows = min(M, un.rows - un.rho0);
                put_piece(s_piece[wave], x, mine.cont_rows);
            }
            pos += take;
            // on to the request of the next tile
            while (pos < end && base + lane64(upto, i) <= pos) {
                if (++i == 64) {
                    base += chunk;
                    rb += 64;
                    i = 0;
                    q = load_lengths(a, rb + lane);
                    own = tiles_of(a, c.lp, M, rb + lane, q);
                    upto = wave_inclusive(own * c.heads);
                    chunk = lane64(upto, 63);
                }
            }
        }
    }
    if (lane == 0) s_share[wave] = mine;
    __syncthreads();

    // Behind a piece that goes on stand the first pieces of the waves behind, up to the one that ends the unit.
    auto follow = [&](int from, bool ended, int rows, bool add) {
        for (int v = from + 1; v < NW && !ended && s_share[v].cont; ++v) {
            ended = s_share[v].cont == 1;
            if (add) add_piece(x, s_piece[v], rows);
        }
        return ended;
    };
    const Share me = s_share[wave];
    float* piece = ws + (int64_t)w * 2 * PIECE;
    if (me.open) {
        if (follow(wave, false, min(M, me.rows - me.rho0), true)) put_out(a, x, me.token0, me.head, me.rho0, me.rows);
        else put_piece(piece + PIECE, x, min(M, me.rows - me.rho0));
    }
    if (wave == 0) {
        int cont = me.cont;
        if (cont) {                                      // of the workgroup before
            x.m = -INFINITY;
            x.l = 0.0f;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) x.o[dt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            add_piece(x, s_piece[0], me.cont_rows);
            cont = follow(0, cont == 1, me.cont_rows, true) ? 1 : 2;
            put_piece(piece, x, me.cont_rows);
        }
        int on = -1;
        for (int v = 0; v < NW; ++v)
            if (s_share[v].open && !follow(v, false, 0, false)) on = v;   // (at most one)
        if (lane == 0) {
            const Share& from = s_share[max(on, 0)];
            shares[w].open = on >= 0;
            shares[w].request = from.request;
            shares[w].head = from.head;
            shares[w].rho0 = from.rho0;
            shares[w].token0 = from.token0;
            shares[w].rows = from.rows;
            shares[w].cont = cont;
        }
    }
}

// Puts the pieces of cut units together, in the order of the keys: the workgroup of the share in which the unit begins.  Its
// waves are four groups of four; a wave of a group runs over every fourth piece with a running maximum, and the four results
// meet in LDS: always in that order.
template <int D>
__global__ __launch_bounds__(1024) void attention_join_shares_kernel(AttentionArgs a, const Share* __restrict__ shares, const float* __restrict__ ws)
{
    constexpr int M = kRows, RB = 256 / D, L4 = D / 4, LDO = D + 4, PIECE = 2 * M + M * LDO, kShares = shares_of(D);
    __shared__ float s_o[16][RB][D], s_m[16][RB], s_l[16][RB];
    const int w = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), slice = wave & 3, group = wave >> 2;
    const Share me = shares[w];
    if (!me.open) return;
    int pieces = 1;
    for (int v = w + 1; v < kShares; v += 64) {
        const int cont = v + lane < kShares ? shares[v + lane].cont : 1;
        const uint64_t stop = __ballot(cont != 2);
        if (stop) {
            pieces += __ffsll((unsigned long long)stop);
            break;
        }
        pieces += 64;
    }
    pieces = min(pieces, kShares - w);
    const int rr = lane / L4, d = lane % L4 * 4;
    constexpr int64_t size = PIECE;
    const float* first = ws + (int64_t)w * 2 * size;
    for (int r0 = 0; r0 < min(M, me.rows - me.rho0); r0 += 4 * RB) {
        const int r = r0 + group * RB + rr, rho = me.rho0 + r;
        const bool on = rr < RB && r < M && rho < me.rows;
        if (on) {
            float top = -INFINITY, sum = 0.0f;
            v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
            for (int p = slice; p < pieces; p += 4) {
                const float* wp = first + (p ? (int64_t)p * 2 * size : size);
                const float mp = wp[r], lp = wp[M + r];
                const v4f xp = *reinterpret_cast<const v4f*>(wp + 2 * M + r * LDO + d);
                const float mn = fmaxf(top, mp), ref = mn == -INFINITY ? 0.0f : mn, f = exp2_fast(top - ref), fp = exp2_fast(mp - ref);
                x = x * f + xp * fp;
                sum = sum * f + lp * fp;
                top = mn;
            }
            *reinterpret_cast<v4f*>(&s_o[wave][rr][d]) = x;
            if (d == 0) {
                s_m[wave][rr] = top;
                s_l[wave][rr] = sum;
            }
        }
        __syncthreads();
        if (on && slice == 0) {
            float top = s_m[wave][rr], sum = 0.0f;
#pragma unroll
            for (int p = 1; p < 4; ++p) top = fmaxf(top, s_m[wave + p][rr]);
            const float ref = top == -INFINITY ? 0.0f : top;
            v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const float f = exp2_fast(s_m[wave + p][rr] - ref);
                sum += s_l[wave + p][rr] * f;
                x += *reinterpret_cast<const v4f*>(&s_o[wave + p][rr][d]) * f;
            }
            const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
            const v4bf y = {(__bf16)(x.x * inv), (__bf16)(x.y * inv), (__bf16)(x.z * inv), (__bf16)(x.w * inv)};
            uint16_t* p = a.out + (int64_t)(me.token0 + rho / a.group) * a.ld_out + (int64_t)(me.head * a.group + rho % a.group) * D + d;
            *reinterpret_cast<v4bf*>(p) = y;
        }
        __syncthreads();
    }
}

// Many rows: one workgroup of four waves per (unit of 128 rows, key/value head, chunk of tiles).  Each wave has 32 rows, and
// the four share every tile of codes, which passes through registers into LDS while the tiles before it are multiplied,
// with a barrier every second tile (every tile with D > 128, where LDS holds fewer; one prompt of 2048 tokens at
// 32 / 8 heads 73.5 -> 70 us; 2048 new tokens of 16384 at 64 / 8 heads, 1.03 TFLOP: 1.18 ms).  The 32 x 32 products leave a lane with 32 of the 64 scores of one row: key h*32 + 16*tt + 4*b + j (h = lane / 32)
// sits in row 8b + 4h + j of the tt-th key operand, so that here, too, the weights of a lane are runs of 16 consecutive keys.
//
// Bound by the vector unit and the products, which seldom overlap: a tile takes a wave 372 vector instructions (SQ_INSTS_VALU) and
// 1024 cycles of products (D = 128).  For 2048 new tokens of 16384 at 64 / 8 heads a SIMD spends 2750 cycles on it, with 1.8 waves on
// average; its vector unit is active in 59 % and its matrix unit busy in 37 % of them (one prompt of 2048 tokens at 32 / 8 heads, where long
// units end alone: 35 % and 20 %, 1.1 waves).  (Keys multiplied as the codes they are, by block-
// scaled E4M3 products with queries in two parts, save 64 conversions a tile and 8 % of the time, 1230 -> 1130 us for 2048 new
// tokens of 16384 at 64 / 8 heads; but their sums are not as exact as fp32 ones, and scores were off by 2^-16 of sum |q k|.)
template <int D>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void attention_tiles_kernel(CacheView c, AttentionArgs a, int units, int paired, int splits, int chunk,
                                                                              float* __restrict__ ws)
{
    constexpr int M = 128, KCH = D / 16, NS = D / 64, DT = D / 32;
    constexpr int STEP = D <= 128 ? 2 : 1, RING = 2 * STEP;   // tiles between two barriers (as many as fit LDS twice), tiles in LDS
    constexpr bool kFar = D > 128;                       // queries in LDS: beside O the registers do not hold them
    __shared__ v4u s_k[RING][kTile * KCH], s_v[RING][D * 4];
    __shared__ v4u s_q[kFar ? 4 : 1][kFar ? KCH : 1][64];
    __shared__ int s_meta[8][4][3];                      // by tile & 7, block of 16 keys: page (-1: none), exponent bytes of keys and values
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), col = lane & 31, h = lane >> 5;
    // A request's last rows see the most keys: they go first. Where all are resident at once (paired), the second half goes the
    // other way: workgroups 256 apart share a compute unit, so that the longest has the shortest beside it (one prompt of 2048
    // tokens at 32 / 8 heads: 75 -> 73 us).
    const int head = blockIdx.x % c.heads, uc = blockIdx.x / c.heads, part = uc % splits, nth = uc / splits, half = (units + 1) / 2;
    const int u = paired && nth >= half ? nth - half : units - 1 - nth;
    Unit un;
    if (!find_unit(a, c.lp, u, M, un)) return;
    const int parts = min(splits, max(1, (un.tiles + chunk - 1) / chunk));
    if (part >= parts) return;
    const int tile_end = part == splits - 1 ? un.tiles : min(un.tiles, (part + 1) * chunk), tile0 = part * chunk;

    const int page = 1 << c.lp;
    const int64_t page_bytes = (int64_t)page * D;
    const int32_t* table = a.table + (int64_t)un.request * a.ld_table;
    auto base_of = [&](int t) __attribute__((always_inline)) { return (t < un.n1 ? t : un.start2 + t - un.n1) * kTile; };

    // staging: this thread's 16-byte pieces of a tile.  LDS rows of keys stand in the order of the operand's rows.
    auto krow_key = [](int row) { return ((row >> 2) & 1) * 32 + (row >> 5) * 16 + ((row >> 3) & 3) * 4 + (row & 3); };
    auto kswz = [](int row) { return KCH == 4 || KCH == 12 ? (row >> 2) & 3 : KCH == 8 ? (row >> 1) & 7 : row & 15; };
    v4u kx[NS], vx[NS];
    auto page_id = [&](int t, int blk) __attribute__((always_inline)) {
        const int i = (base_of(t) + blk * 16) >> c.lp;
        const int id = i < a.width ? table[i] : -1;
        return id >= 0 && id < c.pages ? id : -1;
    };
    auto fetch = [&](int t, v4u (&kr)[NS], v4u (&vr)[NS]) __attribute__((always_inline)) {
        const int kb = base_of(t);
        if (c.lp >= 6) {
            const int64_t at = ((int64_t)uni(max(s_meta[t & 7][0][0], 0)) * c.heads + head) * page_bytes;
            const uint8_t* kp = c.k_codes + at + (kb & (page - 1)) * D;
            const uint8_t* vp = c.v_codes + at + (kb & (page - 1));
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                const int ofs = krow_key((tid + n * 256) / KCH) * D + ((tid + n * 256) % KCH) * 16;
                kr[n] = *reinterpret_cast<const v4u*>(kp + (uint32_t)ofs);
            }
#pragma unroll
            for (int n = 0; n < NS; ++n) vr[n] = *reinterpret_cast<const v4u*>(vp + (uint32_t)((tid & 3) * 16 + (tid / 4 + n * 64) * page));
            return;
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            const int i = tid + n * 256, key = krow_key(i / KCH);
            const int64_t at = (int64_t)max(s_meta[t & 7][key >> 4][0], 0) * c.heads + head;
            kr[n] = *reinterpret_cast<const v4u*>(c.k_codes + at * page_bytes + ((kb + key) & (page - 1)) * D + (i % KCH) * 16);
        }
        const int64_t at = (int64_t)max(s_meta[t & 7][tid & 3][0], 0) * c.heads + head;
        const uint8_t* p = c.v_codes + at * page_bytes + ((kb + (tid & 3) * 16) & (page - 1));
#pragma unroll
        for (int n = 0; n < NS; ++n) vr[n] = *reinterpret_cast<const v4u*>(p + (tid / 4 + n * 64) * page);
    };
    auto stage = [&](int t, const v4u (&kr)[NS], v4u (&vr)[NS]) __attribute__((always_inline)) {
        const int b = t & (RING - 1), there = s_meta[t & 7][tid & 3][0] >= 0 ? un.len - (base_of(t) + (tid & 3) * 16) : 0;
        if (there < 16) {                                // values of keys that are not there: anything may be in their place
            const v4u keep = first_bytes(there);
#pragma unroll
            for (int n = 0; n < NS; ++n) vr[n] &= keep;
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            const int i = tid + n * 256, row = i / KCH, d = tid / 4 + n * 64;
            s_k[b][row * KCH + ((i % KCH) ^ kswz(row))] = kr[n];
            s_v[b][d * 4 + ((tid & 3) ^ ((d >> 2) & 3))] = vr[n];
        }
    };

    // queries: row rho0 + wave*32 + col, as the second operand
    const int rho = un.rho0 + wave * 32 + col, rho_last = min(un.rho0 + wave * 32 + 31, un.rows - 1);
    const bool live = un.rho0 + wave * 32 < un.rows, ok = rho < un.rows;
    const int tok = ok ? rho / a.group : 0, qh = head * a.group + (ok ? rho % a.group : 0);
    const int pos = un.pos0 + tok, pmin = un.pos0 + (un.rho0 + wave * 32) / a.group, pmax = un.pos0 + rho_last / a.group;
    v4u q[kFar ? 1 : KCH];
    {
        const uint16_t* p = a.q + (int64_t)(un.token0 + tok) * a.ld_q + (int64_t)qh * D + h * 16;
#pragma unroll
        for (int i = 0; i < KCH; ++i) {
            const v4u x = ok ? *reinterpret_cast<const v4u*>(p + (i >> 1) * 32 + (i & 1) * 8) : v4u{0, 0, 0, 0};
            if constexpr (kFar) s_q[wave][i][lane] = x;
            else q[i] = x;
        }
    }
    auto query = [&](int i) __attribute__((always_inline)) {
        if constexpr (kFar) return __builtin_bit_cast(v8bf, s_q[wave][i][lane]);
        else return __builtin_bit_cast(v8bf, q[i]);
    };
    const float slope = a.slopes ? a.slopes[qh] * kLog2e : 0.0f;
    const Cap cap = cap_of(a);
    const float mul = cap.mul;
    const bool bent = a.cap > 0.0f || a.slopes != nullptr || !(mul > 0.0f);
    const float by = bent ? 1.0f : mul;
    const bool causal = a.window == 0 && un.prefix == 0;

    v16f o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
    float m = -INFINITY, l = 0.0f;

    auto multiply = [&](int t, int b) __attribute__((always_inline)) {
        const int kb = base_of(t);
        const int kblk = ((col >> 2) & 1) * 2;
        v16f s[2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[tt][i] = 0.0f;
            const float ks = exponent_value(s_meta[t & 7][kblk + tt][1]);
            const int row = tt * 32 + col;
#pragma unroll
            for (int kc = 0; kc < KCH / 2; ++kc) {
                const v4u x = s_k[b][row * KCH + ((kc * 2 + h) ^ kswz(row))];
                s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode8(x.x, x.y, ks), query(kc * 2), s[tt], 0, 0, 0);
                s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode8(x.z, x.w, ks), query(kc * 2 + 1), s[tt], 0, 0, 0);
                if constexpr (kFar) __builtin_amdgcn_sched_barrier(0);      // (all reads at once would not fit the registers)
            }
        }
        bool vok[2];
        int vse[2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            vok[tt] = s_meta[t & 7][h * 2 + tt][0] >= 0;
            vse[tt] = s_meta[t & 7][h * 2 + tt][2];
        }
        const bool whole = kb + kTile <= un.len && __all(vok[0] && vok[1]) &&
                           ((kb + kTile - 1 <= pmin && kb >= window_begin(a, pmax)) || kb + kTile <= un.prefix);
        if (bent) {
            if (a.cap > 0.0f) {
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[tt][i] = capped(s[tt][i], cap);
            } else {
#pragma unroll
                for (int tt = 0; tt < 2; ++tt) s[tt] *= mul;
            }
            if (a.slopes) {
                const float far = (float)(pos - (kb + h * 32));
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[tt][i] -= slope * fabsf(far - (float)(tt * 16 + i));
            }
        }
        if (!whole) {
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                if (causal) {                            // (a third of the instructions)
                    const int hi = vok[tt] ? min(pos + 1, un.len) - (kb + h * 32 + tt * 16) : 0;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[tt][i] = i < hi ? s[tt][i] : -INFINITY;
                    continue;
                }
                const Sight v = sight_of(a, un, vok[tt] ? pos : -1, kb + h * 32 + tt * 16);
                const int pre = vok[tt] ? v.pre : 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[tt][i] = sees(Sight{v.from, v.count, pre}, i) ? s[tt][i] : -INFINITY;
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            float x = s[tt][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) x = fmaxf(x, s[tt][i]);
            top = fmaxf(top, x * by + (float)(vse[tt] - 127));
        }
        top = max_xor32(top);
        if (__any(top > m + kSlack)) {
            const float mn = fmaxf(m, top), f = exp2_fast(m - (mn == -INFINITY ? 0.0f : mn));
            m = mn;
            l *= f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] *= f;
        }
        const float ref = kTop - (m == -INFINITY ? 0.0f : m);
        v8h p[2][2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const float shift = (float)(vse[tt] - 127) + ref;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float w = exp2_fast(__builtin_fmaf(s[tt][i], by, shift));
                sum += w;
                p[tt][i >> 3][i & 7] = (_Float16)w;
            }
            l += sum * exponent_value(254 - vse[tt]);
        }
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const int d = dt * 32 + col;
                const v4u x = s_v[b][d * 4 + ((h * 2 + tt) ^ ((d >> 2) & 3))];
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(decode8h(x.x, x.y), p[tt][0], o[dt], 0, 0, 0);
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(decode8h(x.z, x.w), p[tt][1], o[dt], 0, 0, 0);
                if constexpr (D > 128) __builtin_amdgcn_sched_barrier(0);
            }
        }
    };

    // Tiles go STEP at a time: while they are multiplied, as many behind them are requested, one ahead of each product, and staged,
    // and the pages of as many behind those are looked up, with their ids read another step before.  One barrier a step.
    auto put_meta = [&](int t, int blk, const Block& x) __attribute__((always_inline)) {
        s_meta[t & 7][blk][0] = x.id;
        s_meta[t & 7][blk][1] = x.ks;
        s_meta[t & 7][blk][2] = x.vs;
    };
    if (tid < 8 * STEP && tile0 + tid / 4 < tile_end) put_meta(tile0 + tid / 4, tid & 3, load_block(c, a, un, head, tile0 + tid / 4, tid & 3));
    int ahead = tid < 4 * STEP && tile0 + 2 * STEP + tid / 4 < tile_end ? page_id(tile0 + 2 * STEP + tid / 4, tid & 3) : -1;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < STEP; ++n)
        if (tile0 + n < tile_end) {
            fetch(tile0 + n, kx, vx);
            stage(tile0 + n, kx, vx);
        }
    __syncthreads();
    for (int t = tile0; t < tile_end; t += STEP) {
        const int tm = t + 2 * STEP + tid / 4;           // (of the first 4 STEP lanes; before the codes, which need not have come)
        Block blk = {ahead, 127, 127, {0, 0}};
        if (tid < 4 * STEP && tm < tile_end) {
            if (ahead >= 0) {
                blk.ks = scale_byte(c.k_scales, (int64_t)ahead * c.heads + head);
                blk.vs = scale_byte(c.v_scales, (int64_t)ahead * c.heads + head);
            }
            ahead = tm + STEP < tile_end ? page_id(tm + STEP, tid & 3) : -1;
        }
#pragma unroll
        for (int n = 0; n < STEP; ++n) {
            const int kb = base_of(t + n);
            if (t + n + STEP < tile_end) fetch(t + n + STEP, kx, vx);
            if (t + n < tile_end && live && (kb < un.prefix || (kb <= pmax && kb + kTile > window_begin(a, pmin)))) multiply(t + n, (t + n) & (RING - 1));
            if (t + n + STEP < tile_end) stage(t + n + STEP, kx, vx);
        }
        if (tid < 4 * STEP && tm < tile_end) put_meta(tm, tid & 3, blk);
        __syncthreads();
    }

    l += __shfl_xor(l, 32);
    if (!ok) return;
    if (parts == 1) {
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        uint16_t* p = a.out + (int64_t)(un.token0 + tok) * a.ld_out + (int64_t)qh * D + h * 4;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const v4bf y = {(__bf16)(o[dt][b * 4] * inv), (__bf16)(o[dt][b * 4 + 1] * inv), (__bf16)(o[dt][b * 4 + 2] * inv), (__bf16)(o[dt][b * 4 + 3] * inv)};
                *reinterpret_cast<v4bf*>(p + dt * 32 + b * 8) = y;
            }
    } else {
        float* wo = ws + ((int64_t)(u * c.heads + head) * splits + part) * M * (D + 2);
        const int r = wave * 32 + col;
        if (h == 0) {
            wo[r] = m;
            wo[M + r] = l;
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                *reinterpret_cast<v4f*>(wo + 2 * M + r * D + dt * 32 + b * 8 + h * 4) = v4f{o[dt][b * 4], o[dt][b * 4 + 1], o[dt][b * 4 + 2], o[dt][b * 4 + 3]};
    }
}

// Joins the chunks of the units that were split, in the order of the keys. A wave has 256 / D rows of one unit and head.
template <int D>
__global__ __launch_bounds__(256) void attention_join_kernel(CacheView c, AttentionArgs a, int m, int splits, int chunk, const float* __restrict__ ws)
{
    constexpr int RB = 256 / D, L4 = D / 4;
    const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), blocks = m / (4 * RB);
    const int block = blockIdx.x % blocks, rest = blockIdx.x / blocks, head = rest % c.heads, u = rest / c.heads;
    Unit un;
    if (!find_unit(a, c.lp, u, m, un)) return;
    const int parts = min(splits, max(1, (un.tiles + chunk - 1) / chunk));
    const int rr = lane / L4, d = lane % L4 * 4, r = (block * 4 + wave) * RB + rr, rho = un.rho0 + r;
    if (parts == 1 || rr >= RB || rho >= un.rows) return;
    const int64_t size = (int64_t)m * (D + 2);
    const float* w = ws + (int64_t)(u * c.heads + head) * splits * size;
    float top = -INFINITY, sum = 0.0f;
    v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
        const float* wp = w + p * size;
        const float mp = wp[r], lp = wp[m + r];
        const v4f xp = *reinterpret_cast<const v4f*>(wp + 2 * m + r * D + d);
        const float mn = fmaxf(top, mp), ref = mn == -INFINITY ? 0.0f : mn, f = exp2_fast(top - ref), fp = exp2_fast(mp - ref);
        x = x * f + xp * fp;
        sum = sum * f + lp * fp;
        top = mn;
    }
    *reinterpret_cast<v4bf*>(out_at(a, un.token0, head, rho, D) + d) = finished(x, sum);
}

// How a call is cut up: the same for the workspace query and the launch.  Rows of a request that fill more than two units of 16
// would have their keys read and converted three times and more: they go to the kernel that shares a tile among 128 (units of 16 against
// of 128, joins included, us; D = 128, 8 heads: 8 requests of 4096 keys, 32 rows 28.4 / 29.4, 48 38.8 / 35.8, 96 53.5 / 41.5; one of 16384, 32 rows 28.0 / 28.2,
// 64 30.0 / 30.4, 96 38.1 / 32.6; 64 of 2048, 32 rows 66.7 / 91.6, 64 105 / 159, 96 167 / 164.  At D = 64 and 256 units of 16 stay ahead up to 64 rows: 8 of 4096
// keys, D = 64 24.0 / 27.6, D = 256 45.6 / 52.6; at 96 rows they are behind there too, 32.0 / 30.6 and 57.4 / 55.8).  With
// fewer rows, short batches that fit one workgroup a unit need no join (D = 128, whole units against shares, us: 1 request,
// 8 heads, 1024 keys 10.8 / 13.9, 2048 keys 16.3 / 13.9; 4 requests, 32 heads, 2048 keys 17.4 / 21.2, 4096 keys 29.2 / 30.5;
// 32 requests, 8 heads, 2048 keys 24.9 / 30.6): up to 24 tiles where they leave most of the card idle, else up to 32.
struct Cut {
    enum { kWhole, kShared, kTiles } kind;   // attention_rows_kernel, attention_shares_kernel, attention_tiles_kernel
    int64_t units;                           // bound on the units of one key/value head
    int splits, chunk;                       // kTiles: chunks of tiles per unit, tiles per chunk
    int most;                                // kTiles: chunks before their size is rounded: more with more tiles, never fewer than `splits`
    bool once;                               // kShared: a request's rows are expected to fit one unit, so that its keys are read once
};
constexpr int kTilesM = 128;

static Cut cut_of(const CacheView& c, const AttentionArgs& a, int64_t max_new, int64_t max_len)
{
    Cut o;
    const int64_t rows = (int64_t)a.tokens * a.group;
    if (max_new <= 0 || max_new > a.tokens) max_new = a.tokens;
    if (max_len <= 0 || max_len > ((int64_t)a.width << c.lp)) max_len = (int64_t)a.width << c.lp;
    int64_t tiles = std::max<int64_t>(1, (max_len + kTile - 1) / kTile);
    if (a.window > 0) tiles = std::min<int64_t>(tiles, ((int64_t)a.window + max_new) / kTile + 3);   // (and a short prefix)
    o.splits = o.most = 1;
    o.once = max_new * a.group <= 16;
    o.chunk = (int)std::min<int64_t>(tiles, 1 << 24);
    if (max_new * a.group > 32) {
        o.kind = Cut::kTiles;
        o.units = a.requests == 1 ? (rows + kTilesM - 1) / kTilesM : rows / kTilesM + a.requests;
        const int64_t busy = std::max<int64_t>(1, std::max<int64_t>(std::min<int64_t>(a.requests, a.tokens), (rows + kTilesM - 1) / kTilesM) * c.heads);
        const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({kComputeUnits * 2 / busy, tiles / 8, (int64_t)((1 << 24) - 1) / (o.units * c.heads * 64)}));
        o.most = (int)splits;
        o.chunk = (int)std::min<int64_t>((tiles + splits - 1) / splits, 1 << 24);
        o.splits = (int)((tiles + o.chunk - 1) / o.chunk);
        return o;
    }
    o.units = a.requests == 1 ? (rows + 15) / 16 : rows / 16 + a.requests;
    o.kind = tiles <= (o.units * c.heads <= kComputeUnits / 4 ? 24 : 32) && o.units * c.heads <= kComputeUnits ? Cut::kWhole : Cut::kShared;
    return o;
}

static size_t piece_bytes(int dim, int m) { return (size_t)m * (dim + 2) * sizeof(float); }

static size_t workspace_of(const CacheView& c, const Cut& k, int splits)
{
    if (k.kind == Cut::kShared) return shares_of(c.dim) * (sizeof(Share) + 2 * (32 + 16 * (c.dim + 4)) * sizeof(float));
    return splits == 1 ? 0 : (size_t)k.units * c.heads * splits * piece_bytes(c.dim, kTilesM);
}

// Neither the kind's need nor `most` goes down as tiles become more: enough for every shorter length, and without a window for
// every window.
size_t attention_workspace_bytes(const CacheView& c, const AttentionArgs& a, int64_t max_new, int64_t max_len)
{
    const Cut k = cut_of(c, a, max_new, max_len);
    return workspace_of(c, k, k.most);
}

size_t attention_workspace_used(const CacheView& c, const AttentionArgs& a, int64_t max_new, int64_t max_len)
{
    const Cut k = cut_of(c, a, max_new, max_len);
    return workspace_of(c, k, k.splits);
}

template <int D>
static hipError_t launch_dim(const CacheView& c, const AttentionArgs& a, const Cut& k, float* ws, hipStream_t st)
{
    if (k.kind == Cut::kTiles) {
        const int64_t n = k.units * c.heads * k.splits;
        launch(attention_tiles_kernel<D>, dim3((unsigned)n), 256, 0, st, c, a, (int)k.units, (int)(k.splits == 1 && n <= 2 * kComputeUnits), k.splits, k.chunk, ws);
        if (k.splits > 1)
            launch(attention_join_kernel<D>, dim3((unsigned)(k.units * c.heads * (kTilesM / (4 * (256 / D))))), 256, 0, st, c, a, kTilesM, k.splits, k.chunk, ws);
    } else if (k.kind == Cut::kWhole) {
        constexpr int NW = 8;
        launch(attention_rows_kernel<D, NW>, dim3((unsigned)(k.units * c.heads)), 64 * NW, 0, st, c, a);
    } else {
        Share* shares = reinterpret_cast<Share*>(ws);
        constexpr int n = shares_of(D);
        float* pieces = reinterpret_cast<float*>(shares + n);
        const dim3 block(64 * share_waves(D));
        if (!k.once) launch(attention_shares_kernel<D, 0>, dim3(n), block, 0, st, c, a, shares, pieces);
        else if (c.lp == 7) launch(attention_shares_kernel<D, 1>, dim3(n), block, 0, st, c, a, shares, pieces);
        else launch(attention_shares_kernel<D, 2>, dim3(n), block, 0, st, c, a, shares, pieces);
        launch(attention_join_shares_kernel<D>, dim3(n), 1024, 0, st, a, shares, pieces);
    }
    return hipGetLastError();
}

hipError_t launch_attention(const CacheView& c, const AttentionArgs& a, int64_t max_new, int64_t max_len, float* ws, hipStream_t st)
{
    const Cut k = cut_of(c, a, max_new, max_len);
    switch (c.dim) {
        case 64: return launch_dim<64>(c, a, k, ws, st);
        case 128: return launch_dim<128>(c, a, k, ws, st);
        case 192: return launch_dim<192>(c, a, k, ws, st);
        default: return launch_dim<256>(c, a, k, ws, st);
    }
}

}  // namespace razer
