// Root-mean-square norm with the residual's addition (include/razer_step.h) for gfx950.
//
//   h = x + r;   s = fp32(1 / sqrt(mean(h^2) + eps));   y = (h s) (offset + w)
//
// A row stays in registers between its two uses, so that x, r and w are read once and nothing else is.  The mean is formed
// in 64 bits: a square of an fp32 number is exact there, the order of the sum leaves no trace in the fp32 root but once in
// some 10^8 rows, and codes that are encoded from y come out the same whatever the launch shape.  It costs a conversion and
// one fma per element, on a vector unit that runs 64-bit operations at the 32-bit rate and waits for memory here.
//   Bound by memory in long calls (4096 rows of 8192, bf16 with residual: 268 MB in 47 us, 5.7 TB/s, a large copy's 5.1), and by
// the way of one row through a workgroup in short ones (one row of 4096 2.7 us, 64 rows of 8192 into codes 6.2 us).
#include "razer_encode.hpp"
#include "razer_kernels.hpp"
#include "razer_step.hpp"

namespace razer {

namespace {

struct NormArgs {
    const void* x;
    const void* residual;
    void* sum;
    const void* weight;
    void* out;
    uint8_t* codes;
    uint8_t* scales;
    const float* tensor_scale;
    int64_t ld_x, ld_residual, ld_sum, ld_out, rows;
    uint32_t cols;
    int x_bf16, res_bf16, w_bf16, out_bf16, lb;
    float eps, offset, sv0;
};

// VEC consecutive elements at element i of p as fp32
template <int VEC>
__device__ __forceinline__ void load_f32(float* v, const void* p, uint32_t i, bool bf16)
{
    if (bf16) {
        uint4 t[VEC / 8];
#pragma unroll
        for (int j = 0; j < VEC / 8; ++j) t[j] = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i)[j];
#pragma unroll
        for (int j = 0; j < VEC / 8; ++j) {
            const uint32_t w[4] = {t[j].x, t[j].y, t[j].z, t[j].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                v[8 * j + 2 * q] = u2f(w[q] << 16);
                v[8 * j + 2 * q + 1] = u2f(w[q] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < VEC / 4; ++j) {
            const float4 t = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i)[j];
            v[4 * j] = t.x; v[4 * j + 1] = t.y; v[4 * j + 2] = t.z; v[4 * j + 3] = t.w;
        }
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    v2bf t = {(__bf16)a, (__bf16)b};                                       // v_cvt_pk_bf16_f32: nearest, ties to even
    return __builtin_bit_cast(uint32_t, t);
}
template <int VEC>
__device__ __forceinline__ void store_f32(void* p, uint32_t i, const float* v, bool bf16)
{
    if (bf16) {
#pragma unroll
        for (int j = 0; j < VEC / 8; ++j)
            reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i)[j] =
                make_uint4(pack_bf16(v[8 * j], v[8 * j + 1]), pack_bf16(v[8 * j + 2], v[8 * j + 3]),
                           pack_bf16(v[8 * j + 4], v[8 * j + 5]), pack_bf16(v[8 * j + 6], v[8 * j + 7]));
    } else {
#pragma unroll
        for (int j = 0; j < VEC / 4; ++j)
            reinterpret_cast<float4*>(static_cast<float*>(p) + i)[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    }
}

// 1 / sqrt(mean + eps) from the threads' sums of squares
__device__ __forceinline__ float inverse_rms(double ss, double* part, const NormArgs& a)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
    if (blockDim.x > 64) {
        if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = ss;
        __syncthreads();
        ss = 0.0;
        for (uint32_t i = 0; i < blockDim.x >> 6; ++i) ss += part[i];
    }
    return (float)(1.0 / __builtin_sqrt(ss / (double)a.cols + (double)a.eps));
}

// One workgroup per row; a thread holds N pieces of VEC elements, piece i at ((i threads) + thread) VEC.  G > 0: the pieces
// are runs of 16 elements and go through the block encoder in blocks of 16 G.
template <bool XB, int VEC, int N, int G>
__global__ __launch_bounds__(1024) void norm_kernel(const NormArgs a)
{
    static_assert(G == 0 || VEC == kBlock, "the encoder takes runs of 16");
    __shared__ double part[16];
    const int64_t row = blockIdx.x;
    const uint32_t threads = blockDim.x, tid = threadIdx.x;
    auto row_of = [&](const void* p, int64_t ld, bool bf16) { return static_cast<const uint8_t*>(p) + row * ld * (bf16 ? 2 : 4); };
    const void* x = row_of(a.x, a.ld_x, XB);
    float h[N][VEC], w[N][VEC];                                            // (the weights too ahead of the sum)
    double ss = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t c = (i * threads + tid) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) h[i][j] = 0.0f;
        if (c < a.cols) load_f32<VEC>(h[i], x, c, XB);
    }
    if (a.residual) {
        const void* residual = row_of(a.residual, a.ld_residual, a.res_bf16);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t c = (i * threads + tid) * VEC;
            float r[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) r[j] = 0.0f;
            if (c < a.cols) load_f32<VEC>(r, residual, c, a.res_bf16);
#pragma unroll
            for (int j = 0; j < VEC; ++j) h[i][j] += r[j];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t c = (i * threads + tid) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) w[i][j] = 0.0f;
        if (c < a.cols) load_f32<VEC>(w[i], a.weight, c, a.w_bf16);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) ss = __builtin_fma((double)h[i][j], (double)h[i][j], ss);
    if (a.sum) {
        void* sum = const_cast<uint8_t*>(row_of(a.sum, a.ld_sum, a.res_bf16));
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t c = (i * threads + tid) * VEC;
            if (c < a.cols) store_f32<VEC>(sum, c, h[i], a.res_bf16);
        }
    }
    const float s = inverse_rms(ss, part, a);
    const float delta = G > 0 ? *a.tensor_scale : 1.0f;
    void* out = a.out ? const_cast<uint8_t*>(row_of(a.out, a.ld_out, a.out_bf16)) : nullptr;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t c = (i * threads + tid) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) h[i][j] = (h[i][j] * s) * (a.offset + w[i][j]);
        if (c < a.cols && out) store_f32<VEC>(out, c, h[i], a.out_bf16);
        if constexpr (G > 0) {
            uint32_t lo, hi, meta, sc;
            encode_run<1, G, false>(h[i], delta, a.sv0, 0.0f, false, lo, hi, meta, sc);
            if (c < a.cols) {                                              // (a block's lanes are all inside a row, or none)
                *reinterpret_cast<uint2*>(a.codes + ((row * a.cols + c) >> 1)) = make_uint2(lo, hi);
                if ((tid & (G - 1)) == 0) a.scales[(row * a.cols + c) >> a.lb] = (uint8_t)((meta << 7) | sc);
            }
        }
    }
}

// Rows that no vector fits (odd sizes, strides or addresses): element by element, read twice.  A thread writes an element
// after it has read it for the last time.
__global__ __launch_bounds__(512) void norm_any_kernel(const NormArgs a)
{
    __shared__ double part[16];
    const int64_t row = blockIdx.x;
    auto get = [](const void* p, int64_t i, bool bf16) { return bf16 ? bf16_bits_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i]; };
    auto put = [](void* p, int64_t i, float v, bool bf16) {
        if (bf16) static_cast<uint16_t*>(p)[i] = f32_to_bf16_rne(v);
        else static_cast<float*>(p)[i] = v;
    };
    auto element = [&](uint32_t c) {
        float h = get(a.x, row * a.ld_x + c, a.x_bf16);
        if (a.residual) h += get(a.residual, row * a.ld_residual + c, a.res_bf16);
        return h;
    };
    double ss = 0.0;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
        const double h = (double)element(c);
        ss = __builtin_fma(h, h, ss);
    }
    const float s = inverse_rms(ss, part, a);
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
        const float h = element(c);
        if (a.sum) put(a.sum, row * a.ld_sum + c, h, a.res_bf16);
        if (a.out) put(a.out, row * a.ld_out + c, (h * s) * (a.offset + get(a.weight, c, a.w_bf16)), a.out_bf16);
    }
}

template <bool XB, int VEC, int G>
hipError_t launch_norm_n(const NormArgs& a, hipStream_t st)
{
    const uint32_t vecs = (a.cols + VEC - 1) / VEC;
    auto go = [&](auto kern, uint32_t n) {
        const uint32_t threads = ((vecs + n - 1) / n + 63) & ~63u;
        launch(kern, (uint32_t)a.rows, threads, 0, st, a);
        return hipGetLastError();
    };
    if constexpr (VEC == 8) {
        if (vecs <= 1024) return go(norm_kernel<XB, VEC, 1, 0>, 1);
        return go(norm_kernel<XB, VEC, 4, 0>, 4);
    } else {
        if (vecs <= 1024) return go(norm_kernel<XB, VEC, 1, G>, 1);
        return go(norm_kernel<XB, VEC, 2, G>, 2);
    }
}
template <bool XB>
hipError_t launch_norm_x(const NormArgs& a, hipStream_t st)
{
    if (a.codes) {
        switch (a.lb) {
            case 4: return launch_norm_n<XB, 16, 1>(a, st);
            case 5: return launch_norm_n<XB, 16, 2>(a, st);
            case 6: return launch_norm_n<XB, 16, 4>(a, st);
            default: return launch_norm_n<XB, 16, 8>(a, st);
        }
    }
    return launch_norm_n<XB, 8, 0>(a, st);
}

bool good_dtype(int32_t d) { return d == RAZER_F32 || d == RAZER_BF16; }
int64_t bytes_of(int32_t d) { return d == RAZER_BF16 ? 2 : 4; }

}  // namespace

}  // namespace razer

using namespace razer;

extern "C" razer_status razer_norm(const razer_norm_args* g, void* hip_stream)
{
    if (!g) return RAZER_ERR_NULL;
    if (!good_dtype(g->x_dtype) || !good_dtype(g->weight_dtype) || (g->residual && !good_dtype(g->residual_dtype)) || (g->out && !good_dtype(g->out_dtype)))
        return RAZER_ERR_CONFIG;
    if (!(g->eps >= 0.0f)) return RAZER_ERR_CONFIG;
    int lb = 0;
    float sv0 = 0.0f;
    if (g->codes) {
        SvConfig cfg;
        if (g->cfg.format != RAZER_FMT_ACT || g->cfg.layout != RAZER_LAYOUT_CANONICAL || check_cfg(g->cfg, cfg) != RAZER_OK) return RAZER_ERR_CONFIG;
        lb = cfg.lb;
        sv0 = cfg.sv0;
    }
    if (g->rows < 0 || g->rows >= ((int64_t)1 << 22) || g->cols < 0 || g->cols > 32768) return RAZER_ERR_SHAPE;
    if (g->codes && (g->cols % 32 != 0 || (g->cols & (((int64_t)1 << lb) - 1)) != 0)) return RAZER_ERR_SHAPE;
    if (g->rows == 0 || g->cols == 0) return RAZER_OK;
    if (g->ld_x < g->cols || (g->residual && g->ld_residual < g->cols) || (g->sum && g->ld_sum < g->cols) || (g->out && g->ld_out < g->cols)) return RAZER_ERR_SHAPE;
    if (!g->x || !g->weight || (!g->out && !g->codes && !g->sum) || (g->sum && !g->residual)) return RAZER_ERR_NULL;
    if (g->codes && (!g->scales || !g->tensor_scale)) return RAZER_ERR_NULL;
    bool wide = g->cols % 8 == 0;
    auto check = [&](const void* p, int64_t ld, int32_t dtype) {           // false: not even aligned to its elements
        const uintptr_t u = reinterpret_cast<uintptr_t>(p);
        if (u % 16 != 0 || ld * bytes_of(dtype) % 16 != 0) wide = false;
        return u % bytes_of(dtype) == 0;
    };
    if (!check(g->x, g->ld_x, g->x_dtype) || !check(g->weight, 8, g->weight_dtype) || (g->residual && !check(g->residual, g->ld_residual, g->residual_dtype)) ||
        (g->sum && !check(g->sum, g->ld_sum, g->residual_dtype)) || (g->out && !check(g->out, g->ld_out, g->out_dtype)))
        return RAZER_ERR_ALIGN;
    if (g->codes && (!wide || !aligned16(g->codes) || !aligned16(g->scales) || reinterpret_cast<uintptr_t>(g->tensor_scale) % 4 != 0)) return RAZER_ERR_ALIGN;
    NormArgs a{g->x, g->residual, g->sum, g->weight, g->out, g->codes, g->scales, g->tensor_scale, g->ld_x, g->ld_residual, g->ld_sum, g->ld_out, g->rows,
               (uint32_t)g->cols, g->x_dtype == RAZER_BF16, g->residual_dtype == RAZER_BF16, g->weight_dtype == RAZER_BF16, g->out_dtype == RAZER_BF16, lb, g->eps, g->weight_offset, sv0};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipError_t e;
    if (wide) {
        e = g->x_dtype == RAZER_BF16 ? launch_norm_x<true>(a, st) : launch_norm_x<false>(a, st);
    } else {
        launch(norm_any_kernel, (uint32_t)g->rows, g->cols <= 256 ? 64 : 512, 0, st, a);
        e = hipGetLastError();
    }
    return e == hipSuccess ? RAZER_OK : RAZER_ERR_HIP;
}
