// RaZeR block encoder for gfx950: Eq. 1 (tensor scale), Eq. 2 (block scale),
// Eq. 4 (special-value search) and Eq. 5 (final rounding) of arxiv 2501.04052.
//
// Bit-exactness contract: codes, scales and the tensor scale are those of the literal computation -- every fp32
// operation a single IEEE operation (true division), squared errors summed in fp64 over the block's elements in index
// order (also for blocks of 32, 64, 128 -- the block-size study of Sec. 5.4 -- where the lanes that share a block
// hand the running sum from one to the next), ties broken as documented in razer.h.  The block encoder reaches most
// of these results by cheaper operations that are proven to give the same bits; the proofs are stated there.
// Compile without fast-math.
#include "razer_encode.hpp"
#include "razer_kernels.hpp"

namespace razer {

// ---------------------------------------------------------------- absmax (Eq. 1)
// The running maximum lives in kAbsmaxCells cells of the workspace (workgroup b updates cell
// b % kAbsmaxCells): atomics on a single address serialize at roughly 10 ns each, so a thousand
// workgroups on one cell cost more than the pass over a 32 MB tensor itself.
constexpr int kAbsmaxCells = 64;
constexpr int kAbsmaxBlocks = 256, kAbsmaxRowBlocks = 1024;     // dense; strided rows (one load in flight per lane)
constexpr int64_t kAbsmaxOnceBytes = (int64_t)96 << 20;
__global__ void absmax_init_kernel(uint32_t* ws) { ws[threadIdx.x] = 0u; }

// max over the cells, by every wavefront that needs it (64 lanes, one cell each)
__device__ __forceinline__ float absmax_from_cells(const uint32_t* __restrict__ ws)
{
    uint32_t m = ws[threadIdx.x & 63u];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
    return u2f(m);
}

// Bound by the read.  One workgroup per compute unit with eight loads in flight per lane: more workgroups only add
// atomics and a tail (encoder with this pass, 256 against 1024 workgroups of four loads: bf16 4096 x 4096 27.5 -> 24.8 us,
// fp32 4096 x 4096 49.7 -> 48.0; eight loads alone 27.0, 48.9).  ONCE: a tensor too large to stay in the last-level
// cache until the encoder reads it again is read around the caches (fp32 8192 x 8192 with its decoding 157 -> 146 us, bf16
// 14336 x 4096, 117 MB, 111 -> 101; 67 MB of bf16 would take 42.2 instead of 41.5, hence the line at 96 MiB).
template <typename T, bool ONCE>
__global__ __launch_bounds__(256) void absmax_kernel(const T* __restrict__ x, int64_t rows, int64_t cols,
                                                     int64_t ld, uint32_t* __restrict__ ws)
{
    // 16-byte vectors: 4 floats or 8 bf16.  |x| of finite non-negative floats orders like uint32.
    constexpr int VEC = 16 / sizeof(T);
    __shared__ uint32_t wmax[4];
    uint32_t m = 0;
    auto fold = [&](const uint4& v) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (sizeof(T) == 4) {
                m = max(m, w[j] & 0x7FFFFFFFu);
            } else {
                m = max(m, (w[j] << 16) & 0x7FFFFFFFu);
                m = max(m, w[j] & 0x7FFF0000u);
            }
        }
    };
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    if (ld == cols) {                                   // dense: one flat array of vectors
        const int64_t total = rows * cols / VEC;
        const uint4* p = reinterpret_cast<const uint4*>(x);
        int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
        for (; i + 7 * stride < total; i += 8 * stride) {        // eight loads in flight per lane
            uint4 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (ONCE) v[j] = load_once16(p + i + j * stride);
                else v[j] = p[i + j * stride];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) fold(v[j]);
        }
        for (; i < total; i += stride) fold(p[i]);
    } else {                                            // strided rows: workgroups stride over rows
        const int64_t vec_per_row = cols / VEC;
        for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
            const uint4* p = reinterpret_cast<const uint4*>(x + r * ld);
            for (int64_t c = threadIdx.x; c < vec_per_row; c += blockDim.x) fold(p[c]);
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
    if ((threadIdx.x & 63) == 0) wmax[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) atomicMax(ws + (blockIdx.x % kAbsmaxCells), max(max(wmax[0], wmax[1]), max(wmax[2], wmax[3])));
}

// ---------------------------------------------------------------- block encoder
// A thread encodes runs of 16 elements; G = block / 16 consecutive lanes share a block: they
// agree on the block maximum (hence on the scale) by exchanging their run's maximum, and on the
// special value.
//
// What bounds it: written out literally (IEEE division, four fp64 error sums) an element costs about 220 clocks of
// a SIMD, twice what its bytes take from memory.  Two things make it cheaper without changing a bit:
//  * division.  y = 1 / den is one IEEE division per block; q = x y, then twice q += (x - q den) y with the residual
//    in one fma.  The first correction makes q faithful, and for a faithful q, a correctly rounded reciprocal and an
//    exact residual the second yields the correctly rounded quotient (Markstein's theorem); 5 operations instead of
//    ~12.  It needs normal operands: den below 2^-70 and tensor scales above 2^60 take the literal path (an element
//    whose residual is still subnormal is below 2^-30 after scaling and leaves no trace in a sum that decides anything).
//  * the special-value search.  Candidate v lowers an element's squared error by (v - q)(2 x - q - v) when that is
//    positive; sign and zero of that product are exact in fp32 (2 x - q is exact, and so is the difference to v where
//    it is close to it), so "no element takes v" and the elements that take it are known exactly, and the sums of the
//    gains to a relative error below (elements + 8) 2^-23.  The candidate with the largest gain has the smallest error
//    where the others are further away than that bound.  Where one other is not, the fp64 sums of Eq. 4 are formed for
//    those two alone (nearest_two): 16-bit data, with few distinct magnitudes, ties in about one block of 400, so one
//    wave in seven goes there.  Only what is left -- three candidates that close, non-finite blocks, blocks beyond 512
//    scales -- takes the literal chain.
// A thread has one run until the launch has 2^20; such launches wait for loads and for the slowest wave, the larger
// ones for vector issue with as many waves as registers allow.  Hence the next run is fetched while one is encoded
// (AHEAD) for 16-bit elements (8 registers, 3 % at 4096 x 4096) and for fp32 weights in blocks of 16 (11008 x 4096 with
// Eq. 1's pass 78.2 -> 76.0), not where the 16 registers of fp32 cost more waves (blocks of 64 and 128, 3-5 %) or launches
// seldom reach 2^20 runs (activations); scaled 16-bit elements are kept for nearest_two, fp32 ones are scaled again there.
// Measured against the kernel that formed all four fp64 sums for every block (us per dispatch, tensor scale given; in
// parentheses with ties decided by the literal chain): bf16 activations 4096 wide, 64 rows 5.0 (5.8) -> 5.0, 512 rows
// 6.1 (6.9) -> 5.6, 1024 rows 8.3 (8.8) -> 7.6, 4096 rows 20.2 (18.1) -> 15.6; bf16 weights in blocks of 128, 256 rows
// 7.1 (10.7) -> 6.9, 4096 rows 45.0 (27.4) -> 20.6; fp32 weights 11008 x 4096 in blocks of 16 62.0 (41.5) -> 39.3 (206 MB,
// 5.2 TB/s), of 128 120 (49.6) -> 42.4.

template <typename T, int FMT, int G>
__global__ __launch_bounds__(256) void encode_kernel(const T* __restrict__ x, int64_t rows, int64_t cols,
                                                     int64_t ld, float sv0, float sv1,
                                                     const uint32_t* __restrict__ absmax_ws,
                                                     float* __restrict__ tensor_scale, int given_scale,
                                                     uint8_t* __restrict__ codes, uint8_t* __restrict__ scales)
{
    constexpr int NV = (int)sizeof(T);                                    // 16-byte vectors per run
    constexpr bool B16 = sizeof(T) == 2, AHEAD = B16 || (G == 1 && FMT == 0);
    const int64_t nb = cols / kBlock, runs = rows * nb;
    const int64_t first_run = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, stride = (int64_t)gridDim.x * blockDim.x;
    auto load = [&](uint4 (&v)[NV], int64_t run) {
        // dense rows are one array of runs; only strided ones need the row number
        int64_t src = run * kBlock;
        if (ld != cols) {
            const int64_t r = run / nb;
            src = r * ld + (run - r * nb) * kBlock;
        }
        const uint4* xp = reinterpret_cast<const uint4*>(x + src);
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = xp[j];
    };
    uint4 next[NV];
    if (first_run < runs) load(next, first_run);

    float delta32;
    if (given_scale) {
        delta32 = *tensor_scale;
    } else {
        float amax = absmax_from_cells(absmax_ws);
        constexpr float kDenom = (FMT == 0) ? 180.0f : (FMT == 1) ? 2688.0f : 11.994140625f;   // Qmax_scale * 6
        delta32 = (amax == 0.0f) ? 1.0f : amax / kDenom;
        if (first_run == 0) *tensor_scale = delta32;
    }

    // several runs per thread
#pragma unroll 1
    for (int64_t gid = first_run; gid < runs; gid += stride) {
        float xv[kBlock];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t w[4] = {next[j].x, next[j].y, next[j].z, next[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (sizeof(T) == 4) {
                    xv[4 * j + i] = u2f(w[i]);
                } else {
                    xv[8 * j + 2 * i + 0] = u2f(w[i] << 16);
                    xv[8 * j + 2 * i + 1] = u2f(w[i] & 0xFFFF0000u);
                }
            }
        }
        if (AHEAD) load(next, gid + stride < runs ? gid + stride : gid);

        uint32_t lo, hi, meta, sc;
        encode_run<FMT, G, B16>(xv, delta32, sv0, sv1, !given_scale, lo, hi, meta, sc);
        *reinterpret_cast<uint2*>(codes + gid * 8) = make_uint2(lo, hi);
        if ((gid & (G - 1)) == 0) {                                           // (a row holds whole blocks)
            if (FMT == 2) reinterpret_cast<uint16_t*>(scales)[gid / G] = (uint16_t)((meta << 14) | sc);
            else scales[gid / G] = (uint8_t)((meta << (FMT == 0 ? 6 : 7)) | sc);
        }
        if (!AHEAD && gid + stride < runs) load(next, gid + stride);
    }
}

// ---------------------------------------------------------------- host launchers
constexpr int64_t kEncodeBlocks = 4096;    // workgroups of the encoder (1024 .. one run per thread: within 4 % of each other)
template <typename T, int FMT>
static void launch_encode(int lb, unsigned grid, unsigned threads, hipStream_t st, const T* x, int64_t rows,
                          int64_t cols, int64_t ld, SvConfig cfg, const uint32_t* ws, float* tensor_scale, int given,
                          uint8_t* codes, uint8_t* scales)
{
#define RAZER_ENC(G) launch(encode_kernel<T, FMT, G>, grid, threads, 0, st, x, rows, cols, ld, cfg.sv0, cfg.sv1, ws, tensor_scale, given, codes, scales)
    switch (lb) {
        case 4: RAZER_ENC(1); break;
        case 5: RAZER_ENC(2); break;
        case 6: RAZER_ENC(4); break;
        default: RAZER_ENC(8); break;
    }
#undef RAZER_ENC
}

template <typename T>
static hipError_t launch_quantize_t(int fmt, SvConfig cfg, const T* x, int64_t rows, int64_t cols, int64_t ld,
                                    uint8_t* codes, uint8_t* scales, float* tensor_scale, int given,
                                    uint32_t* ws, hipStream_t st)
{
    if (rows == 0 || cols == 0) {
        if (!given) {                       // an empty tensor gets the all-zero tensor's scale of 1
            launch(absmax_init_kernel, 1, kAbsmaxCells, 0, st, ws);
            if (fmt == 0) launch_encode<T, 0>(4, 1, 64, st, x, 0, 16, 16, cfg, ws, tensor_scale, 0, codes, scales);
            else launch_encode<T, 1>(4, 1, 64, st, x, 0, 16, 16, cfg, ws, tensor_scale, 0, codes, scales);
        }
        return hipGetLastError();
    }
    if (!given) {
        launch(absmax_init_kernel, 1, kAbsmaxCells, 0, st, ws);
        constexpr int VEC = 16 / sizeof(T);
        int64_t total = rows * (cols / VEC);
        int64_t blocks = (total + 255) / 256;
        const int64_t most = ld == cols ? kAbsmaxBlocks : kAbsmaxRowBlocks;
        if (blocks > most) blocks = most;
        if (rows * cols * (int64_t)sizeof(T) > kAbsmaxOnceBytes)
            launch(absmax_kernel<T, true>, (unsigned)blocks, 256, 0, st, x, rows, cols, ld, ws);
        else
            launch(absmax_kernel<T, false>, (unsigned)blocks, 256, 0, st, x, rows, cols, ld, ws);
    }
    int64_t nblk = rows * (cols / kBlock);
    unsigned grid = (unsigned)((nblk + 255) / 256 < kEncodeBlocks ? (nblk + 255) / 256 : kEncodeBlocks);
    if (fmt == 0) launch_encode<T, 0>(cfg.lb, grid, 256, st, x, rows, cols, ld, cfg, ws, tensor_scale, given, codes, scales);
    else if (fmt == 1) launch_encode<T, 1>(cfg.lb, grid, 256, st, x, rows, cols, ld, cfg, ws, tensor_scale, given, codes, scales);
    else launch(encode_kernel<T, 2, 8>, grid, 256, 0, st, x, rows, cols, ld, cfg.sv0, cfg.sv1, ws, tensor_scale, given, codes, scales);
    return hipGetLastError();
}

hipError_t launch_quantize(int fmt, SvConfig cfg, const void* x, int dtype_bf16, int64_t rows, int64_t cols,
                           int64_t ld, uint8_t* codes, uint8_t* scales, float* tensor_scale, int given,
                           void* ws, hipStream_t st)
{
    if (dtype_bf16)
        return launch_quantize_t<uint16_t>(fmt, cfg, (const uint16_t*)x, rows, cols, ld, codes, scales,
                                           tensor_scale, given, (uint32_t*)ws, st);
    return launch_quantize_t<float>(fmt, cfg, (const float*)x, rows, cols, ld, codes, scales, tensor_scale,
                                    given, (uint32_t*)ws, st);
}

}  // namespace razer
