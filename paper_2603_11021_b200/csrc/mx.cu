// Quantisation to microscaled 4-bit floating point, back to bf16, and products of such a matrix with up to 64 rows of bf16 activations
// (see include/llvq.h and mx.cuh).  None of it uses the tables of the context's code: the context gives the device and its error words.
#include <type_traits>

#include "kernels_common.cuh"
#include "mx_batch.h"
#include "mx_tensor.cuh"

namespace {

using namespace llvq;

constexpr int kMxThreads = 256;

// ---- quantisation ---------------------------------------------------------------------------------------------------------------
// Four lanes per block of 32, eight elements each.  scale = 2^(exponent of the largest magnitude - 2): the largest element lands in [4, 8), what is
// above 6 becomes 6.  A warp takes kMxUnroll pieces of eight blocks of one row, so that its loads overlap and its addresses are worked
// out once.  Bound by HBM: the input is read once and a quarter (bf16) or an eighth (binary32) of its bytes written.
constexpr int kMxUnroll = 4;

template <typename T> struct Wide;      // eight elements as they are loaded
template <> struct Wide<float> { float4 a, b; };
template <> struct Wide<__nv_bfloat16> { uint4 a; };
template <> struct Wide<__half> { uint4 a; };

__device__ __forceinline__ void widen(const Wide<float>& w, float v[8])
{
    v[0] = w.a.x; v[1] = w.a.y; v[2] = w.a.z; v[3] = w.a.w; v[4] = w.b.x; v[5] = w.b.y; v[6] = w.b.z; v[7] = w.b.w;
}
__device__ __forceinline__ void widen(const Wide<__nv_bfloat16>& w, float v[8])
{
    const uint32_t u[4] = {w.a.x, w.a.y, w.a.z, w.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
__device__ __forceinline__ void widen(const Wide<__half>& w, float v[8])
{
    const uint32_t u[4] = {w.a.x, w.a.y, w.a.z, w.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

// The larger of m and |v|; NaN if either is.
__device__ __forceinline__ float max_abs(float m, float v)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(v)));
    return r;
}

// wide: rows start on 16-byte boundaries
template <typename T>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_kernel(const T* __restrict__ x, int64_t rows, uint32_t cols, int64_t ld, uint32_t kb, uint32_t pitch, bool wide, uint8_t* __restrict__ codes,
                   uint8_t* __restrict__ scales)
{
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t lane = threadIdx.x & 31u, parts = (pitch + 8u * kMxUnroll - 1u) / (8u * kMxUnroll);
    const int64_t row = (int64_t)blockIdx.x * (kMxThreads / 32) + (threadIdx.x >> 5);
    if (row >= rows) return;
    const T* from = x + row * ld;
    uint8_t *codes_row = codes + row * (int64_t)(kb * kMxBlockBytes), *scales_row = scales + row * (int64_t)pitch;
    for (uint32_t part = blockIdx.y; part < parts; part += gridDim.y) {
        const uint32_t c0 = part * (256u * kMxUnroll) + lane * 8u, b0 = c0 >> 5;
        float v[kMxUnroll][8];
        if (wide && (part + 1u) * (256u * kMxUnroll) <= cols) {
            Wide<T> w[kMxUnroll];
#pragma unroll
            for (int u = 0; u < kMxUnroll; ++u) w[u] = *reinterpret_cast<const Wide<T>*>(from + c0 + u * 256);
#pragma unroll
            for (int u = 0; u < kMxUnroll; ++u) widen(w[u], v[u]);
        } else {
#pragma unroll
            for (int u = 0; u < kMxUnroll; ++u) {
                const uint32_t c = c0 + u * 256;
                if (wide && c + 8u <= cols) widen(*reinterpret_cast<const Wide<T>*>(from + c), v[u]);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[u][j] = c + j < cols ? to_float(from[c + j]) : 0.0f;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kMxUnroll; ++u) {
            float most = fabsf(v[u][0]);
#pragma unroll
            for (int j = 1; j < 8; ++j) most = max_abs(most, v[u][j]);
            most = max_abs(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max_abs(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const uint32_t exponent = __float_as_uint(most) >> 23;         // 255: an infinity or a NaN among them
            const uint32_t e = exponent == 255u ? 255u : max(exponent, 2u) - 2u;
            const float unit = __uint_as_float((254u - min(e, 252u)) << 23);      // 2^(127 - e) (255: not used); the product is exact unless it is
            float q[8];                                                         // far below the smallest element
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = v[u][j] * unit;
            const uint32_t w = e == 255u ? 0u : mx_pack8(q), b = b0 + u * 8u;
            if (b < kb) *reinterpret_cast<uint32_t*>(codes_row + (c0 + u * 256u) / 2u) = w;
            if ((lane & 3u) == 0u && b < pitch) scales_row[b] = b < kb ? (uint8_t)e : (uint8_t)0;
        }
    }
}

// ---- product with up to 64 rows of activations -------------------------------------------------------------------------------------
// Y[n][r] = sum_k X[n][k] W[r][k] on m16n8k16 tiles in binary16: 16 rows of W against 8 of X.  An e2m1 element is a binary16 number that one
// instruction per two elements makes; the scale of a block of 32 multiplies the block's sum in binary32.  Activations become binary16 as well:
// the 512 columns of a chunk of a row of X are multiplied with the power of two that brings their largest finite magnitude to [2^14, 2^15), which
// leaves every bf16 number exact down to 2^-31 of that magnitude and puts smaller ones off by at most 2^-39 of it, far below the rounding of
// the sums (binary32, 2^-24 of the same magnitude).  Where a weight of zero takes the largest out of the sum, those of other blocks are what counts: if a number
// that would not be exact is in a block of 32 whose largest is below 2^-12 of the chunk's, every block of the chunk has a factor of its own.
//
// A thread block streams W: kWarps warps multiply, 16 rows by 512 columns each per stage, RG x 16 rows by KG x 512 columns together, RG x KG = kWarps.
// The next warp copies their codes with TMA (rows of 128 bytes, swizzled, so that ldmatrix reads 16 bytes of eight rows without conflicts and hands each
// lane the word of codes whose elements are its own in the tile) and their scales.  X: one row is brought and converted by four more warps;
// several rows are converted once ahead by a kernel of their own and copied by one more warp, and W is read while that kernel still runs.  The stages in
// flight are what hides the latency of HBM, which bounds the kernel for up to about 16 rows of X (4.25 bits per weight, read once: 128256 x 4096,
// one row, 58 us in calls back to back, 74 % of the measured bandwidth); beyond, the products do.
constexpr int kChunk = 512;                              // columns of a warp's part of a stage
constexpr int kXWarps = 4;
constexpr uint32_t kXPitch = kChunk * 2 + 64;            // bytes: eight rows' 16-byte reads meet no bank twice; the exponent is behind the columns,
constexpr uint32_t kXOwn = kChunk * 2 + 16;              // and here, where it is kOwn, those of the 16 blocks, a byte each
constexpr int kOwn = 1000;
template <int kWarps, bool kPre> struct Stream {         // kWarps multiply; kPre: X comes as mx_stream_split_kernel left it
    static constexpr int kThreads = (kWarps + 1 + (kPre ? 1 : kXWarps)) * 32;
    static constexpr uint32_t kCodes = kWarps * 16 * (kChunk / 2), kScales = kWarps * 16 * 16;      // bytes per stage, whatever RG and KG
};
constexpr size_t kStreamSmem = 227 * 1024 - 1024;        // dynamic shared memory that a launch may use

struct MxStream {
    int64_t n_out, k_in;
    uint32_t kb, chunks, tiles;                          // blocks per row, chunks of 512 columns, tiles of 16 RG rows
    const __nv_bfloat16* x;
    int batch, x_align;                                  // rows of X; elements of X that one load may take: 8, 4, 2 or 1
    uint8_t* x_chunks;                                   // X as binary16 in global memory (several rows), see mx_stream_split_kernel
    int rg_log2, stages;
    uint32_t stage_bytes, part_at;                       // of a stage; where the sums of warps that share rows are (KG > 1)
    void* y;
    uint32_t* flags;
};

__device__ __forceinline__ void ldsm4(uint32_t r[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

__device__ __forceinline__ uint4 lds128(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ uint32_t lds32(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ int lds_s8(uint32_t addr)
{
    int v;
    asm volatile("ld.shared.s8 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ void sts128(uint32_t addr, uint4 v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// The eight elements of a word of codes as binary16 pairs.
__device__ __forceinline__ void mx_expand_f16(uint32_t w, uint32_t h[4])
{
    asm("{\n .reg .b8 b0, b1, b2, b3;\n mov.b32 {b0, b1, b2, b3}, %4;\n"
        " cvt.rn.f16x2.e2m1x2 %0, b0;\n cvt.rn.f16x2.e2m1x2 %1, b1;\n cvt.rn.f16x2.e2m1x2 %2, b2;\n cvt.rn.f16x2.e2m1x2 %3, b3;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}

__device__ __forceinline__ void mma_f16(float d[4], const uint32_t a[4], uint32_t b0, uint32_t b1, const float c[4])
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

// Eight elements of row n of X from column k on; zero past the end.
__device__ __forceinline__ uint4 load_x8(const MxStream& a, int n, int64_t k)
{
    const __nv_bfloat16* p = a.x + (int64_t)n * a.k_in + k;
    const bool whole = k + 8 <= a.k_in;
    if (whole && a.x_align == 8) return __ldg(reinterpret_cast<const uint4*>(p));
    if (whole && a.x_align == 4) {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(p)), v = __ldg(reinterpret_cast<const uint2*>(p) + 1);
        return make_uint4(u.x, u.y, v.x, v.y);
    }
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (whole && a.x_align == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __ldg(reinterpret_cast<const uint32_t*>(p) + j);
    } else {
        const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (k + j < a.k_in) w[j >> 1] |= (uint32_t)__ldg(q + j) << (16 * (j & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Largest and smallest magnitudes of pairs of bf16, per half of a word.  most: 0x80 more than the largest finite one (an infinity or a NaN becomes negative);
// least: one less than the smallest that is not zero (zero becomes the largest of all).
constexpr uint32_t kMostNone = 0x00800080u, kLeastNone = 0xffffffffu;
__device__ __forceinline__ void most_and_least(uint32_t& most, uint32_t& least, const uint4& v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t size = w[i] & 0x7fff7fffu;
        most = __viaddmax_s16x2(size, 0x00800080u, most);
        least = __viaddmin_u16x2(size, 0xffffffffu, least);
    }
}
__device__ __forceinline__ uint32_t most_of(uint32_t most) { return max(most & 0xffffu, most >> 16) - 0x80u; }
__device__ __forceinline__ uint32_t least_of(uint32_t least) { return min(least & 0xffffu, least >> 16) + 1u; }

__device__ __forceinline__ uint32_t to_f16(uint32_t pair, float factor)
{
    return f16_pair(__uint_as_float(pair << 16) * factor, __uint_as_float(pair & 0xffff0000u) * factor);
}

// The exponent of the factor for a largest finite magnitude m (as bf16 bits): at most 125 (which leaves all numbers below 2^-110 exact), and 0 where m is zero.
__device__ __forceinline__ int factor_of(uint32_t m) { return m == 0u ? 0 : min(14 - ((int)(m >> 7) - 127), 125); }

__device__ __forceinline__ void half_to_f16(uint4& v, int f)
{
    const float factor = __uint_as_float((uint32_t)(f + 127) << 23);
    v = make_uint4(to_f16(v.x, factor), to_f16(v.y, factor), to_f16(v.z, factor), to_f16(v.w, factor));
}

// The 512 columns of a chunk of a row of X as they were loaded (columns 8 lane .. and 256 + 8 lane ..) to binary16, in place; the exponent of the factor,
// or kOwn where blocks have their own: then own[h] is that of the block of v[h].
__device__ __forceinline__ int chunk_to_f16(uint4 v[2], int own[2])
{
    uint32_t most[2] = {kMostNone, kMostNone}, least[2] = {kLeastNone, kLeastNone};
    most_and_least(most[0], least[0], v[0]);
    most_and_least(most[1], least[1], v[1]);
    const uint32_t m = __reduce_max_sync(0xffffffffu, most_of(__vmaxu2(most[0], most[1]))), exponent = m >> 7;
    auto inexact = [&](uint32_t smallest) { return exponent > max(smallest >> 7, 1u) + 31u; };      // its last bit is below 2^-24, binary16's smallest step
    if (__any_sync(0xffffffffu, inexact(least_of(__vminu2(least[0], least[1]))))) {      // seldom so
        bool differ = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t big = most_of(most[h]), small = least_of(least[h]);
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) { big = max(big, __shfl_xor_sync(0xffffffffu, big, o)); small = min(small, __shfl_xor_sync(0xffffffffu, small, o)); }
            differ |= inexact(small) && (big >> 7) + 12u < exponent;
            own[h] = factor_of(big);
        }
        if (__any_sync(0xffffffffu, differ)) {
            half_to_f16(v[0], own[0]);
            half_to_f16(v[1], own[1]);
            return kOwn;
        }
    }
    const int f = factor_of(m);
    half_to_f16(v[0], f);
    half_to_f16(v[1], f);
    return f;
}

// Several rows of X, once for all thread blocks: [chunk][row][kXPitch bytes], a warp per row and chunk.
__global__ void __launch_bounds__(256)
mx_stream_split_kernel(MxStream a)
{
    pdl_wait();
    pdl_launch_dependents();                             // behind the wait: what the next kernel reads ahead of its own was written before this one
    const int lane = threadIdx.x & 31;
    const uint32_t unit = blockIdx.x * 8u + (threadIdx.x >> 5), chunk = unit / (uint32_t)a.batch;
    if (chunk >= a.chunks) return;
    const int n = (int)(unit - chunk * (uint32_t)a.batch);
    const int64_t k = (int64_t)chunk * kChunk + lane * 8;
    uint4 v[2] = {load_x8(a, n, k), load_x8(a, n, k + 256)};
    int own[2];
    const int f = chunk_to_f16(v, own);
    uint8_t* to = a.x_chunks + (uint64_t)unit * kXPitch;
    *reinterpret_cast<uint4*>(to + lane * 16) = v[0];
    *reinterpret_cast<uint4*>(to + 512 + lane * 16) = v[1];
    if (lane == 0) *reinterpret_cast<int*>(to + 1024) = f;
    if (f == kOwn && (lane & 3) == 0) {
        reinterpret_cast<int8_t*>(to)[kXOwn + (lane >> 2)] = (int8_t)own[0];
        reinterpret_cast<int8_t*>(to)[kXOwn + 8 + (lane >> 2)] = (int8_t)own[1];
    }
}

// d * 2^h in two steps, for h that binary32 may not hold; NaN for the scale byte 255
__device__ __forceinline__ float scale_far(float d, uint32_t e, int f)
{
    const int h = (int)e - 127 - f, h1 = h / 2, h2 = h - h1;               // -127 - 125 <= h <= 127 + 113: both halves are normal exponents
    const float s1 = e == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(h1 + 127) << 23);
    return d * s1 * __uint_as_float((uint32_t)(h2 + 127) << 23);
}

template <int kWarps, int kTiles, bool kF32, bool kPre>
__global__ void __launch_bounds__(Stream<kWarps, kPre>::kThreads, 1)
mx_stream_kernel(const __grid_constant__ CUtensorMap codes, const __grid_constant__ CUtensorMap scales, MxStream a)
{
    constexpr uint32_t kCodes = Stream<kWarps, kPre>::kCodes, kScales = Stream<kWarps, kPre>::kScales;
    extern __shared__ uint8_t st_smem[];
    __shared__ uint64_t full[8], empty[8];
    const uint32_t base = (smem_u32(st_smem) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rg_n = 1 << a.rg_log2, kg_n = kWarps >> a.rg_log2;
    const uint32_t rows = 16u << a.rg_log2, steps = (a.chunks + kg_n - 1) / kg_n;      // steps: stages per tile
    constexpr uint32_t x_at = kCodes + kScales;          // inside a stage
    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) { mbar_init(full + s, kPre ? 2 : 1 + kXWarps); mbar_init(empty + s, kWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (!kPre) pdl_wait();                               // else the warp of X waits, and nothing is written before X has come
    bool ok = true;
    uint32_t s = 0, phase = 0;                           // stage and its phase
    auto next = [&] { if (++s == (uint32_t)a.stages) { s = 0; phase ^= 1u; } };
    if (warp == kWarps) {
        if (lane == 0) {
            uint32_t it = 0;
            for (uint32_t tile = blockIdx.x; tile < a.tiles && ok; tile += gridDim.x) {
                for (uint32_t step = 0; step < steps; ++step, ++it) {
                    if (it >= (uint32_t)a.stages) ok = mbar_wait(empty + s, phase ^ 1u);
                    if (!ok) break;
                    const uint32_t at = base + s * a.stage_bytes;
                    mbar_expect(full + s, kCodes + kScales);
                    for (int g = 0; g < kg_n; ++g) {     // what lies past the end of a row reads as zero
                        const int chunk = (int)(step * kg_n + g);
                        tma_load_2d(at + g * rows * (kChunk / 2), &codes, chunk * (kChunk / 2), (int)(tile * rows), full + s);
                        tma_load_2d(at + g * rows * (kChunk / 2) + rows * 128u, &codes, chunk * (kChunk / 2) + 128, (int)(tile * rows), full + s);
                        tma_load_2d(at + kCodes + g * rows * 16u, &scales, chunk * 16, (int)(tile * rows), full + s);
                    }
                    next();
                }
            }
        }
    } else if (kPre && warp > kWarps) {
        if (lane == 0) {
            pdl_wait();
            uint32_t it = 0;
            for (uint32_t tile = blockIdx.x; tile < a.tiles && ok; tile += gridDim.x) {
                for (uint32_t step = 0; step < steps; ++step, ++it) {
                    if (it >= (uint32_t)a.stages) ok = mbar_wait(empty + s, phase ^ 1u);
                    if (!ok) break;
                    const uint32_t chunk = step * kg_n, count = min((uint32_t)kg_n, a.chunks - chunk), bytes = count * a.batch * kXPitch;
                    mbar_expect(full + s, bytes);
                    bulk_load(base + s * a.stage_bytes + x_at, a.x_chunks + (uint64_t)chunk * a.batch * kXPitch, bytes, full + s);
                    next();
                }
            }
        }
    } else if (warp > kWarps) {
        const int me = warp - kWarps - 1, items = kg_n * a.batch;
        uint32_t it = 0;
        for (uint32_t tile = blockIdx.x; tile < a.tiles && ok; tile += gridDim.x) {
            for (uint32_t step = 0; step < steps; ++step, ++it) {
                if (it >= (uint32_t)a.stages) ok = __all_sync(0xffffffffu, mbar_wait(empty + s, phase ^ 1u));
                if (!ok) break;
                const uint32_t at = base + s * a.stage_bytes;
                constexpr int kAhead = 4;
                for (int i0 = me; i0 < items; i0 += kXWarps * kAhead) {
                    uint4 v[kAhead][2];
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const int i = i0 + u * kXWarps, g = i / a.batch, n = i - g * a.batch;
                        const int64_t k = (int64_t)(step * kg_n + g) * kChunk + lane * 8;
                        if (i < items) { v[u][0] = load_x8(a, n, k); v[u][1] = load_x8(a, n, k + 256); }
                    }
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const int i = i0 + u * kXWarps;
                        if (i >= items) break;           // the same for the whole warp
                        int own[2];
                        const int f = chunk_to_f16(v[u], own);
                        const uint32_t to = at + x_at + i * kXPitch;
                        sts128(to + lane * 16u, v[u][0]);
                        sts128(to + 512u + lane * 16u, v[u][1]);
                        if (lane == 0) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + 1024u), "r"(f) : "memory");
                        if (f == kOwn && (lane & 3) == 0)
                            asm volatile("st.shared.s8 [%0], %1;\n st.shared.s8 [%0 + 8], %2;" ::"r"(to + kXOwn + (lane >> 2)), "r"(own[0]), "r"(own[1]) : "memory");
                    }
                }
                __syncwarp();
                if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(full + s)) : "memory");
                next();
            }
        }
    } else {
        const int rg = warp & (rg_n - 1), kg = warp >> a.rg_log2, g = lane >> 2, t = lane & 3;
        // where ldmatrix finds this lane's row: rows 0-7 of a block, 8-15 of it, then the same of the next block
        const uint32_t mrow = (uint32_t)rg * 16u + (lane & 7) + (lane & 8), mblock = (uint32_t)lane >> 4;
        const uint32_t row_at = (uint32_t)kg * rows * (kChunk / 2) + mrow * 128u, swizzle = mrow & 7u;
        const uint32_t scale_at = kCodes + ((uint32_t)kg * rows + rg * 16u + g) * 16u;
        const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t tile = blockIdx.x; tile < a.tiles && ok; tile += gridDim.x) {
            float acc[kTiles][4] = {};
            for (uint32_t step = 0; step < steps; ++step) {
                ok = __all_sync(0xffffffffu, mbar_wait_copies(full + s, phase));
                if (!ok) break;
                const uint32_t at = base + s * a.stage_bytes, first = (step * kg_n + kg) * 16u;       // first block
                if (first < a.kb) {
                    const uint4 e0 = lds128(at + scale_at), e1 = lds128(at + scale_at + 128u);
                    uint32_t ea[4] = {e0.x, e0.y, e0.z, e0.w}, eb[4] = {e1.x, e1.y, e1.z, e1.w};
                    if (a.kb - first < 16u) {            // bytes past the row's last block are not scales: 2^0 instead
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t left = a.kb - first, b = 4u * j, valid = left <= b ? 0u : left - b >= 4u ? 0xffffffffu : (1u << (8u * (left - b))) - 1u;
                            ea[j] = (ea[j] & valid) | (0x7f7f7f7fu & ~valid);
                            eb[j] = (eb[j] & valid) | (0x7f7f7f7fu & ~valid);
                        }
                    }
                    // Scales from 2^-63 to 2^64 (bits 7 and 6 differ) and activations whose factor is not far from one: sums times scales stay well inside
                    // binary32, and the factor is taken off once per chunk.  Else both exponents are added block by block, at half the speed or less: so for a
                    // warp's 16 rows and 512 columns with a block of zeros (scale 0) among them (28672 x 8192 with a tenth of the blocks zero: one row of X
                    // 56 us instead of 33, 16 rows 86 instead of 41), and where blocks of X have factors of their own (57 and 67).
                    uint32_t usual = 0x80808080u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) usual &= (ea[j] ^ (ea[j] << 1)) & (eb[j] ^ (eb[j] << 1));
                    int f[kTiles][2];
                    bool near = usual == 0x80808080u;
#pragma unroll
                    for (int n = 0; n < kTiles; ++n)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            f[n][c] = (int)lds32(at + x_at + (kg * a.batch + min(n * 8 + 2 * t + c, a.batch - 1)) * kXPitch + 1024u);
                            near &= f[n][c] >= -30 && f[n][c] <= 50;
                        }
                    const uint32_t codes_at = (at + row_at) | ((mblock ^ swizzle) << 4), x_row = at + x_at + kg * a.batch * kXPitch + t * 16u;
                    uint32_t xs[kTiles];                 // this lane's row of X for each tile: the last one again where there are no more
#pragma unroll
                    for (int n = 0; n < kTiles; ++n) xs[n] = x_row + min(n * 8 + g, a.batch - 1) * kXPitch;
                    float part[kTiles][4] = {};
                    auto chunk = [&](auto fast) {
#pragma unroll (kTiles <= 2 ? 2 : 1)
                        for (int box = 0; box < 2; ++box) {
#pragma unroll
                            for (int b = 0; b < 8; b += 2) {
                                uint32_t w[4], h[4][4];
                                ldsm4(w, (codes_at + box * rows * 128u) ^ (b * 16u));
#pragma unroll
                                for (int i = 0; i < 4; ++i) mx_expand_f16(w[i], h[i]);
                                const uint32_t wa = box == 0 ? ea[b >> 2] : ea[2 + (b >> 2)], wb = box == 0 ? eb[b >> 2] : eb[2 + (b >> 2)];
#pragma unroll
                                for (int q = 0; q < 2; ++q) {
                                    constexpr uint32_t kExponent = 0x7f800000u;
                                    const int j = (b + q) & 3;
                                    const uint32_t sa = (j < 3 ? wa << (23 - 8 * j) : wa >> 1) & kExponent, sb = (j < 3 ? wb << (23 - 8 * j) : wb >> 1) & kExponent;
                                    const uint32_t lo[4] = {h[2 * q][0], h[2 * q + 1][0], h[2 * q][1], h[2 * q + 1][1]};
                                    const uint32_t hi[4] = {h[2 * q][2], h[2 * q + 1][2], h[2 * q][3], h[2 * q + 1][3]};
#pragma unroll
                                    for (int n = 0; n < kTiles; ++n) {
                                        const uint4 x = lds128(xs[n] + box * 512u + (b + q) * 64u);
                                        float d[4];
                                        mma_f16(d, lo, x.x, x.y, zero);
                                        mma_f16(d, hi, x.z, x.w, d);
                                        if constexpr (decltype(fast)::value) {
                                            part[n][0] += d[0] * __uint_as_float(sa); part[n][1] += d[1] * __uint_as_float(sa);
                                            part[n][2] += d[2] * __uint_as_float(sb); part[n][3] += d[3] * __uint_as_float(sb);
                                        } else {
                                            int g[2];
#pragma unroll
                                            for (int c = 0; c < 2; ++c)
                                                g[c] = f[n][c] != kOwn ? f[n][c] : lds_s8(at + x_at + (kg * a.batch + min(n * 8 + 2 * t + c, a.batch - 1)) * kXPitch + kXOwn + box * 8 + b + q);
                                            part[n][0] += scale_far(d[0], sa >> 23, g[0]); part[n][1] += scale_far(d[1], sa >> 23, g[1]);
                                            part[n][2] += scale_far(d[2], sb >> 23, g[0]); part[n][3] += scale_far(d[3], sb >> 23, g[1]);
                                        }
                                    }
                                }
                            }
                        }
                    };
                    if (__all_sync(0xffffffffu, near)) {
                        chunk(std::true_type{});
#pragma unroll
                        for (int n = 0; n < kTiles; ++n)
#pragma unroll
                            for (int j = 0; j < 4; ++j) acc[n][j] += part[n][j] * __uint_as_float((uint32_t)(127 - f[n][j & 1]) << 23);
                    } else {
                        chunk(std::false_type{});
#pragma unroll
                        for (int n = 0; n < kTiles; ++n)
#pragma unroll
                            for (int j = 0; j < 4; ++j) acc[n][j] += part[n][j];
                    }
                }
                __syncwarp();
                if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(empty + s)) : "memory");
                next();
            }
            if (kg_n == 1 && !ok) break;
            const int64_t row0 = (int64_t)tile * rows;
            auto put = [&](int n, int64_t row, float v) {
                if (n >= a.batch || row >= a.n_out) return;
                if (kF32) static_cast<float*>(a.y)[(int64_t)n * a.n_out + row] = v;
                else static_cast<__nv_bfloat16*>(a.y)[(int64_t)n * a.n_out + row] = __float2bfloat16_rn(v);
            };
            if (kg_n == 1) {
#pragma unroll
                for (int n = 0; n < kTiles; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) put(n * 8 + 2 * t + (j & 1), row0 + rg * 16 + g + 8 * (j >> 1), acc[n][j]);
            } else {
                float* part = reinterpret_cast<float*>(st_smem + (base - smem_u32(st_smem)) + a.part_at);       // [kg][column][row]
#pragma unroll
                for (int n = 0; n < kTiles; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) part[(kg * kTiles * 8 + n * 8 + 2 * t + (j & 1)) * (int)rows + rg * 16 + g + 8 * (j >> 1)] = acc[n][j];
                ok = all_well(ok, kWarps * 32);
                if (!ok) break;
                for (int i = threadIdx.x; i < a.batch * (int)rows; i += kWarps * 32) {
                    const int n = i / (int)rows, r = i & (int)(rows - 1);
                    float v = 0.0f;
                    for (int k = 0; k < kg_n; ++k) v += part[(k * kTiles * 8 + n) * (int)rows + r];
                    put(n, row0 + r, v);
                }
                asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");      // the sums are read before the next tile's are written
            }
        }
    }
    if (!ok) atomicOr(a.flags, (uint32_t)LLVQ_FLAG_WAIT_TIMEOUT);
}

// Sizes whose byte counts leave 63 bits, or dimensions that the kernels' indices do not hold.
bool mx_too_large(int64_t rows, int64_t cols) { return rows > 0x7fffffffll || cols > (1ll << 30); }

// none: the matrix has no columns, and its arrays may be null
int mx_check(const llvq_ctx* ctx, bool none, const uint8_t* d_codes, const uint8_t* d_scales)
{
    if (!ctx || ctx->device < 0 || (!none && (!d_codes || !d_scales))) return LLVQ_EINVAL;
    return aligned(d_codes, 16) && aligned(d_scales, 16) ? LLVQ_OK : LLVQ_EALIGN;
}

template <typename T>
cudaError_t launch_quantize(const void* x, int64_t rows, int64_t cols, int64_t ld, uint8_t* codes, uint8_t* scales, cudaStream_t st)
{
    const bool wide = aligned(x, 16) && ld % (16 / (int64_t)sizeof(T)) == 0;
    const uint32_t pitch = (uint32_t)mx_scale_pitch(cols), parts = (pitch + 8u * kMxUnroll - 1u) / (8u * kMxUnroll);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((rows + kMxThreads / 32 - 1) / (kMxThreads / 32)), std::min(parts, 65535u)); cfg.blockDim = dim3(kMxThreads); cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, mx_quantize_kernel<T>, static_cast<const T*>(x), rows, (uint32_t)cols, ld, (uint32_t)mx_blocks(cols), pitch, wide, codes, scales);
}

template <int kWarps, int kTiles, bool kF32, bool kPre>
int launch_stream(const llvq_ctx* ctx, const CUtensorMap& codes, const CUtensorMap& scales, const MxStream& a, unsigned grid, size_t smem, cudaStream_t st)
{
    if (!set_smem<mx_stream_kernel<kWarps, kTiles, kF32, kPre>>(ctx, smem)) return LLVQ_ECUDA;
    const cudaError_t r = launch_pdl(mx_stream_kernel<kWarps, kTiles, kF32, kPre>, grid, Stream<kWarps, kPre>::kThreads, smem, st, codes, scales, a);
    return r == cudaSuccess ? launch_status() : LLVQ_ECUDA;
}

// Whether weights go through registers (mx_stream_kernel) or to the tensor cores as they are (mx_batch_product).  us: 4096 x 4096, 17 / 24 / 32 rows of X
// 11.0 / 11.3 / 14.1 and 14.5 / 15.5 / 16.0; 11008 x 4096 17.3 / 17.4 / 22.6 and 16.2 / 16.8 / 17.7; 28672 x 8192, 17 rows 63 and 38.
bool takes_stream(int64_t n_out, int64_t k_in, int batch) { return batch <= 16 || (batch <= 32 && n_out <= (1ll << 25) / k_in); }

uint64_t stream_x_bytes(int64_t k_in, int batch) { return (uint64_t)(k_in + kChunk - 1) / kChunk * (uint64_t)batch * kXPitch; }

// batch up to 32; work: stream_x_bytes() of device memory for more than one row
int mx_stream_product(const llvq_ctx* ctx, const uint8_t* d_codes, const uint8_t* d_scales, int64_t n_out, int64_t k_in, const uint16_t* d_x, int batch,
                      void* d_y, int y_dtype, uint8_t* work, cudaStream_t st)
{
    MxStream a{};
    a.n_out = n_out; a.k_in = k_in; a.kb = (uint32_t)mx_blocks(k_in); a.chunks = (a.kb + 15) / 16;
    a.x = reinterpret_cast<const __nv_bfloat16*>(d_x); a.batch = batch; a.y = d_y; a.flags = ctx->dev.flags; a.x_chunks = work;
    a.x_align = 8;
    while (a.x_align > 1 && (!aligned(d_x, 2 * (size_t)a.x_align) || (batch > 1 && k_in % a.x_align != 0))) a.x_align /= 2;
    const int tiles = (batch + 7) / 8;
    // Warps and rows of a tile by what they should take, in ns: the rounds over the SMs, each with the tile's share of W (17 bytes per block) and, half as
    // dear, of X at 35 bytes per ns, and an end; with two stages at least and no more warps along a row than it has chunks.  16 warps take
    // 0.7 us longer to start; eight are slower at the products (28672 x 8192, us with 16 / 8: one row 32.0 / 39.2, eight 31.0 / 32.2, 16 rows 40.8 / 47.4)
    // and make room for stages (8192 x 8192, 16 rows: 22.9 / 16.0; 2048 x 4096, one row 4.2 / 3.5, 16 rows 13.0 / 6.2).
    const int slower = batch == 1 ? 123 : batch <= 8 ? 103 : 116;      // per cent
    uint64_t best = ~0ull;
    size_t smem = 0;
    int warps = 0;
    for (int w = tiles <= 2 ? 16 : 8; w >= 8; w /= 2) {
        for (int l = w == 16 ? 4 : 3; l >= 0; --l) {
            const int kg = w >> l;
            if (kg > 1 && kg / 2 >= (int)a.chunks) break;
            const uint32_t stage = ((uint32_t)w * (16u * (kChunk / 2) + 16u * 16u) + (uint32_t)(kg * batch) * kXPitch + 1023u) & ~1023u;
            const uint32_t part = kg > 1 ? (uint32_t)kg * tiles * 8u * (16u << l) * 4u : 0u;
            const int stages = (int)std::min<size_t>(6, (kStreamSmem - 1024 - part) / stage);
            if (stages < 2) continue;
            const uint64_t count = ((uint64_t)n_out + (16u << l) - 1) / (16u << l), rounds = (count + ctx->sm_count - 1) / ctx->sm_count;
            const uint64_t bytes = (uint64_t)a.kb * ((16u << l) * 17u + (uint64_t)batch * 34u);
            const uint64_t cost = rounds * (bytes / 35u + 100u) * (w == 8 ? slower : 100) / 100u + (w == 16 ? 700u : 0u);
            if (cost >= best) continue;
            best = cost;
            warps = w;
            a.rg_log2 = l; a.tiles = (uint32_t)count; a.stage_bytes = stage; a.stages = stages; a.part_at = (uint32_t)stages * stage;
            smem = 1024 + a.part_at + part;
        }
    }
    if (best == ~0ull) return LLVQ_EUNSUPPORTED;
    CUtensorMap codes, scales;
    if (!make_byte_map(ctx->device, d_codes, mx_code_pitch(k_in), n_out, 128, 16 << a.rg_log2, true, &codes) ||
        !make_byte_map(ctx->device, d_scales, mx_scale_pitch(k_in), n_out, 16, 16 << a.rg_log2, false, &scales)) return LLVQ_ECUDA;
    const unsigned grid = std::min<unsigned>(a.tiles, (unsigned)ctx->sm_count);
    if (batch > 1) {
        const uint64_t split = ((uint64_t)a.chunks * batch + 7) / 8;
        if (split > 0x7fffffff) return LLVQ_EUNSUPPORTED;
        if (launch_pdl(mx_stream_split_kernel, (unsigned)split, 256, 0, st, a) != cudaSuccess) return LLVQ_ECUDA;
    }
    auto launch = [&](auto w) {
        constexpr int kWarps = decltype(w)::value;
        return batch == 1 ? y_dtype == LLVQ_F32 ? launch_stream<kWarps, 1, true, false>(ctx, codes, scales, a, grid, smem, st)
                                                : launch_stream<kWarps, 1, false, false>(ctx, codes, scales, a, grid, smem, st)
               : tiles == 1 ? launch_stream<kWarps, 1, false, true>(ctx, codes, scales, a, grid, smem, st)
                            : launch_stream<kWarps, 2, false, true>(ctx, codes, scales, a, grid, smem, st);
    };
    if (tiles == 3) return launch_stream<8, 3, false, true>(ctx, codes, scales, a, grid, smem, st);
    if (tiles == 4) return launch_stream<8, 4, false, true>(ctx, codes, scales, a, grid, smem, st);
    return warps == 16 ? launch(std::integral_constant<int, 16>{}) : launch(std::integral_constant<int, 8>{});
}

}  // namespace

extern "C" {

int64_t llvq_mx_code_pitch(int64_t cols) { return cols < 0 ? 0 : mx_code_pitch(cols); }
int64_t llvq_mx_scale_pitch(int64_t cols) { return cols < 0 ? 0 : mx_scale_pitch(cols); }
int llvq_device(const llvq_ctx* ctx) { return ctx ? ctx->device : -1; }

int llvq_mx_quantize(const llvq_ctx* ctx, const void* d_x, int x_dtype, int64_t rows, int64_t cols, int64_t ld, uint8_t* d_codes, uint8_t* d_scales,
                     void* stream)
{
    if (ctx && ctx->device >= 0 && (rows == 0 || cols == 0)) return LLVQ_OK;      // nothing to do: pointers may be null
    if (int e = mx_check(ctx, false, d_codes, d_scales)) return e;
    if (!d_x || rows < 0 || cols < 0 || ld < cols || x_dtype < LLVQ_F32 || x_dtype > LLVQ_F16) return LLVQ_EINVAL;
    if (!aligned(d_x, x_dtype == LLVQ_F32 ? 4 : 2)) return LLVQ_EALIGN;
    if (mx_too_large(rows, cols)) return LLVQ_EUNSUPPORTED;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return LLVQ_ECUDA;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t r = x_dtype == LLVQ_F32    ? launch_quantize<float>(d_x, rows, cols, ld, d_codes, d_scales, st)
                          : x_dtype == LLVQ_BF16 ? launch_quantize<__nv_bfloat16>(d_x, rows, cols, ld, d_codes, d_scales, st)
                                                 : launch_quantize<__half>(d_x, rows, cols, ld, d_codes, d_scales, st);
    return r == cudaSuccess ? launch_status() : LLVQ_ECUDA;
}

int llvq_mx_gemv(const llvq_ctx* ctx, const uint8_t* d_codes, const uint8_t* d_scales, int64_t n_out, int64_t k_in, const uint16_t* d_x_bf16, void* d_y,
                 int y_dtype, void* stream)
{
    if (ctx && ctx->device >= 0 && n_out == 0) return LLVQ_OK;
    if (int e = mx_check(ctx, k_in == 0, d_codes, d_scales)) return e;
    if ((!d_x_bf16 && k_in != 0) || !d_y || n_out < 0 || k_in < 0 || (y_dtype != LLVQ_F32 && y_dtype != LLVQ_BF16)) return LLVQ_EINVAL;
    if (!aligned(d_x_bf16, 2) || !aligned(d_y, y_dtype == LLVQ_F32 ? 4 : 2)) return LLVQ_EALIGN;
    if (n_out > (1ll << 30) || k_in > (1ll << 30)) return LLVQ_EUNSUPPORTED;      // TMA coordinates
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return LLVQ_ECUDA;
    if (k_in == 0) return cudaMemsetAsync(d_y, 0, (size_t)n_out * (y_dtype == LLVQ_F32 ? 4 : 2), (cudaStream_t)stream) == cudaSuccess ? LLVQ_OK : LLVQ_ECUDA;
    return mx_stream_product(ctx, d_codes, d_scales, n_out, k_in, d_x_bf16, 1, d_y, y_dtype, nullptr, (cudaStream_t)stream);
}

size_t llvq_mx_small_batch_bytes(const llvq_ctx* ctx, int64_t n_out, int64_t k_in, int batch)
{
    if (!ctx || ctx->device < 0 || n_out <= 0 || k_in <= 0 || batch <= 0 || batch > 64 || n_out > (1ll << 30) || k_in > (1ll << 30)) return 0;
    return batch == 1 ? 0 : takes_stream(n_out, k_in, batch) ? (size_t)stream_x_bytes(k_in, batch) : mx_batch_bytes(ctx, n_out, k_in, batch);
}

int llvq_mx_gemm_small_batch(const llvq_ctx* ctx, const uint8_t* d_codes, const uint8_t* d_scales, int64_t n_out, int64_t k_in, const uint16_t* d_x_bf16,
                             int batch, uint16_t* d_y_bf16, void* d_work, void* stream)
{
    if (ctx && ctx->device >= 0 && (n_out == 0 || batch == 0)) return LLVQ_OK;
    if (int e = mx_check(ctx, k_in == 0, d_codes, d_scales)) return e;
    if ((!d_x_bf16 && k_in != 0) || !d_y_bf16 || n_out < 0 || k_in < 0 || batch < 0) return LLVQ_EINVAL;
    if (!aligned(d_x_bf16, 2) || !aligned(d_y_bf16, 2) || !aligned(d_work, 256)) return LLVQ_EALIGN;
    if (batch > 64 || n_out > (1ll << 30) || k_in > (1ll << 30)) return LLVQ_EUNSUPPORTED;
    if (batch > 1 && k_in > 0 && !d_work) return LLVQ_EINVAL;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return LLVQ_ECUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if (k_in == 0) return cudaMemsetAsync(d_y_bf16, 0, (size_t)n_out * batch * 2, st) == cudaSuccess ? LLVQ_OK : LLVQ_ECUDA;
    uint8_t* work = static_cast<uint8_t*>(d_work);
    return takes_stream(n_out, k_in, batch) ? mx_stream_product(ctx, d_codes, d_scales, n_out, k_in, d_x_bf16, batch, d_y_bf16, LLVQ_BF16, work, st)
                                 : mx_batch_product(ctx, d_codes, d_scales, n_out, k_in, d_x_bf16, batch, d_y_bf16, work, st);
}

}  // extern "C"
