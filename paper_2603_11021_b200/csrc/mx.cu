// Quantisation to microscaled 4-bit floating point, back to bf16, and products of such a matrix with up to 64 rows of bf16 activations
// (see include/llvq.h and mx.cuh).  None of it uses the tables of the context's code: the context gives the device and its error words.
#include "kernels_common.cuh"
#include "mx.cuh"

namespace {

using namespace llvq;

constexpr int kMxThreads = 256;

// ---- quantisation ---------------------------------------------------------------------------------------------------------------
// Four lanes per block of 32, eight elements each; the largest exponent of the block is the exponent of its largest magnitude, found
// on the bit patterns.  scale = 2^(exponent - 2): the largest element lands in [4, 8), what is above 6 becomes 6.  A warp takes eight
// blocks of a row at a time (their eight scale bytes are one store) and kMxUnroll such pieces together, so that its loads overlap.
// Bound by HBM: the input is read once and a quarter (bf16) of its bytes written.
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

// wide: rows start on 16-byte boundaries
template <typename T>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_kernel(const T* __restrict__ x, int64_t rows, int64_t cols, int64_t ld, uint32_t pieces, bool wide, uint8_t* __restrict__ codes,
                   uint8_t* __restrict__ scales)
{
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t lane = threadIdx.x & 31u;
    const int64_t kb = mx_blocks(cols), total = rows * (int64_t)pieces;
    const int64_t first = ((int64_t)blockIdx.x * (kMxThreads / 32) + (threadIdx.x >> 5)) * kMxUnroll;
    int64_t row = first / pieces;
    uint32_t piece = (uint32_t)(first - row * pieces);
    float v[kMxUnroll][8];
    int64_t at_row[kMxUnroll];
    uint32_t at_piece[kMxUnroll];
#pragma unroll
    for (int u = 0; u < kMxUnroll; ++u) {
        at_row[u] = first + u < total ? row : -1;
        at_piece[u] = piece;
        if (++piece == pieces) { piece = 0; ++row; }
        const int64_t c = (int64_t)at_piece[u] * 256 + lane * 8;
        const T* p = x + at_row[u] * ld + c;
        if (at_row[u] >= 0 && wide && c + 8 <= cols) {
            widen(*reinterpret_cast<const Wide<T>*>(p), v[u]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[u][j] = at_row[u] >= 0 && c + j < cols ? to_float(p[j]) : 0.0f;
        }
    }
#pragma unroll
    for (int u = 0; u < kMxUnroll; ++u) {
        if (at_row[u] < 0) break;                       // the same for the whole warp
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(v[u][j]) & 0x7fffffffu);
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int exponent = (int)(most >> 23);         // 255: an infinity or a NaN among them
        const uint32_t e = exponent == 255 ? 255u : (uint32_t)max(exponent - 2, 0);
        const float unit = e == 255u ? 0.0f : __uint_as_float((254u - e) << 23);       // 2^(127 - e): e is at most 252, a multiplication that is exact
        uint32_t w = 0;                                                              // unless the product is far below the smallest element
        if (e != 255u) {
            float q[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = v[u][j] * unit;
            w = mx_pack8(q);
        }
        const int64_t block = (int64_t)at_piece[u] * 8 + (lane >> 2);
        if (block < kb) *reinterpret_cast<uint32_t*>(codes + at_row[u] * (kb * kMxBlockBytes) + block * kMxBlockBytes + (lane & 3u) * 4) = w;
        // the eight scale bytes, those past the row's end zero, by the first lane
        uint32_t byte = block < kb ? e : 0u;
        byte |= __shfl_down_sync(0xffffffffu, byte, 4) << 8;
        byte |= __shfl_down_sync(0xffffffffu, byte, 8) << 16;
        const uint32_t above = __shfl_down_sync(0xffffffffu, byte, 16);
        if (lane == 0) *reinterpret_cast<uint2*>(scales + at_row[u] * (int64_t)pieces * 8 + at_piece[u] * 8) = make_uint2(byte, above);
    }
}

// ---- product with up to 64 rows of activations -------------------------------------------------------------------------------------
// y[n][r] = sum_k x[n][k] w[r][k] on m16n8k16 tiles: 16 rows of W against 8 of X.  Sums over k may run in any order, so a lane keeps
// the whole block that its 16-byte load brought: in step s of the eight that 128 columns take, the four places of the tile that belong to
// the lane (row g = lane / 4, places 2t, 2t+1, 2t+8, 2t+9, t = lane % 4) hold four elements of block t of the 128 columns, and the lane that
// holds the X side of the same places (column n = lane / 4) reads the same elements.  Elements j and j + 4 of a word of codes sit in the two
// halves of the word, so a pair of bf16 weights takes two shifts and two logical operations: sign to bit 15, exponent and mantissa to bits
// 8..6, which is the value times 2^-126, an exact (for 0.5 subnormal) bf16 number; one multiplication by 2^126 times the block's scale makes
// it the weight, exact wherever the weight is a bf16 number.  Weights are used once, so they never see shared memory.
// Bound by HBM for few rows of X (4.25 bits per weight, each read once).
constexpr int kMxChunks = 4;            // chunks of 128 columns whose codes a warp loads together: 16 bytes of scales per row

__device__ __forceinline__ void mma_bf16(float d[4], const uint32_t a[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// Elements j and j + 4 of a word of codes, as bf16 times 2^-126.
template <int j>
__device__ __forceinline__ uint32_t mx_pair(uint32_t w)
{
    const uint32_t sign = j == 3 ? w : w << (12 - 4 * j), low = j < 2 ? w << (6 - 4 * j) : w >> (4 * j - 6);
    return (sign & 0x80008000u) | (low & 0x01c001c0u);
}

// What a block's pairs are multiplied with, as two bf16: first = 2^126 times the scale where that is a bf16 number (scales up to 2), second = 1;
// else 2^126 and the scale.
struct MxFactor { uint32_t first, second; };
__device__ __forceinline__ MxFactor mx_factor(uint32_t e)
{
    const uint32_t f = e <= 128u ? (e + 126u) << 7 : 253u << 7, s = e <= 128u ? 127u << 7 : e == 255u ? 0x7fc0u : e << 7;
    return {f | f << 16, s | s << 16};
}

struct MxProduct {
    const uint8_t *codes, *scales;
    int64_t n_out, k_in, kb, pitch;
    const __nv_bfloat16* x;
    int batch, x_align;                 // elements of X that one load may take: 8, 4, 2 or 1
    void* y;
    int split;                          // warps that share the columns of 16 rows: a power of two
};

// Eight elements of row n of X from column k on; zero past the end.
__device__ __forceinline__ uint4 load_x8(const MxProduct& a, int n, int64_t k)
{
    const __nv_bfloat16* p = a.x + (int64_t)n * a.k_in + k;
    if (k + 8 <= a.k_in && a.x_align == 8) return __ldg(reinterpret_cast<const uint4*>(p));
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (k + 8 <= a.k_in && a.x_align == 4) {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(p)), v = __ldg(reinterpret_cast<const uint2*>(p) + 1);
        return make_uint4(u.x, u.y, v.x, v.y);
    }
    if (k + 8 <= a.k_in && a.x_align == 2) {
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

template <int kTiles, bool kF32>
__global__ void __launch_bounds__(kMxThreads)
mx_product_kernel(MxProduct a)
{
    __shared__ float part[kMxThreads / 32][kTiles][8][17];     // per warp: 16 rows x 8 columns per tile (17: no two of a column in one bank)
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int share = warp % a.split, team = warp / a.split, teams = kMxThreads / 32 / a.split;
    const int64_t row0 = ((int64_t)blockIdx.x * teams + team) * 16;
    const int64_t r0 = min(row0 + g, a.n_out - 1), r1 = min(row0 + g + 8, a.n_out - 1);
    const uint8_t *c0 = a.codes + r0 * a.kb * kMxBlockBytes, *c1 = a.codes + r1 * a.kb * kMxBlockBytes;
    const uint8_t *s0 = a.scales + r0 * a.pitch, *s1 = a.scales + r1 * a.pitch;
    float acc[kTiles][4] = {};
    if (row0 < a.n_out) {
        for (int64_t b0 = (int64_t)share * (4 * kMxChunks); b0 < a.kb; b0 += (int64_t)a.split * (4 * kMxChunks)) {      // blocks b0 .. b0 + 15
            uint4 w[2][kMxChunks];
#pragma unroll
            for (int c = 0; c < kMxChunks; ++c) {
                const int64_t b = b0 + 4 * c + t;
                const bool in = b < a.kb;
                w[0][c] = in ? __ldcs(reinterpret_cast<const uint4*>(c0 + b * kMxBlockBytes)) : make_uint4(0u, 0u, 0u, 0u);
                w[1][c] = in ? __ldcs(reinterpret_cast<const uint4*>(c1 + b * kMxBlockBytes)) : make_uint4(0u, 0u, 0u, 0u);
            }
            const uint4 e0 = __ldg(reinterpret_cast<const uint4*>(s0 + b0)), e1 = __ldg(reinterpret_cast<const uint4*>(s1 + b0));
            const uint32_t e[2][4] = {{e0.x, e0.y, e0.z, e0.w}, {e1.x, e1.y, e1.z, e1.w}};
#pragma unroll
            for (int c = 0; c < kMxChunks; ++c) {
                const int64_t b = b0 + 4 * c + t;
                uint32_t ea = (e[0][c] >> (8 * t)) & 255u, eb = (e[1][c] >> (8 * t)) & 255u;
                if (b >= a.kb) { ea = 0u; eb = 0u; }            // bytes past the row's last block are not scales
                const MxFactor fa = mx_factor(ea), fb = mx_factor(eb);
                const bool large = __any_sync(0xffffffffu, max(ea, eb) > 128u);
                const uint32_t wa[4] = {w[0][c].x, w[0][c].y, w[0][c].z, w[0][c].w}, wb[4] = {w[1][c].x, w[1][c].y, w[1][c].z, w[1][c].w};
                uint32_t p[8][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[2 * i][0] = mul_bf16x2(mx_pair<0>(wa[i]), fa.first); p[2 * i][1] = mul_bf16x2(mx_pair<0>(wb[i]), fb.first);
                    p[2 * i][2] = mul_bf16x2(mx_pair<1>(wa[i]), fa.first); p[2 * i][3] = mul_bf16x2(mx_pair<1>(wb[i]), fb.first);
                    p[2 * i + 1][0] = mul_bf16x2(mx_pair<2>(wa[i]), fa.first); p[2 * i + 1][1] = mul_bf16x2(mx_pair<2>(wb[i]), fb.first);
                    p[2 * i + 1][2] = mul_bf16x2(mx_pair<3>(wa[i]), fa.first); p[2 * i + 1][3] = mul_bf16x2(mx_pair<3>(wb[i]), fb.first);
                }
                if (large) {
#pragma unroll
                    for (int s = 0; s < 8; ++s) {
                        p[s][0] = mul_bf16x2(p[s][0], fa.second); p[s][1] = mul_bf16x2(p[s][1], fb.second);
                        p[s][2] = mul_bf16x2(p[s][2], fa.second); p[s][3] = mul_bf16x2(p[s][3], fb.second);
                    }
                }
#pragma unroll
                for (int n = 0; n < kTiles; ++n) {
                    float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};      // 128 columns by the tensor core, the rest of the sum in binary32 with rounding
                    const int col = n * 8 + g;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint4 v = make_uint4(0u, 0u, 0u, 0u);
                        if (col < a.batch) v = load_x8(a, col, b * kMxBlock + 8 * i);
                        mma_bf16(d, p[2 * i], __byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632));
                        mma_bf16(d, p[2 * i + 1], __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[n][j] += d[j];
                }
            }
        }
    }
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
        part[warp][n][2 * t][g] = acc[n][0]; part[warp][n][2 * t + 1][g] = acc[n][1];
        part[warp][n][2 * t][g + 8] = acc[n][2]; part[warp][n][2 * t + 1][g + 8] = acc[n][3];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < teams * 16 * a.batch; i += kMxThreads) {
        const int r = i & 15, m = (i >> 4) % teams, n = (i >> 4) / teams;
        const int64_t row = ((int64_t)blockIdx.x * teams + m) * 16 + r;
        if (row >= a.n_out) continue;
        float s = 0.0f;
        for (int j = 0; j < a.split; ++j) s += part[m * a.split + j][n >> 3][n & 7][r];
        if (kF32) static_cast<float*>(a.y)[(int64_t)n * a.n_out + row] = s;
        else static_cast<__nv_bfloat16*>(a.y)[(int64_t)n * a.n_out + row] = __float2bfloat16_rn(s);
    }
}

// Sizes whose byte counts leave 63 bits, or dimensions that the kernels' indices do not hold.
bool mx_too_large(int64_t rows, int64_t cols) { return rows > (1ll << 31) || cols > (1ll << 31); }

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
    const uint32_t pieces = (uint32_t)(mx_scale_pitch(cols) / 8);
    const int64_t per_cta = kMxThreads / 32 * kMxUnroll, ctas = (rows * (int64_t)pieces + per_cta - 1) / per_cta;
    if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_pdl(mx_quantize_kernel<T>, (unsigned)ctas, kMxThreads, 0, st, static_cast<const T*>(x), rows, cols, ld, pieces, wide, codes, scales);
}

int mx_product(const llvq_ctx* ctx, const uint8_t* d_codes, const uint8_t* d_scales, int64_t n_out, int64_t k_in, const uint16_t* d_x, int batch, void* d_y,
               int y_dtype, cudaStream_t st)
{
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return LLVQ_ECUDA;
    if (k_in == 0) return cudaMemsetAsync(d_y, 0, (size_t)n_out * batch * (y_dtype == LLVQ_F32 ? 4 : 2), st) == cudaSuccess ? LLVQ_OK : LLVQ_ECUDA;
    MxProduct a{};
    a.codes = d_codes; a.scales = d_scales; a.n_out = n_out; a.k_in = k_in; a.kb = mx_blocks(k_in); a.pitch = mx_scale_pitch(k_in);
    a.x = reinterpret_cast<const __nv_bfloat16*>(d_x); a.batch = batch; a.y = d_y;
    a.x_align = 8;
    while (a.x_align > 1 && (!aligned(d_x, 2 * (size_t)a.x_align) || (batch > 1 && k_in % a.x_align != 0))) a.x_align /= 2;
    a.split = 1;
    while (a.split < kMxThreads / 32 && a.split * 4 * kMxChunks < a.kb) a.split *= 2;
    const int64_t rows_per_cta = 16 * (kMxThreads / 32 / a.split), ctas = (n_out + rows_per_cta - 1) / rows_per_cta;
    const int tiles = (batch + 7) / 8;
    cudaError_t r;
#define MX_PRODUCT(TILES)                                                                                                                     \
    r = y_dtype == LLVQ_F32 ? launch_pdl(mx_product_kernel<TILES, true>, (unsigned)ctas, kMxThreads, 0, st, a)                                \
                            : launch_pdl(mx_product_kernel<TILES, false>, (unsigned)ctas, kMxThreads, 0, st, a)
    if (tiles <= 1) MX_PRODUCT(1);
    else if (tiles <= 2) MX_PRODUCT(2);
    else if (tiles <= 4) MX_PRODUCT(4);
    else MX_PRODUCT(8);
#undef MX_PRODUCT
    return r == cudaSuccess ? launch_status() : LLVQ_ECUDA;
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
    return r == cudaSuccess ? launch_status() : r == cudaErrorInvalidValue ? LLVQ_EUNSUPPORTED : LLVQ_ECUDA;
}

int llvq_mx_gemv(const llvq_ctx* ctx, const uint8_t* d_codes, const uint8_t* d_scales, int64_t n_out, int64_t k_in, const uint16_t* d_x_bf16, void* d_y,
                 int y_dtype, void* stream)
{
    if (ctx && ctx->device >= 0 && n_out == 0) return LLVQ_OK;
    if (int e = mx_check(ctx, k_in == 0, d_codes, d_scales)) return e;
    if ((!d_x_bf16 && k_in != 0) || !d_y || n_out < 0 || k_in < 0 || (y_dtype != LLVQ_F32 && y_dtype != LLVQ_BF16)) return LLVQ_EINVAL;
    if (!aligned(d_x_bf16, 2) || !aligned(d_y, y_dtype == LLVQ_F32 ? 4 : 2)) return LLVQ_EALIGN;
    if (mx_too_large(n_out, k_in)) return LLVQ_EUNSUPPORTED;
    return mx_product(ctx, d_codes, d_scales, n_out, k_in, d_x_bf16, 1, d_y, y_dtype, (cudaStream_t)stream);
}

int llvq_mx_gemm_small_batch(const llvq_ctx* ctx, const uint8_t* d_codes, const uint8_t* d_scales, int64_t n_out, int64_t k_in, const uint16_t* d_x_bf16,
                             int batch, uint16_t* d_y_bf16, void* stream)
{
    if (ctx && ctx->device >= 0 && (n_out == 0 || batch == 0)) return LLVQ_OK;
    if (int e = mx_check(ctx, k_in == 0, d_codes, d_scales)) return e;
    if ((!d_x_bf16 && k_in != 0) || !d_y_bf16 || n_out < 0 || k_in < 0 || batch < 0) return LLVQ_EINVAL;
    if (!aligned(d_x_bf16, 2) || !aligned(d_y_bf16, 2)) return LLVQ_EALIGN;
    if (batch > 64 || mx_too_large(n_out, k_in)) return LLVQ_EUNSUPPORTED;
    return mx_product(ctx, d_codes, d_scales, n_out, k_in, d_x_bf16, batch, d_y_bf16, LLVQ_BF16, (cudaStream_t)stream);
}

}  // extern "C"
