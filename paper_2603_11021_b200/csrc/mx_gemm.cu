// Product of two matrices in microscaled 4-bit floating point on the tensor cores' own block-scaled instruction (see include/llvq.h and mx.cuh):
// Y[t][i] = sum_k X[t][k] W[i][k], both operands as llvq_mx_quantize leaves them, sums in binary32, Y in bf16.
#include "kernels_common.cuh"
#include "mx_tensor.cuh"
#include "mx_tiles.h"

namespace {

using namespace llvq;

// tcgen05.mma.kind::mxf4 takes e2m1 operands from shared memory and one e8m0 scale per row and 32 columns from tensor memory: nothing of
// either operand passes through registers.  A thread block computes tiles of kRt x 128 rows of W (128 lanes of tensor memory each) by kBn tokens
// (columns), 256 columns of both operands (128 bytes of codes per row) per stage:
//   warp 0      copies codes with TMA (swizzled rows of 128 bytes; what lies past the matrix reads as zero)
//   warps 2, 3  lay the scales of W and X out as tcgen05.cp wants them: of 128 rows and 4 blocks, 512 bytes, row r at 16 (r % 32) + 4 (r / 32).
//               A lane copies 16 scales of four rows 32 apart ahead (the rows' padding is for that) and stores four times 16 bytes of them in
//               two stages.  (With TMA, whose time goes by rows whatever their length, they took as long as half of the codes.)
//   warp 1      copies the scales to tensor memory and issues four MMAs of 64 columns per 128 rows and stage
//   warps 4-11  take the accumulators out as bf16, hand them back, then write Y
// Large products are bound by what TMA and L2 bring, so the large tile is the one that reads least per product: 256 rows by 224 tokens fill tensor
// memory with two accumulators and the scales of two stages (60 KB per stage for 1.75 times the products of 128 x 256, which reads 48 KB).  There is one set
// of accumulators: taking it out costs the tensor cores a few hundred of the tens of thousands of cycles of a tile.
constexpr int kMmThreads = 384;
constexpr int kMmGroup = 16;                              // row tiles that are walked together, for L2
constexpr uint32_t kStageCodes = 128;                     // bytes of a row's codes per stage: 256 columns

constexpr int kRawAhead = 3;                              // scales under way, of two stages each

template <int kRt, int kBn> struct MmShape {
    static constexpr int kRows = 128 * kRt, kBHalves = kBn > 128 ? 2 : 1;      // rows of W; groups of 128 tokens
    static constexpr uint32_t kA = kRows * kStageCodes, kB = kBn * kStageCodes, kScales = 2 * (kRt + kBHalves) * kScaleAtom;
    static constexpr uint32_t kStage = kA + kB + kScales; // a multiple of 1024
    static constexpr int kStages = kRt == 2 ? 3 : kBn == 256 ? 4 : kBn == 128 ? 6 : 7;
    static constexpr uint32_t kScaleCols = 8 * (kRt + kBHalves);               // columns of tensor memory that a stage's scales take
    static constexpr int kScaleBufs = kRt == 2 ? 2 : kStages;                  // a place per stage where tensor memory has them
    static constexpr uint32_t kCols = kRt * kBn + kScaleBufs * kScaleCols, kTmem = kCols > 256 ? 512 : kCols > 128 ? 256 : 128;
    static constexpr uint32_t kRaw = (kRt + kBHalves) * 128 * 16;      // scales as they come, of two stages
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kStage + kRawAhead * kRaw + 256;
    static_assert(kStage % 1024 == 0 && kCols <= kTmem && kSmem <= 227 * 1024, "");
};

struct MmArgs {
    const uint8_t *w_scales, *x_scales;
    int64_t n_out, tokens;
    uint32_t kb, pitch, k_stages;                         // blocks per row, bytes per row of scales, stages per tile
    uint32_t tiles_m, tiles_n;
    __nv_bfloat16* y;
    uint32_t* flags;
};

// e2m1 x e2m1 with e8m0 scales -> f32, both operands K-major, M = 128, N = n; the scales of the k-th pair of blocks of a column of scales
__device__ __forceinline__ uint32_t instr_desc_mxf4(uint32_t n, uint32_t pair)
{
    return (2u * pair) << 4 | 1u << 7 | 1u << 10 | (n >> 3) << 17 | 1u << 23 | (128u >> 4) << 24 | (2u * pair) << 29;
}

__device__ __forceinline__ void umma_mxf4(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t a_scales, uint32_t b_scales, uint32_t accumulate)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
                 " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(a_scales), "r"(b_scales), "r"(accumulate) : "memory");
}

// 32 consecutive accumulator columns of this thread's lane, as pairs of bf16.
__device__ __forceinline__ void tmem_ld32_bf16(uint32_t taddr, uint32_t v[16])
{
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = bf16_pair(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
}

__device__ __forceinline__ void mm_tile(const MmArgs& a, uint32_t tile, uint32_t& m, uint32_t& n)
{
    const uint32_t per_group = kMmGroup * a.tiles_n, group = tile / per_group, in = tile - group * per_group;
    const uint32_t high = min((uint32_t)kMmGroup, a.tiles_m - group * kMmGroup);
    n = in / high;
    m = group * kMmGroup + (in - n * high);
}

template <int kRt, int kBn>
__global__ void __launch_bounds__(kMmThreads, 1)
mx_gemm_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map, MmArgs a)
{
    using S = MmShape<kRt, kBn>;
    extern __shared__ uint8_t mm_smem[];
    const uint32_t base = (smem_u32(mm_smem) + 1023u) & ~1023u;
    uint64_t* bars = reinterpret_cast<uint64_t*>(mm_smem + (base - smem_u32(mm_smem)) + S::kStages * S::kStage + kRawAhead * S::kRaw);
    uint64_t *full = bars, *empty = bars + S::kStages, *acc_full = bars + 2 * S::kStages, *acc_empty = acc_full + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 1);
    const int warp = warp_number(), lane = threadIdx.x & 31;

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) { mbar_init(full + s, 3); mbar_init(empty + s, 1); }      // TMA, scales of W, scales of X
        mbar_init(acc_full, 1);
        mbar_init(acc_empty, 8);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(tmem_slot, S::kTmem);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_wait();

    const uint32_t tiles = a.tiles_m * a.tiles_n;
    bool ok = true;
    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            for (uint32_t tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
                uint32_t m, n;
                mm_tile(a, tile, m, n);
                for (uint32_t k = 0; k < a.k_stages && ok; ++k, ++it) {
                    const uint32_t s = it % S::kStages, round = it / S::kStages;
                    if (round > 0) ok = mbar_wait(empty + s, (round - 1u) & 1u);
                    if (!ok) break;
                    const uint32_t at = base + s * S::kStage;
                    mbar_expect(full + s, S::kA + S::kB);
                    tma_load_2d(at, &w_map, (int)(k * kStageCodes), (int)(m * S::kRows), full + s);
                    tma_load_2d(at + S::kA, &x_map, (int)(k * kStageCodes), (int)(n * kBn), full + s);
                }
            }
        }
    } else if (warp == 1) {
        uint32_t done = 0, s = 0, phase = 0, it = 0, old = 0, old_phase = 0;
        const uint64_t da0 = smem_desc_sw128(base), db0 = smem_desc_sw128(base + S::kA), sc0 = smem_desc(base + S::kA + S::kB, 0u, 128u);
        for (uint32_t tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x, ++done) {
            if (done > 0) ok = __all_sync(0xffffffffu, mbar_wait(acc_empty, (done - 1u) & 1u));
            for (uint32_t k = 0; k < a.k_stages && ok; ++k) {
                ok = __all_sync(0xffffffffu, mbar_wait_copies(full + s, phase));
                if (!ok) break;
                // fewer places of scales than stages: the MMAs that read this one are waited for (those of the stage before are still running)
                if (S::kScaleBufs < S::kStages && it >= (uint32_t)S::kScaleBufs) {
                    ok = __all_sync(0xffffffffu, mbar_wait(empty + old, old_phase));
                    if (!ok) break;
                    if (++old == (uint32_t)S::kStages) { old = 0; old_phase ^= 1u; }
                }
                tc_fence_after();
                const uint32_t off = s * (S::kStage >> 4), ta = tmem + kRt * kBn + (S::kScaleBufs == 2 ? it & 1u : s) * S::kScaleCols, tb = ta + 8 * kRt;
                const uint64_t da = da0 + off, db = db0 + off, sc = sc0 + off;
                if (elect_one()) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {         // blocks 0-3 and 4-7 of the stage
#pragma unroll
                        for (int g = 0; g < kRt; ++g) scales_to_tmem(ta + h * 4 * kRt + 4 * g, sc + (g * 2 + h) * (kScaleAtom >> 4));
#pragma unroll
                        for (int g = 0; g < S::kBHalves; ++g) scales_to_tmem(tb + h * 4 * S::kBHalves + 4 * g, sc + (2 * kRt + g * 2 + h) * (kScaleAtom >> 4));
                    }
#pragma unroll
                    for (int g = 0; g < kRt; ++g)
#pragma unroll
                        for (int q = 0; q < 4; ++q)       // 64 columns: 32 bytes on along the rows, two blocks on along the scales
                            umma_mxf4(tmem + g * kBn, da + g * (128 * kStageCodes >> 4) + 2 * q, db + 2 * q, instr_desc_mxf4(kBn, q & 1), ta + (q >> 1) * 4 * kRt + 4 * g,
                                      tb + 4 * S::kBHalves * (q >> 1), k > 0 || q > 0);
                    umma_commit(empty + s);
                }
                __syncwarp();
                ++it;
                if (++s == (uint32_t)S::kStages) { s = 0; phase ^= 1u; }
            }
            if (ok && elect_one()) umma_commit(acc_full);
            __syncwarp();
        }
    } else if (warp < 4) {
        const bool of_w = warp == 2;
        constexpr int kGroups = kRt > S::kBHalves ? kRt : S::kBHalves;      // of 128 rows
        const int groups = of_w ? kRt : S::kBHalves;
        const uint8_t* scales = of_w ? a.w_scales : a.x_scales;
        const int64_t rows = of_w ? a.n_out : a.tokens;
        const uint32_t raw = base + S::kStages * S::kStage + (of_w ? 0u : kRt * 2048u);
        // a lane copies what it will read itself: its own copies are all that it waits for
        uint32_t ask_tile = blockIdx.x, ask_k = 0, ask_at = 0, at = 0;
        int64_t ask_row = 0;
        auto ask = [&] {
            if (ask_tile < tiles) {
                if (ask_k == 0) {
                    uint32_t m, n;
                    mm_tile(a, ask_tile, m, n);
                    ask_row = (of_w ? (int64_t)m * S::kRows : (int64_t)n * kBn) + lane;
                }
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    if (g >= groups) continue;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int64_t row = ask_row + 128 * g + 32 * i;
                        const bool there = row < rows;
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(raw + ask_at * S::kRaw + g * 2048u + (lane + 32 * i) * 16u),
                                     "l"(there ? scales + row * a.pitch + ask_k * 8u : scales), "r"(there ? 16u : 0u) : "memory");
                    }
                }
                ask_k += 2;
                if (ask_k >= a.k_stages) { ask_k = 0; ask_tile += gridDim.x; }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (++ask_at == (uint32_t)kRawAhead) ask_at = 0;
        };
        for (int e = 0; e < kRawAhead - 1; ++e) ask();
        uint32_t it = 0;
        for (uint32_t tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
            ScaleQuad now[kGroups];
            for (uint32_t k = 0; k < a.k_stages && ok; ++k, ++it) {
                if ((k & 1u) == 0u) {
                    ask();
                    asm volatile("cp.async.wait_group %0;" ::"n"(kRawAhead - 1) : "memory");
#pragma unroll
                    for (int g = 0; g < kGroups; ++g)
                        if (g < groups) read_scales(now[g], raw + at * S::kRaw + g * 2048u, lane);
                    if (++at == (uint32_t)kRawAhead) at = 0;
                }
                const uint32_t s = it % S::kStages, round = it / S::kStages;
                if (round > 0) ok = __all_sync(0xffffffffu, mbar_wait(empty + s, (round - 1u) & 1u));
                if (!ok) break;
                const uint32_t at = base + s * S::kStage + S::kA + S::kB + (of_w ? 0u : 2 * kRt * kScaleAtom);
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    if (g >= groups) continue;
                    const uint32_t to = at + 2 * g * kScaleAtom, first = (k / 2) * 16u;
                    if ((k & 1u) == 0u) {
                        store_scales<0>(to, now[g], a.kb, first, lane);
                        store_scales<1>(to + kScaleAtom, now[g], a.kb, first, lane);
                    } else {
                        store_scales<2>(to, now[g], a.kb, first, lane);
                        store_scales<3>(to + kScaleAtom, now[g], a.kb, first, lane);
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(full + s)) : "memory");
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        // a quarter of the lanes each, of one accumulator, or of half of its columns where there is one
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        constexpr int kCols = kRt == 2 ? kBn : kBn / 2;   // of this warp
        uint32_t done = 0;
        for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x, ++done) {
            uint32_t m, n;
            mm_tile(a, tile, m, n);
            ok = __all_sync(0xffffffffu, mbar_wait(acc_full, done & 1u));
            if (!ok) break;
            tc_fence_after();
            uint32_t v[kCols / 2];
#pragma unroll
            for (int c = 0; c < kCols / 32; ++c) tmem_ld32_bf16(tmem + ((uint32_t)quarter << 21) + half * kCols + 32 * c, v + 16 * c);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(acc_empty)) : "memory");
            const int64_t row = (int64_t)m * S::kRows + (kRt == 2 ? 128 * half : 0) + 32 * quarter + lane, token = (int64_t)n * kBn + (kRt == 2 ? 0 : half * kCols);
            if (row < a.n_out) {
                __nv_bfloat16* y = a.y + token * a.n_out + row;
                const int left = (int)min((int64_t)kCols, a.tokens - token);
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    if (c < left) *y = __ushort_as_bfloat16((unsigned short)(v[c >> 1] >> (16 * (c & 1))));
                    y += a.n_out;
                }
            }
        }
    }
    if (!ok) atomicOr(a.flags, (uint32_t)LLVQ_FLAG_WAIT_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, S::kTmem);
}

template <int kTile>
int launch_mx_gemm(const llvq_ctx* ctx, const uint8_t* x_codes, const uint8_t* w_codes, int64_t k_in, MmArgs a, cudaStream_t st)
{
    constexpr int kRt = kMxTiles[kTile].rows / 128, kBn = kMxTiles[kTile].tokens;
    using S = MmShape<kRt, kBn>;
    CUtensorMap w_map, x_map;
    const int64_t pitch = mx_code_pitch(k_in);
    if (!make_byte_map(ctx->device, w_codes, pitch, a.n_out, (int)kStageCodes, S::kRows, true, &w_map) ||
        !make_byte_map(ctx->device, x_codes, pitch, a.tokens, (int)kStageCodes, kBn, true, &x_map)) return LLVQ_ECUDA;
    if (!set_smem<mx_gemm_kernel<kRt, kBn>>(ctx, S::kSmem)) return LLVQ_ECUDA;
    a.tiles_m = (uint32_t)((a.n_out + S::kRows - 1) / S::kRows);
    a.tiles_n = (uint32_t)((a.tokens + kBn - 1) / kBn);
    const unsigned grid = (unsigned)std::min<uint64_t>((uint64_t)a.tiles_m * a.tiles_n, (uint64_t)ctx->sm_count);
    return launch_pdl(mx_gemm_kernel<kRt, kBn>, grid, kMmThreads, S::kSmem, st, w_map, x_map, a) == cudaSuccess ? launch_status() : LLVQ_ECUDA;
}

}  // namespace

extern "C" int llvq_mx_gemm(const llvq_ctx* ctx, const uint8_t* d_x_codes, const uint8_t* d_x_scales, int64_t tokens, const uint8_t* d_codes,
                            const uint8_t* d_scales, int64_t n_out, int64_t k_in, uint16_t* d_y_bf16, void* stream)
{
    if (ctx && ctx->device >= 0 && (n_out == 0 || tokens == 0)) return LLVQ_OK;       // nothing to do: pointers may be null
    if (!ctx || ctx->device < 0 || n_out < 0 || tokens < 0 || k_in < 0 || !d_y_bf16) return LLVQ_EINVAL;
    if (k_in > 0 && (!d_x_codes || !d_x_scales || !d_codes || !d_scales)) return LLVQ_EINVAL;
    if (!aligned(d_x_codes, 16) || !aligned(d_x_scales, 16) || !aligned(d_codes, 16) || !aligned(d_scales, 16) || !aligned(d_y_bf16, 2)) return LLVQ_EALIGN;
    if (n_out > (1ll << 30) || tokens > (1ll << 30) || k_in > (1ll << 30)) return LLVQ_EUNSUPPORTED;      // TMA coordinates
    if (((n_out + 127) / 128) * ((tokens + 63) / 64) > (1ll << 31)) return LLVQ_EUNSUPPORTED;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return LLVQ_ECUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if (k_in == 0) return cudaMemsetAsync(d_y_bf16, 0, (size_t)n_out * tokens * 2, st) == cudaSuccess ? LLVQ_OK : LLVQ_ECUDA;
    MmArgs a{};
    a.w_scales = d_scales; a.x_scales = d_x_scales; a.n_out = n_out; a.tokens = tokens; a.kb = (uint32_t)mx_blocks(k_in); a.pitch = (uint32_t)mx_scale_pitch(k_in);
    a.k_stages = (a.kb + 7) / 8; a.y = reinterpret_cast<__nv_bfloat16*>(d_y_bf16); a.flags = ctx->dev.flags;
    switch (mx_tile_of(n_out, tokens, a.k_stages, ctx->sm_count)) {
        case 0: return launch_mx_gemm<0>(ctx, d_x_codes, d_codes, k_in, a, st);
        case 1: return launch_mx_gemm<1>(ctx, d_x_codes, d_codes, k_in, a, st);
        case 2: return launch_mx_gemm<2>(ctx, d_x_codes, d_codes, k_in, a, st);
        default: return launch_mx_gemm<3>(ctx, d_x_codes, d_codes, k_in, a, st);
    }
}
