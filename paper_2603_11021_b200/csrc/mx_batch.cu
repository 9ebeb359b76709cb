// Product of a microscaled 4-bit matrix with 2 to 64 rows of bf16 activations on the tensor cores' block-scaled instruction
// (see include/llvq.h and mx.cuh).
#include "kernels_common.cuh"
#include "mx_tensor.cuh"
#include "mx_batch.h"

namespace {

using namespace llvq;

// tcgen05.mma.kind::mxf8f6f4 multiplies e2m1 with e4m3, each with a power of two per row and 32 columns, so W goes to the tensor cores as it is stored
// and no weight passes through a register.  A bf16 number is three e4m3 numbers: with s = 2^(E - 7), E the exponent of the largest finite
// magnitude of the 32 columns,
//     x = s q1 + 2^-5 s q2 + 2^-23 s q3,   q1 = rn(x / s),  q2 = rn of 2^5 times what is left,  q3 = rn of 2^23 times what is left then.
// |x / s| < 256; q1 and q2 take four significant bits each, which is all of a bf16 number down to 2^-14 of the block's largest; with q3 it is exact
// down to 2^-19 of it, and what is smaller is off by at most 2^-27 of it, below the rounding of a sum in binary32 that holds the largest.
// A row of X is three columns of the product, added up in binary32 at the end.
//
// First kernel: the three terms of X, laid out as the second copies them (chunks of 128 columns: rows of 128 bytes, swizzled, then their scales),
// once for all thread blocks.  Second kernel: tiles of 256 rows of W (two accumulators that share what is read of X) by all of X.  The steps of
// 128 columns of all tiles are dealt out evenly in one line, so every SM reads the same share of W whatever the shape; a tile that several
// thread blocks share is added up by whichever is done last, in the order of the blocks.
//   warp 17     codes, as they are, with TMA: 64 bytes of 256 rows per step, kBatchPacked steps ahead
//   warps 8-15  two groups of four, every other step each: 8 bytes (16 elements) of codes to every 16 bytes of the operand: the form in which the
//               instruction takes 4-bit operands
//   warp 16     the scales of W    warp 18: X    warp 19: the MMAs, eight per step    warps 0-7: the accumulators and Y
// It begins to read W while the first kernel still runs (which waits for everything before it first).
// Bound by shared memory at 64 rows of X (28672 x 8192: 98 000 cycles, 1400 of them a step; 54 us at 1965 MHz, 63 in calls back to back, when the power limit
// leaves 1665): per step the MMAs read 80 KB (640 cycles at 128 bytes), codes are written, read and spread (512, the spread ones into every other pair of
// banks), X is written (200).  Fewer rows of X: by that and the latency of HBM.
constexpr int kBatchRows = 256, kBatchCols = 128, kBatchThreads = 640;
constexpr uint32_t kBatchA = kBatchRows * kBatchCols;     // bytes of a step's weights as operand, a byte of room per element
constexpr uint32_t kBatchCode = kBatchA / 2;              // and as they are stored
constexpr int kBatchPacked = 4, kBatchX = 3;              // steps of codes and of X in shared memory; of operands 3 for up to 32 rows of X, else 2
static_assert(kBatchPacked % 2 == 0, "");                 // a place in the ring of codes belongs to one of the two groups: each sees every phase of its barriers
constexpr int kRawScales = 3;                             // boxes of scales under way: 256 rows, 16 blocks, for four steps each

__host__ __device__ inline uint32_t batch_npad(int batch) { return (3u * (uint32_t)batch + 15u) / 16u * 16u; }
__host__ __device__ inline uint32_t batch_x_bytes(uint32_t npad) { return npad * 128u + 2u * kScaleAtom; }      // of a chunk

// The workspace: X in chunks, a counter per tile, a byte per chunk and row of X (not finite), sums of tiles that are shared (two per thread block).
struct BatchWork {
    uint64_t x, counters, notes, parts, bytes;
};
__host__ __device__ inline uint64_t up256(uint64_t v) { return (v + 255) / 256 * 256; }
BatchWork batch_work(int64_t n_out, int64_t k_in, int batch, int sms)
{
    const uint64_t chunks = (uint64_t)(k_in + kBatchCols - 1) / kBatchCols, tiles = (uint64_t)(n_out + kBatchRows - 1) / kBatchRows;
    BatchWork w;
    w.x = 0;
    w.counters = up256(chunks * batch_x_bytes(batch_npad(batch)));
    w.notes = w.counters + up256(tiles * 4);
    w.parts = w.notes + up256(chunks * batch);
    w.bytes = w.parts + (uint64_t)sms * 2 * kBatchRows * batch * 4;
    return w;
}

struct BatchArgs {
    const uint8_t *codes, *scales;
    int64_t n_out, k_in, code_pitch;
    uint32_t kb, scale_pitch, steps, tiles;               // blocks per row; steps of 128 columns per tile
    const __nv_bfloat16* x;
    int batch;
    bool x_quads;                                         // four elements of X may be loaded at once
    uint32_t npad, stages;
    uint8_t* x_chunks;
    uint32_t* counters;
    uint8_t* notes;
    float* parts;
    __nv_bfloat16* y;
    uint32_t* flags;
};

__device__ __forceinline__ uint32_t e4m3x4(const float v[4])
{
    uint32_t r;
    asm("{\n .reg .b16 lo, hi;\n cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n mov.b32 %0, {lo, hi};\n}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]));
    return r;
}

__device__ __forceinline__ void e4m3x4_values(uint32_t w, float v[4])
{
    uint32_t a, b;
    asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %2;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n cvt.rn.f16x2.e4m3x2 %1, hi;\n}" : "=r"(a), "=r"(b) : "r"(w));
    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&a)), q = __half22float2(*reinterpret_cast<const __half2*>(&b));
    v[0] = p.x; v[1] = p.y; v[2] = q.x; v[3] = q.y;
}

// A warp per row of X and chunk of 128 columns, four columns per lane.
__global__ void __launch_bounds__(256)
mx_batch_split_kernel(BatchArgs a)
{
    pdl_wait();
    pdl_launch_dependents();                              // behind the wait: what the next kernel reads ahead of its own was written before this one
    const int lane = threadIdx.x & 31;
    const uint32_t unit = blockIdx.x * 8u + (threadIdx.x >> 5);
    for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < a.tiles; i += gridDim.x * 256u) a.counters[i] = 0u;
    if (unit >= a.steps * (uint32_t)a.batch) return;
    const uint32_t chunk = unit / (uint32_t)a.batch, n = unit - chunk * (uint32_t)a.batch;
    const int64_t k = (int64_t)chunk * kBatchCols + lane * 4;
    const __nv_bfloat16* p = a.x + (int64_t)n * a.k_in + k;
    uint32_t w[2] = {0u, 0u};
    if (a.x_quads && k + 4 <= a.k_in) {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
        w[0] = u.x; w[1] = u.y;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (k + j < a.k_in) w[j >> 1] |= (uint32_t)__ldg(reinterpret_cast<const unsigned short*>(p) + j) << (16 * (j & 1));
    }
    float v[4];
    uint32_t most = 0, note = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t bits = (w[j >> 1] >> (16 * (j & 1))) & 0xffffu, size = bits & 0x7fffu;
        v[j] = __uint_as_float(bits << 16);
        if (size < 0x7f80u) most = max(most, size);
        else note |= size == 0x7f80u ? 1u : 2u;
        if (size >= 0x7f80u) v[j] = __uint_as_float(0x7fc00000u);        // no infinity in e4m3: the row's results are NaN, which mx_batch_kernel looks into
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    const uint32_t any = __any_sync(0xffffffffu, note & 2u) ? 2u : __any_sync(0xffffffffu, note & 1u) ? 1u : 0u;
    if (lane == 0) a.notes[(uint64_t)chunk * a.batch + n] = (uint8_t)any;
    uint8_t* to = a.x_chunks + (uint64_t)chunk * batch_x_bytes(a.npad);
    uint8_t* scales = to + a.npad * 128u;
    const int s1 = max((int)(most >> 7) - 7, 0);
#pragma unroll
    for (int term = 0; term < 3; ++term) {
        const int s = max(s1 - (term == 0 ? 0 : term == 1 ? 5 : 23), 0);
        const float up = __uint_as_float((uint32_t)(254 - s) << 23), down = mx_scale_value((uint32_t)s);      // s <= 247
        const uint32_t row = 3u * n + term;
        float q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = v[j] * up;
        const uint32_t packed = e4m3x4(q);
        *reinterpret_cast<uint32_t*>(to + row * 128u + ((((uint32_t)lane >> 2) ^ (row & 7u)) << 4) + (lane & 3u) * 4u) = packed;
        if ((lane & 7) == 0) scales[(row >> 7) * kScaleAtom + (row & 31u) * 16u + ((row & 127u) >> 5) * 4u + (lane >> 3)] = (uint8_t)s;
        e4m3x4_values(packed, q);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] -= q[j] * down;
    }
    if (n == 0) {                                         // rows that fill up the tile
        for (uint32_t row = 3u * a.batch; row < a.npad; ++row) {
            *reinterpret_cast<uint32_t*>(to + row * 128u + lane * 4u) = 0u;
            if (lane == 0) *reinterpret_cast<uint32_t*>(scales + (row >> 7) * kScaleAtom + (row & 31u) * 16u + ((row & 127u) >> 5) * 4u) = 0u;
        }
    }
}

// e2m1 (A) x e4m3 (B) with e8m0 scales, byte `id` of the words of scales -> f32, both operands K-major, M = 128, N = n
__device__ __forceinline__ uint32_t instr_desc_mxf4_f8(uint32_t n, uint32_t id)
{
    return id << 4 | 5u << 7 | 0u << 10 | (n >> 3) << 17 | 1u << 23 | (128u >> 4) << 24 | id << 29;
}

__device__ __forceinline__ void umma_mxf8f6f4(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t a_scales, uint32_t b_scales, uint32_t accumulate)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
                 " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(a_scales), "r"(b_scales), "r"(accumulate) : "memory");
}

__device__ __forceinline__ void arrive(uint64_t* bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory"); }

// The share of thread block i of `blocks`: steps [i * units / blocks, (i + 1) * units / blocks) of all tiles in one line.
__device__ __forceinline__ uint64_t share_begin(uint64_t units, uint32_t blocks, uint32_t i) { return units * i / blocks; }
__device__ __forceinline__ uint32_t share_owner(uint64_t units, uint32_t blocks, uint64_t u) { return (uint32_t)(((u + 1) * blocks - 1) / units); }

__device__ __forceinline__ void put_y(const BatchArgs& a, int64_t row, int n, float v) { a.y[(int64_t)n * a.n_out + row] = __float2bfloat16_rn(v); }

// Eight bits to the highest bits of eight nibbles.
__device__ __forceinline__ uint32_t nibble_tops(uint32_t bits)
{
    bits = (bits | bits << 12) & 0x000f000fu;
    bits = (bits | bits << 6) & 0x03030303u;
    return ((bits | bits << 3) & 0x11111111u) << 3;
}

// Rows of X that hold an infinity and no NaN (bits of `rows`), which the three terms cannot hold, for one row of W per thread: infinity times what is not
// zero is an infinity, times zero NaN, and what is finite does not matter beside it.  So signs and zeros of the codes that meet an infinity decide, 32 of
// them at a time: one load of a row's block per thread, and the infinities of a block of X by ballot.  All lanes of the warp come here.
// (28672 x 8192, 64 rows: 54 us without an infinity, 109 with one, 280 with nothing else; 12 ms where rows of W also have one sign and no zero, so that nothing
// is decided before the end.)
__device__ __noinline__ void mend_row(const BatchArgs& a, uint64_t rows, int64_t row)
{
    const int lane = threadIdx.x & 31;
    const bool there = row < a.n_out;
    const uint8_t* codes = a.codes + (there ? row : 0) * a.code_pitch;
    const uint8_t* scales = a.scales + (there ? row : 0) * a.scale_pitch;
    bool nan = !there;                                    // a block that is NaN, wherever it is
    for (uint32_t b = 0; b < a.kb; ++b) nan |= scales[b] == 255;
    for (; rows; rows &= rows - 1u) {
        const int n = __ffsll((long long)rows) - 1;
        const unsigned short* x = reinterpret_cast<const unsigned short*>(a.x) + (int64_t)n * a.k_in;
        bool up = nan, down = nan;                        // products that are +inf and -inf; both: NaN
        for (uint32_t c = 0; c < a.steps && !__all_sync(0xffffffffu, up && down); ++c) {
            if (a.notes[(uint64_t)c * a.batch + n] != 1u) continue;
            for (uint32_t b = 4u * c; b < min(4u * c + 4u, a.kb); ++b) {
                const int64_t k = (int64_t)b * kMxBlock + lane;
                const uint32_t v = k < a.k_in ? x[k] : 0u;
                const uint32_t plus = __ballot_sync(0xffffffffu, v == 0x7f80u), minus = __ballot_sync(0xffffffffu, v == 0xff80u);
                if ((plus | minus) == 0u) continue;
                const uint4 block = *reinterpret_cast<const uint4*>(codes + (int64_t)b * kMxBlockBytes);
                const uint32_t w[4] = {block.x, block.y, block.z, block.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t p = nibble_tops(plus >> (8 * i) & 255u), m = nibble_tops(minus >> (8 * i) & 255u), some = (w[i] & 0x77777777u) + 0x77777777u;
                    const bool zero = ((p | m) & ~some) != 0u;
                    up |= zero || ((p & ~w[i]) | (m & w[i])) != 0u;
                    down |= zero || ((p & w[i]) | (m & ~w[i])) != 0u;
                }
            }
        }
        if (there) put_y(a, row, n, __uint_as_float(up && down ? 0x7fc00000u : up ? 0x7f800000u : 0xff800000u));
    }
}

// A place in a ring of n and its phase.
struct Ring {
    uint32_t at = 0, phase = 0;
    __device__ __forceinline__ void next(uint32_t n, uint32_t by = 1u) { at += by; if (at >= n) { at -= n; phase ^= 1u; } }
};

__global__ void __launch_bounds__(kBatchThreads, 1)
mx_batch_kernel(const __grid_constant__ CUtensorMap code_map, const __grid_constant__ CUtensorMap scale_map, BatchArgs a)
{
    constexpr uint32_t kStage = kBatchA + 1024u;          // a step's weights and their scales
    extern __shared__ uint8_t mb_smem[];
    __shared__ uint64_t code_full[kBatchPacked], code_empty[kBatchPacked], full[3], empty[3], x_full[kBatchX], x_empty[kBatchX], raw_full[kRawScales], acc_full, acc_empty;
    __shared__ uint32_t tmem_slot, last_slot;
    __shared__ unsigned long long mend_rows;
    const uint32_t base = (smem_u32(mb_smem) + 1023u) & ~1023u, stages = a.stages;
    const uint32_t x_bytes = batch_x_bytes(a.npad), codes = base + stages * kStage, raw = codes + kBatchPacked * kBatchCode, x_at = raw + kRawScales * kBatchRows * 16u;
    const int warp = warp_number(), lane = threadIdx.x & 31;
    const uint64_t units = (uint64_t)a.tiles * a.steps, begin = share_begin(units, gridDim.x, blockIdx.x), end = share_begin(units, gridDim.x, blockIdx.x + 1);

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int e = 0; e < kBatchPacked; ++e) { mbar_init(code_full + e, 1); mbar_init(code_empty + e, 4); }
        for (int e = 0; e < 3; ++e) { mbar_init(full + e, 4 + 1); mbar_init(empty + e, 1); }        // four warps of codes, scales
        for (int e = 0; e < kBatchX; ++e) { mbar_init(x_full + e, 1); mbar_init(x_empty + e, 1); }
        for (int e = 0; e < kRawScales; ++e) mbar_init(raw_full + e, 1);
        mbar_init(&acc_full, 1);
        mbar_init(&acc_empty, 8);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 19) tmem_alloc(&tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    bool ok = true;
    const uint32_t total = (uint32_t)(end - begin);
    uint32_t tile = (uint32_t)(begin / a.steps), step = (uint32_t)(begin - (uint64_t)tile * a.steps), it = 0;      // it: steps so far
    auto advance = [&] { ++it; if (++step == a.steps) { step = 0; ++tile; } };

    if (warp >= 8 && warp < 16) {
        const uint32_t p = threadIdx.x & 127u, j = p & 3u, r = p >> 2;      // 16 bytes of a row; rows r, r + 32, ...
        const uint32_t to = r * 128u + (((2u * j) ^ (r & 7u)) << 4);      // the second half's place differs in the lowest bit
        Ring in, out;
        it = (uint32_t)(warp - 8) >> 2;
        in.next(kBatchPacked, it);
        out.next(stages, it);
        for (; it < total; it += 2) {
            ok = __all_sync(0xffffffffu, mbar_wait_copies(code_full + in.at, in.phase));
            if (!ok) break;
            uint4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w) : "r"(codes + in.at * kBatchCode + p * 16u + i * 2048u) : "memory");
            if (it >= stages) ok = __all_sync(0xffffffffu, mbar_wait(empty + out.at, out.phase ^ 1u));
            if (!ok) break;
            const uint32_t at = base + out.at * kStage + to;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(at + i * 4096u), "r"(v[i].x), "r"(v[i].y) : "memory");
                asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"((at ^ 16u) + i * 4096u), "r"(v[i].z), "r"(v[i].w) : "memory");
            }
            fence_async_smem();
            __syncwarp();
            // The codes' place is given back only now: the stores above had what was read in their registers.  Right behind the loads, other lanes' loads may
            // still be on their way, and where shared memory is busy the next codes overtake them.
            if (lane == 0) { arrive(full + out.at); arrive(code_empty + in.at); }
            in.next(kBatchPacked, 2u);
            out.next(stages, 2u);
        }
    } else if (warp == 17) {
        if (lane == 0) {
            Ring e;
            while (it < total) {
                if (it >= (uint32_t)kBatchPacked) ok = mbar_wait(code_empty + e.at, e.phase ^ 1u);
                if (!ok) break;
                mbar_expect(code_full + e.at, kBatchCode);
                tma_load_2d(codes + e.at * kBatchCode, &code_map, (int)(step * 64u), (int)(tile * kBatchRows), code_full + e.at);
                e.next(kBatchPacked);
                advance();
            }
        }
    } else if (warp == 16) {
        // boxes of scales are asked for kRawScales ahead; a box is in registers while its four words are stored
        uint32_t ask_it = 0, ask_tile = tile, ask_step = step;
        Ring asked, box, out;
        auto ask = [&] {
            if (ask_it >= total) return;
            if (lane == 0) {
                mbar_expect(raw_full + asked.at, kBatchRows * 16u);
                tma_load_2d(raw + asked.at * (kBatchRows * 16u), &scale_map, (int)(ask_step / 4u * 16u), (int)(ask_tile * kBatchRows), raw_full + asked.at);
            }
            asked.next(kRawScales);
            const uint32_t steps = min(4u - (ask_step & 3u), a.steps - ask_step);
            ask_it += steps;
            ask_step += steps;
            if (ask_step == a.steps) { ask_step = 0; ++ask_tile; }
        };
        for (int e = 0; e < kRawScales; ++e) ask();
        ScaleQuad now[2];
        bool fresh = true;
        while (it < total) {
            const uint32_t quad = step / 4u;
            if (fresh) {
                ok = __all_sync(0xffffffffu, mbar_wait_copies(raw_full + box.at, box.phase));
                if (!ok) break;
                read_scales(now[0], raw + box.at * (kBatchRows * 16u), lane);
                read_scales(now[1], raw + box.at * (kBatchRows * 16u) + 2048u, lane);
                box.next(kRawScales);
            }
            const bool was_fresh = fresh;
            fresh = (step & 3u) == 3u || step + 1u == a.steps;
            if (it >= stages) ok = __all_sync(0xffffffffu, mbar_wait(empty + out.at, out.phase ^ 1u));
            if (!ok) break;
            const uint32_t at = base + out.at * kStage + kBatchA;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t half = at + h * kScaleAtom;
                switch (step & 3u) {
                    case 0: store_scales<0>(half, now[h], a.kb, quad * 16u, lane); break;
                    case 1: store_scales<1>(half, now[h], a.kb, quad * 16u, lane); break;
                    case 2: store_scales<2>(half, now[h], a.kb, quad * 16u, lane); break;
                    default: store_scales<3>(half, now[h], a.kb, quad * 16u, lane);
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) arrive(full + out.at);
            if (was_fresh) ask();                         // into the box's place: the stores above had a part of every load in their registers
            out.next(stages);
            advance();
        }
    } else if (warp == 18) {
        if (lane == 0) {
            pdl_wait();
            Ring e;
            while (it < total) {
                if (it >= (uint32_t)kBatchX) ok = mbar_wait(x_empty + e.at, e.phase ^ 1u);
                if (!ok) break;
                mbar_expect(x_full + e.at, x_bytes);
                bulk_load(x_at + e.at * x_bytes, a.x_chunks + (uint64_t)step * x_bytes, x_bytes, x_full + e.at);
                e.next(kBatchX);
                advance();
            }
        }
    } else if (warp == 19) {
        uint32_t done = 0;
        Ring in, x;
        const uint64_t da0 = smem_desc_sw128(base), db0 = smem_desc_sw128(x_at), sa0 = smem_desc(base + kBatchA, 0u, 128u), sb0 = smem_desc(x_at + a.npad * 128u, 0u, 128u);
        const uint32_t id0 = instr_desc_mxf4_f8(a.npad, 0), x16 = x_bytes >> 4;
        const bool wide = a.npad > 128u;
        while (it < total && ok) {
            const uint32_t stop = min(total, it + (a.steps - step));
            if (done > 0) ok = __all_sync(0xffffffffu, mbar_wait(&acc_empty, (done - 1u) & 1u));
            for (uint32_t more = 0; it < stop && ok; more = 1u) {
                ok = __all_sync(0xffffffffu, mbar_wait_copies(x_full + x.at, x.phase) && mbar_wait_copies(full + in.at, in.phase));
                if (!ok) break;
                tc_fence_after();
                // scales have a place per stage; with two of them the step's number gives the same place without the ring (58.6 -> 54.9 us)
                const uint32_t off = in.at * (kStage >> 4), x_off = x.at * x16, ta = tmem + 384u + (stages == 2u ? it & 1u : in.at) * 16u, tb = ta + 8u;
                const uint64_t da = da0 + off, db = db0 + x_off, sa = sa0 + off, sb = sb0 + x_off;
                if (elect_one()) {
                    scales_to_tmem(ta, sa);
                    scales_to_tmem(ta + 4u, sa + (kScaleAtom >> 4));
                    scales_to_tmem(tb, sb);
                    if (wide) scales_to_tmem(tb + 4u, sb + (kScaleAtom >> 4));
#pragma unroll
                    for (int h = 0; h < 2; ++h)           // rows 0-127 and 128-255 of the tile
#pragma unroll
                        for (int q = 0; q < 4; ++q)       // 32 columns: 32 bytes on along the rows of either operand, the next byte of the scales
                            umma_mxf8f6f4(tmem + 192u * h, da + 1024u * h + 2 * q, db + 2 * q, id0 | (uint32_t)q << 4 | (uint32_t)q << 29, ta + 4u * h, tb, q > 0 ? 1u : more);
                    umma_commit(empty + in.at);
                    umma_commit(x_empty + x.at);
                }
                __syncwarp();
                in.next(stages);
                x.next(kBatchX);
                advance();
            }
            if (ok && elect_one()) umma_commit(&acc_full);
            __syncwarp();
            ++done;
        }
    } else {
        pdl_wait();
        uint32_t done = 0, odd_from = 0xffffffffu, odd_to = 0;      // the first and last tile with a result of this block's that is NaN
        for (; it < total; ++tile, ++done) {
            const uint64_t tile_begin = (uint64_t)tile * a.steps;
            it += a.steps - step;
            step = 0;
            ok = all_well(mbar_wait_copies(&acc_full, done & 1u), 256);
            if (!ok) break;
            tc_fence_after();
            const uint32_t from = share_owner(units, gridDim.x, tile_begin), to = share_owner(units, gridDim.x, tile_begin + a.steps - 1);
            const bool whole = from == to;
            const int r = warp * 32 + lane;
            const int64_t row = (int64_t)tile * kBatchRows + r;
            const uint32_t acc = tmem + ((uint32_t)(warp & 3) << 21) + (warp >= 4 ? 192u : 0u);
            // where a block's sums of this tile are: slot 0 for its first tile, 1 for its last.  Blocks behind the first of the tile begin in it.
            const uint64_t slot_floats = (uint64_t)(kBatchRows * a.batch);
            const uint32_t from_slot = share_begin(units, gridDim.x, from) == tile_begin ? 0u : 1u;
            auto slot = [&](uint32_t block) { return a.parts + ((uint64_t)block * 2 + (block == from ? from_slot : 0u)) * slot_floats + r; };
            float* part = slot(blockIdx.x);
            bool odd = false;
            for (int n0 = 0; n0 < a.batch; n0 += 16) {
                float v[48];
#pragma unroll
                for (int h = 0; h < 3; ++h)
                    if (3u * n0 + 16u * h < a.npad) tmem_ld16(acc + 3u * n0 + 16u * h, v + 16 * h);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    if (n0 + j >= a.batch) break;
                    const float sum = v[3 * j] + (v[3 * j + 1] + v[3 * j + 2]);
                    if (!whole) __stcg(part + (n0 + j) * kBatchRows, sum);
                    else if (row < a.n_out) { put_y(a, row, n0 + j, sum); odd |= sum != sum; }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive(&acc_empty);
            if (!whole) {                                 // the last of the blocks that share the tile adds their sums up
                __threadfence();
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (threadIdx.x == 0) last_slot = atomicAdd(a.counters + tile, 1u) == to - from;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                const bool last = last_slot != 0u;
                if (last) {
                    __threadfence();
                    // 16 rows of X of two blocks at a time, so that their loads overlap
                    for (int n0 = 0; n0 < a.batch; n0 += 16) {
                        float sum[16] = {};
                        for (uint32_t b = from; b <= to; b += 2) {
                            float v[2][16];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float* p = slot(min(b + h, to)) + n0 * kBatchRows;
#pragma unroll
                                for (int j = 0; j < 16; ++j) v[h][j] = b + h <= to && n0 + j < a.batch ? __ldcg(p + j * kBatchRows) : 0.0f;
                            }
#pragma unroll
                            for (int h = 0; h < 2; ++h)
#pragma unroll
                                for (int j = 0; j < 16; ++j) sum[j] += v[h][j];
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (n0 + j < a.batch && row < a.n_out) { put_y(a, row, n0 + j, sum[j]); odd |= sum[j] != sum[j]; }
                    }
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
            }
            if (odd) { odd_from = min(odd_from, tile); odd_to = tile; }
        }
        // Behind all tiles, where nobody waits for these warps: in between, rows full of infinities let the waits of the others run out.  A row of X with an
        // infinity is NaN in every result so far, so the first and last tile where one was seen are tiles that this block has written, as are all between them.
        if (ok && !all_well(odd_from == 0xffffffffu, 256)) {
            if (threadIdx.x == 0) mend_rows = 0ull;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            for (int n = warp; n < a.batch; n += 8) {
                uint32_t notes = 0;
                for (uint32_t c = lane; c < a.steps; c += 32) notes |= a.notes[(uint64_t)c * a.batch + n];
                if (__reduce_or_sync(0xffffffffu, notes) == 1u && lane == 0) atomicOr(&mend_rows, 1ull << n);
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
            const uint64_t rows = mend_rows;
            odd_from = __reduce_min_sync(0xffffffffu, odd_from);
            odd_to = __reduce_max_sync(0xffffffffu, odd_to);
            if (rows != 0u && odd_from != 0xffffffffu)
                for (uint32_t t = odd_from; t <= odd_to; ++t) mend_row(a, rows, (int64_t)t * kBatchRows + warp * 32 + lane);
        }
    }
    if (!ok) atomicOr(a.flags, (uint32_t)LLVQ_FLAG_WAIT_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 19) tmem_dealloc(tmem, 512);
}

}  // namespace

namespace llvq {

size_t mx_batch_bytes(const llvq_ctx* ctx, int64_t n_out, int64_t k_in, int batch) { return (size_t)batch_work(n_out, k_in, batch, ctx->sm_count).bytes; }

int mx_batch_product(const llvq_ctx* ctx, const uint8_t* d_codes, const uint8_t* d_scales, int64_t n_out, int64_t k_in, const uint16_t* d_x, int batch,
                     uint16_t* d_y, uint8_t* work, cudaStream_t st)
{
    BatchArgs a{};
    a.codes = d_codes; a.scales = d_scales; a.n_out = n_out; a.k_in = k_in; a.code_pitch = mx_code_pitch(k_in); a.scale_pitch = (uint32_t)mx_scale_pitch(k_in);
    a.kb = (uint32_t)mx_blocks(k_in); a.steps = (a.kb + 3) / 4; a.tiles = (uint32_t)((n_out + kBatchRows - 1) / kBatchRows);
    a.x = reinterpret_cast<const __nv_bfloat16*>(d_x); a.batch = batch; a.x_quads = aligned(d_x, 8) && (batch == 1 || k_in % 4 == 0);
    a.npad = batch_npad(batch); a.y = reinterpret_cast<__nv_bfloat16*>(d_y); a.flags = ctx->dev.flags;
    const BatchWork w = batch_work(n_out, k_in, batch, ctx->sm_count);
    a.x_chunks = work + w.x; a.counters = reinterpret_cast<uint32_t*>(work + w.counters); a.notes = work + w.notes; a.parts = reinterpret_cast<float*>(work + w.parts);
    const uint64_t split = ((uint64_t)a.steps * batch + 7) / 8;
    if (split > 0x7fffffff) return LLVQ_EUNSUPPORTED;
    if (launch_pdl(mx_batch_split_kernel, (unsigned)split, 256, 0, st, a) != cudaSuccess) return LLVQ_ECUDA;
    // A thread block per SM.  Few tiles: as many blocks per tile as take least, at 0.4 us a step and 0.3 us per block, and 16 rows of X, for adding up
    // (4096 x 4096, 20 rows: 9 blocks per tile 18.5 us, 4 of them 14.8 us).
    const uint64_t sms = (uint64_t)ctx->sm_count;
    uint64_t blocks = sms;
    if (a.tiles * 2ull <= sms) {
        uint64_t best = ~0ull;
        for (uint64_t s = 1; s <= std::min<uint64_t>(sms / a.tiles, a.steps); ++s) {
            const uint64_t cost = (a.steps + s - 1) / s * 4 + (s > 1 ? 3 * s * ((uint64_t)(batch + 15) / 16) : 0);
            if (cost < best) { best = cost; blocks = s * a.tiles; }
        }
    }
    const unsigned grid = (unsigned)std::min<uint64_t>((uint64_t)a.tiles * a.steps, blocks);
    a.stages = a.npad <= 96 ? 3u : 2u;
    const size_t smem = 1024 + (size_t)a.stages * (kBatchA + 1024u) + kBatchPacked * kBatchCode + kRawScales * kBatchRows * 16 + (size_t)kBatchX * batch_x_bytes(a.npad);
    CUtensorMap code_map, scale_map;
    if (!make_byte_map(ctx->device, a.codes, a.code_pitch, a.n_out, kBatchCols / 2, kBatchRows, false, &code_map) ||
        !make_byte_map(ctx->device, a.scales, a.scale_pitch, a.n_out, 16, kBatchRows, false, &scale_map)) return LLVQ_ECUDA;
    if (!set_smem<mx_batch_kernel>(ctx, smem)) return LLVQ_ECUDA;
    return launch_pdl(mx_batch_kernel, grid, kBatchThreads, smem, st, code_map, scale_map, a) == cudaSuccess ? launch_status() : LLVQ_ECUDA;
}

}  // namespace llvq
