// What the kernels on microscaled 4-bit matrices share: tensor maps of byte rows, and scales on their way to tensor memory.
#pragma once
#include "launch_host.h"
#include "mx.cuh"
#include "umma.cuh"

namespace llvq {

constexpr uint32_t kScaleAtom = 512;                      // scales of 128 rows and 4 blocks: row r at 16 (r % 32) + 4 (r / 32), block j at byte j

// One lane of a warp whose lanes are all here.  Loops that issue MMAs are run by the whole warp and only the instructions themselves by this lane: with the
// loop in a branch on the lane's number 28672 x 8192 took 667 us instead of 543 for 4096 tokens, and 85 instead of 64 for 64 rows.
__device__ __forceinline__ bool elect_one()
{
    uint32_t is;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(is));
    return is != 0u;
}

// The warp's number, known to the compiler to be the same for all its lanes.
__device__ __forceinline__ int warp_number() { return __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0); }

// Named barrier 1 for `threads` threads, which also learn whether all of them are well: where one's wait ran out, all leave together, so that nobody is left
// at a barrier.
__device__ __forceinline__ bool all_well(bool well, int threads)
{
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.and.pred q, 1, %2, p;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"((uint32_t)well), "r"(threads) : "memory");
    return r != 0u;
}

// 512 bytes of scales from shared memory to four columns of tensor memory, for all four quarters of its lanes.
__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint64_t desc)      // desc = smem_desc(address, 0, 128)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// 16 scales (16 neighbouring blocks) of the rows l, l + 32, l + 64, l + 96 of 128, from a box of rows of 16 bytes in shared memory.
struct ScaleQuad { uint4 v[4]; };
__device__ __forceinline__ void read_scales(ScaleQuad& q, uint32_t smem, int lane)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(q.v[i].x), "=r"(q.v[i].y), "=r"(q.v[i].z), "=r"(q.v[i].w) : "r"(smem + (lane + 32 * i) * 16) : "memory");
}

__device__ __forceinline__ uint32_t word_of(const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// Word j of a quad (blocks first_block + 4 j ...) as an atom of scales; bytes of blocks past the row's last are zero.
template <int j>
__device__ __forceinline__ void store_scales(uint32_t smem, const ScaleQuad& q, uint32_t kb, uint32_t first_block, int lane)
{
    const uint32_t b = first_block + 4u * j, left = b < kb ? kb - b : 0u, keep = left >= 4u ? 0xffffffffu : (1u << (8u * left)) - 1u;
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(smem + lane * 16), "r"(word_of(q.v[0], j) & keep), "r"(word_of(q.v[1], j) & keep),
                 "r"(word_of(q.v[2], j) & keep), "r"(word_of(q.v[3], j) & keep) : "memory");
}

// `bytes` (a multiple of 16) from global to shared memory, both on 16-byte boundaries, counted on bar.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar)
{
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

// A tensor map of rows of bytes: boxes of `width` bytes by `box` rows.  (The driver's function asks for a current context: see make_x_map.)
inline bool make_byte_map(int device, const uint8_t* p, int64_t pitch, int64_t rows, int width, int box, bool swizzle, CUtensorMap* map)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t size[2] = {(cuuint32_t)width, (cuuint32_t)box}, steps[2] = {1, 1};
    auto made = [&] {
        return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(p), dims, strides, size, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                      swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    return made() || (cudaSetDevice(device) == cudaSuccess && made());
}

}  // namespace llvq
