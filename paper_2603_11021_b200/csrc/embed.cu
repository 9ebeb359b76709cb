// Rows of a table by token, times a scale, and the gradient of that with respect to the table; and the rows of a 4-bit matrix in order, which
// is its dequantisation (see include/llvq.h and mx.cuh).
#include <cooperative_groups.h>

#include "kernels_common.cuh"
#include "mx.cuh"

namespace {

using namespace llvq;

// ---- lookup -------------------------------------------------------------------------------------------------------------------------
// A thread writes whole 16-byte pieces of an output row, on 16-byte boundaries whatever the row's own alignment; the elements that belong there
// are taken out of the one or two aligned words of the source that hold them.  A group of lanes (32, or as many as a short row has pieces) takes
// kRowUnits pieces per lane of one row, all requested before the first is written, so that row, token and addresses are worked out once for them.
// Bound by HBM (and by latency for few tokens): each row is read and written once.
constexpr int kRowThreads = 256, kRowUnits = 4;

struct Rows {
    const uint8_t *src, *src_end;       // the table, or codes
    const uint8_t* scales;              // of codes
    int64_t src_pitch, scale_pitch;     // bytes per row
    int64_t vocab, n, dim, ld;          // ld: elements from one output row to the next
    const void* tokens;                 // null: row i of the table is row i of the output
    int token_bytes;
    uint8_t* out;
    float scale;
    uint32_t units, parts;              // pieces per output row; parts of kRowUnits pieces per lane that they make
    int lanes_log2;                     // lanes of a group
    unsigned long long* bad_index;
};

__device__ __forceinline__ int64_t load_token(const void* tokens, int bytes, int64_t i)
{
    return bytes == 8 ? __ldg(static_cast<const long long*>(tokens) + i) : (int64_t)__ldg(static_cast<const int*>(tokens) + i);
}

__device__ __forceinline__ uint32_t shift_words(uint32_t a, uint32_t b, uint32_t bytes) { return __funnelshift_r(a, b, bytes * 8u); }

// The 16 bytes at p (any multiple of 2 bytes).  around: the aligned 32 bytes that hold them may be read.
__device__ __forceinline__ uint4 load16(const uint8_t* p, bool around)
{
    const uint32_t k = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15u;
    if (k == 0u) return __ldg(reinterpret_cast<const uint4*>(p));
    if (around) {
        const uint4* lo = reinterpret_cast<const uint4*>(p - k);
        const uint4 a = __ldg(lo), b = __ldg(lo + 1);
        uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        if (k & 8u) {
#pragma unroll
            for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
        }
        if (k & 4u) {
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
        }
        return make_uint4(shift_words(w[0], w[1], k & 3u), shift_words(w[1], w[2], k & 3u), shift_words(w[2], w[3], k & 3u), shift_words(w[3], w[4], k & 3u));
    }
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 1] |= (uint32_t)__ldg(reinterpret_cast<const unsigned short*>(p) + i) << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T> __device__ __forceinline__ T scaled(T x, float s);
template <> __device__ __forceinline__ float scaled(float x, float s) { return x * s; }
template <> __device__ __forceinline__ __nv_bfloat16 scaled(__nv_bfloat16 x, float s) { return __float2bfloat16_rn(__bfloat162float(x) * s); }
template <> __device__ __forceinline__ __half scaled(__half x, float s) { return __float2half_rn(__half2float(x) * s); }

// Elements c .. c + 7 of a row of codes, times scale, as bf16; those past the row's last block are zero.
__device__ __forceinline__ uint4 mx_row8(const uint8_t* codes, const uint8_t* scales, uint32_t kb, uint32_t c, float scale)
{
    const uint32_t* words = reinterpret_cast<const uint32_t*>(codes);
    const uint32_t i = c >> 3, b = c >> 5, s = c & 7u;
    uint32_t w = __ldg(words + i);
    if (s) w = __funnelshift_r(w, i + 1u < kb * 4u ? __ldg(words + i + 1u) : 0u, 4u * s);
    const float f0 = mx_scale_value(__ldg(scales + b));
    const uint32_t left = 32u - (c & 31u);               // elements of this block from c on
    const float f1 = left < 8u && b + 1u < kb ? mx_scale_value(__ldg(scales + b + 1u)) : f0;
    float v[8];
    mx_expand8(w, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = v[j] * (j < (int)left ? f0 : f1) * scale;      // the first product is exact
    return make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
}

// Element c alone.
__device__ __forceinline__ __nv_bfloat16 mx_element(const uint8_t* codes, const uint8_t* scales, uint32_t c, float scale)
{
    float v[8];
    mx_expand8((uint32_t)__ldg(codes + (c >> 1)) >> (4u * (c & 1u)) & 15u, v);
    return __float2bfloat16_rn(v[0] * mx_scale_value(__ldg(scales + (c >> 5))) * scale);
}

// Two products with one factor.
__device__ __forceinline__ void scale_pair(float& x, float& y, float f)
{
    asm("{\n .reg .b64 a, b;\n mov.b64 a, {%0, %1};\n mov.b64 b, {%2, %2};\n mul.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a;\n}" : "+f"(x), "+f"(y) : "f"(f));
}

// The same for c a multiple of 8: one word, one block.
__device__ __forceinline__ uint4 mx_word8(uint32_t w, uint32_t e, float scale, bool times)
{
    const float f = mx_scale_value(e);
    float v[8];
    mx_expand8(w, v);
#pragma unroll
    for (int j = 0; j < 8; j += 2) scale_pair(v[j], v[j + 1], f);
    if (times) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) scale_pair(v[j], v[j + 1], scale);
    }
    return make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
}

// kEven: every output row starts on a 16-byte boundary.  kWhole: and is a whole number of pieces, as is every row of the table
template <typename T, bool kMx, bool kEven, bool kWhole>
__global__ void __launch_bounds__(kRowThreads)
rows_kernel(Rows a)
{
    constexpr int E = 16 / (int)sizeof(T);
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t lanes = 1u << a.lanes_log2, in = threadIdx.x & (lanes - 1u);
    const int64_t row = (((int64_t)blockIdx.x * kRowThreads) >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
    if (row >= a.n) return;
    const int64_t src = a.tokens ? load_token(a.tokens, a.token_bytes, row) : row;
    const bool known = src >= 0 && src < a.vocab;
    if (!known && in == 0 && blockIdx.y == 0) atomicAdd(a.bad_index, 1ull);
    T* out = reinterpret_cast<T*>(a.out) + row * a.ld;
    const uint8_t* from = a.src + (known ? src : 0) * a.src_pitch;
    const uint8_t* scales = a.scales + (known ? src : 0) * a.scale_pitch;
    const uint32_t kb = (uint32_t)mx_blocks(a.dim), dim = (uint32_t)a.dim;
    // elements ahead of the first boundary
    const uint32_t head = kEven ? 0u : ((16u - ((uint32_t)reinterpret_cast<uintptr_t>(out) & 15u)) & 15u) / (uint32_t)sizeof(T);
    for (uint32_t part = blockIdx.y; part < a.parts; part += gridDim.y) {
        const uint32_t q0 = part * (lanes * kRowUnits) + in;
        uint4 val[kRowUnits];
        if constexpr (kWhole) {
            const bool times = a.scale != 1.0f;
            if (kMx) {
                uint32_t w[kRowUnits], e[kRowUnits];
#pragma unroll
                for (int u = 0; u < kRowUnits; ++u) {
                    const uint32_t q = min(q0 + u * lanes, a.units - 1u);
                    w[u] = __ldg(reinterpret_cast<const uint32_t*>(from) + q);
                    e[u] = __ldg(scales + (q >> 2));
                }
#pragma unroll
                for (int u = 0; u < kRowUnits; ++u) val[u] = mx_word8(w[u], e[u], a.scale, times);
            } else {
#pragma unroll
                for (int u = 0; u < kRowUnits; ++u) val[u] = __ldg(reinterpret_cast<const uint4*>(from) + min(q0 + u * lanes, a.units - 1u));
                if (times) {
#pragma unroll
                    for (int u = 0; u < kRowUnits; ++u) {
                        T* v = reinterpret_cast<T*>(&val[u]);
#pragma unroll
                        for (int j = 0; j < E; ++j) v[j] = scaled(v[j], a.scale);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kRowUnits; ++u)
                if (q0 + u * lanes < a.units) reinterpret_cast<uint4*>(out)[q0 + u * lanes] = known ? val[u] : make_uint4(0u, 0u, 0u, 0u);
        } else {
            if constexpr (kMx && kEven) {                    // word and scale of every piece first
                uint32_t w[kRowUnits], e[kRowUnits];
#pragma unroll
                for (int u = 0; u < kRowUnits; ++u) {
                    const uint32_t q = q0 + u * lanes;
                    const bool there = known && q < a.units;
                    w[u] = there ? __ldg(reinterpret_cast<const uint32_t*>(from) + q) : 0u;
                    e[u] = there ? __ldg(scales + (q >> 2)) : 0u;
                }
#pragma unroll
                for (int u = 0; u < kRowUnits; ++u) val[u] = mx_word8(w[u], e[u], a.scale, true);
            }
            // pieces that are whole; the elements ahead of the first boundary and behind the last one by a lane each
            const uint32_t whole = dim > head ? (dim - head) / E : 0u, from_here = kEven && kMx ? 0u : head;
            const bool inside = from >= a.src + 16 && from + a.src_pitch + 16 <= a.src_end;      // also what lies 16 bytes around the row is in the table
            if constexpr (!(kMx && kEven)) {
#pragma unroll
                for (int u = 0; u < kRowUnits; ++u) {
                    const uint32_t q = min(q0 + u * lanes, whole - 1u), at = from_here + q * E;
                    if (whole == 0u) continue;
                    if constexpr (kMx) val[u] = mx_row8(from, scales, kb, at, a.scale);
                    else {
                        const T* p = reinterpret_cast<const T*>(from) + at;
                        val[u] = load16(reinterpret_cast<const uint8_t*>(p), inside);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kRowUnits; ++u) {
                const uint32_t q = q0 + u * lanes;
                if (!kMx && a.scale != 1.0f) {
                    T* v = reinterpret_cast<T*>(&val[u]);
#pragma unroll
                    for (int j = 0; j < E; ++j) v[j] = scaled(v[j], a.scale);
                }
                if (q < whole) *reinterpret_cast<uint4*>(out + from_here + q * E) = known ? val[u] : make_uint4(0u, 0u, 0u, 0u);
            }
            if (part == 0) {
                const uint32_t tail = from_here + whole * E, edges = dim > head ? head + (dim - tail) : dim;
                for (uint32_t i = in; i < edges; i += lanes) {
                    const uint32_t c = dim > head && (int)i >= (int)head ? tail + (i - head) : i;
                    T v = T(0.0f);
                    if (known) {
                        if constexpr (kMx) v = mx_element(from, scales, c, a.scale);
                        else v = a.scale != 1.0f ? scaled(reinterpret_cast<const T*>(from)[c], a.scale) : reinterpret_cast<const T*>(from)[c];
                    }
                    out[c] = v;
                }
            }
        }
    }
}

template <typename T, bool kMx>
int launch_rows(Rows a, cudaStream_t st)
{
    constexpr int E = 16 / (int)sizeof(T);
    const bool even = aligned(a.out, 16) && a.ld % E == 0;
    a.units = (uint32_t)((a.dim + E - 1) / E) + (even ? 0u : 1u);
    a.lanes_log2 = 0;
    while (a.lanes_log2 < 5 && (1u << a.lanes_log2) < a.units) ++a.lanes_log2;
    const uint32_t per_part = kRowUnits << a.lanes_log2;
    a.parts = (a.units + per_part - 1) / per_part;
    const int64_t rows_per_cta = kRowThreads >> a.lanes_log2, ctas = (a.n + rows_per_cta - 1) / rows_per_cta;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas, std::min(a.parts, 65535u)); cfg.blockDim = dim3(kRowThreads); cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    const bool whole = even && a.dim % E == 0 && (kMx || aligned(a.src, 16));
    const cudaError_t r = whole  ? cudaLaunchKernelEx(&cfg, rows_kernel<T, kMx, true, true>, a)
                          : even ? cudaLaunchKernelEx(&cfg, rows_kernel<T, kMx, true, false>, a)
                                 : cudaLaunchKernelEx(&cfg, rows_kernel<T, kMx, false, false>, a);
    return r == cudaSuccess ? launch_status() : LLVQ_ECUDA;
}

// ---- gradient -----------------------------------------------------------------------------------------------------------------------
// grad[v] = scale * sum of dy[i] over the i with token v, in an order that the inputs alone fix: the positions are sorted by token
// (stably), pieces of kPiece sorted positions are summed one position after the other in binary32, and the sums of a token whose positions
// lie in several pieces are added in the order of the pieces.  No floating-point atomics.
// Four kernels: the sort (up to kRankTokens tokens every token's place by comparison with all others, on all SMs; beyond, digit by digit in one
// cluster of thread blocks) while the next kernel clears all rows; then the sums, then those of them that reach across pieces.
// Bound by HBM: dy is read and the gradient written once, and the rows that tokens name are written a second time.
constexpr int kSortCtas = 8, kSortWarps = 32, kSortBits = 9, kSortBins = 1 << kSortBits;
// Gradients of 20000 x 256: 2048 tokens 15.0 us by comparison, 8192 tokens 35.8 us by comparison and 24.5 us by digits, 2049 tokens by digits 18.8 us.
constexpr int kRankTokens = 2048, kRankWarps = 8;
constexpr int kClearBytes = 64 << 10;   // per thread block: many short ones write faster than a few that stay (2.1 GB: 300 us against 340)
constexpr int kSpan = 256;              // columns per warp of the sums: eight per lane
constexpr int kSumWarps = 8;

struct EmbedGrad {
    const void* tokens;
    int token_bytes;
    int64_t n, vocab, dim, padding;
    uint32_t *key[2], *pos[2];          // sorted from one into the other, digit by digit
    int passes, bits;                   // digits of `bits` bits
    int sorted;                         // which of the two is sorted at the end
    int piece;                          // sorted positions per warp of the sums, at most 32
    const void* dy;
    void* grad;
    bool wide, accumulate;              // rows of dy and grad start on 16-byte boundaries; add to what grad holds
    float scale;
    float* part;                        // [pieces][2][dim rounded up to kSpan]: sums of tokens that reach across pieces
    unsigned long long* bad_index;
};

// What a token is sorted by: vocab, behind all others, where it has no row.
__device__ __forceinline__ uint32_t key_of(const EmbedGrad& a, int64_t token)
{
    return token < 0 || token >= a.vocab || token == a.padding ? (uint32_t)a.vocab : (uint32_t)token;
}

// Up to kRankTokens tokens: the place of each is the number of smaller keys and of equal ones ahead of it.  A thread block places 32 tokens, one per
// lane, and its warps share the others, all of which it holds in shared memory (rounded up to whole groups with keys that are larger than all).
__global__ void __launch_bounds__(kRankWarps * 32)
embed_rank_kernel(EmbedGrad a)
{
    extern __shared__ __align__(16) uint32_t rank_keys[];
    __shared__ uint32_t places[kRankWarps][32];
    pdl_wait();
    pdl_launch_dependents();                             // behind the wait: the clearing kernel does not wait, and may write what an earlier kernel read
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t n = (uint32_t)a.n, groups = (n + 31u) / 32u;
    constexpr int kAhead = 8;                            // tokens that a thread has requested
    for (uint32_t i0 = threadIdx.x; i0 < groups * 32u; i0 += kAhead * kRankWarps * 32) {
        int64_t token[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) token[u] = load_token(a.tokens, a.token_bytes, min(i0 + u * (kRankWarps * 32u), n - 1u));
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t i = i0 + u * (kRankWarps * 32u), k = key_of(a, token[u]);
            if (i < n && k == (uint32_t)a.vocab && token[u] != a.padding && i / 32u == blockIdx.x) atomicAdd(a.bad_index, 1ull);
            if (i < groups * 32u) rank_keys[i] = i < n ? k : 0xffffffffu;
        }
    }
    __syncthreads();
    const uint32_t mine = rank_keys[blockIdx.x * 32u + lane];
    uint32_t place = 0;
    for (uint32_t g = warp; g < groups; g += kRankWarps) {
        const uint4* k = reinterpret_cast<const uint4*>(rank_keys + g * 32u);
        if (g == blockIdx.x) {
#pragma unroll
            for (int j = 0; j < 32; ++j) { const uint32_t other = rank_keys[g * 32u + j]; place += other < mine || (other == mine && j < lane) ? 1u : 0u; }
        } else {
            const uint32_t border = mine + (g < blockIdx.x ? 1u : 0u);      // equal keys ahead count; keys are below 2^31
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint4 v = k[j];
                place += (v.x < border ? 1u : 0u) + (v.y < border ? 1u : 0u) + (v.z < border ? 1u : 0u) + (v.w < border ? 1u : 0u);
            }
        }
    }
    places[warp][lane] = place;
    __syncthreads();
    const uint32_t i = blockIdx.x * 32u + lane;
    if (warp == 0 && i < n) {
#pragma unroll
        for (int w = 1; w < kRankWarps; ++w) place += places[w][lane];
        a.key[a.sorted][place] = mine;
        a.pos[a.sorted][place] = i;
    }
}

// One digit.  A warp takes a contiguous run of items, 32 at a time, in both loops; place of an item = items of smaller digits + of the same
// digit in earlier thread blocks, warps and steps + in lower lanes.
__device__ void sort_digit(const EmbedGrad& a, int pass, uint32_t* hist, uint32_t* total, uint32_t* base, uint32_t* warp_sum)
{
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, bins = 1 << a.bits, shift = pass * a.bits;
    const uint32_t rank = cluster.block_rank();
    const int64_t runs = kSortCtas * kSortWarps, run = (a.n + runs * 32 - 1) / (runs * 32) * 32;
    const int64_t begin = min((rank * kSortWarps + warp) * run, a.n), end = min(begin + run, a.n);
    const uint32_t *key = a.key[pass & 1], *pos = a.pos[pass & 1];
    uint32_t *key_out = a.key[(pass & 1) ^ 1], *pos_out = a.pos[(pass & 1) ^ 1];
    uint32_t* mine = hist + warp * kSortBins;
    const uint32_t below = (1u << lane) - 1u;
    auto item = [&](int64_t i) -> uint32_t { return pass > 0 ? key[i] : key_of(a, load_token(a.tokens, a.token_bytes, i)); };
    for (int b = lane; b < bins; b += 32) mine[b] = 0u;
    __syncwarp();
    for (int64_t i = begin; i < end; i += 32) {
        const bool in = i + lane < end;
        const uint32_t k = in ? item(i + lane) : 0u;
        if (pass == 0 && in && k == (uint32_t)a.vocab && load_token(a.tokens, a.token_bytes, i + lane) != a.padding) atomicAdd(a.bad_index, 1ull);
        const uint32_t d = in ? (k >> shift) & (uint32_t)(bins - 1) : 0xffffffffu;
        const uint32_t same = __match_any_sync(0xffffffffu, d);
        if (in && (same & below) == 0u) mine[d] += (uint32_t)__popc(same);
        __syncwarp();
    }
    __syncthreads();
    if (tid < bins) {                                    // counts of the warps -> places inside this thread block's share of the digit
        uint32_t sum = 0;
        for (int w = 0; w < kSortWarps; ++w) { const uint32_t c = hist[w * kSortBins + tid]; hist[w * kSortBins + tid] = sum; sum += c; }
        total[tid] = sum;
    }
    cluster.sync();
    uint32_t before = 0, all = 0;
    if (tid < bins) {
        for (int c = 0; c < kSortCtas; ++c) {
            const uint32_t v = *cluster.map_shared_rank(total + tid, c);
            if (c < (int)rank) before += v;
            all += v;
        }
    }
    uint32_t upto = all;                                 // inclusive sums over the digits
    for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    if (tid < bins) {
        uint32_t ahead = 0;
        for (int w = 0; w < warp; ++w) ahead += warp_sum[w];
        base[tid] = ahead + upto - all + before;
    }
    __syncthreads();
    for (int b = lane; b < bins; b += 32) mine[b] += base[b];
    __syncwarp();
    for (int64_t i = begin; i < end; i += 32) {
        const bool in = i + lane < end;
        const uint32_t k = in ? item(i + lane) : 0u;
        const uint32_t d = in ? (k >> shift) & (uint32_t)(bins - 1) : 0xffffffffu;
        const uint32_t same = __match_any_sync(0xffffffffu, d);
        uint32_t at = 0;
        if (in) at = mine[d] + (uint32_t)__popc(same & below);
        __syncwarp();
        if (in && (same & below) == 0u) mine[d] += (uint32_t)__popc(same);
        __syncwarp();
        if (in) {
            key_out[at] = k;
            pos_out[at] = pass > 0 ? pos[i + lane] : (uint32_t)(i + lane);
        }
    }
    cluster.sync();                                      // the next digit, and its counters, after all of this one; what was written is seen
}

__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortWarps * 32, 1)
embed_sort_kernel(EmbedGrad a)
{
    extern __shared__ __align__(16) uint32_t sort_smem[];
    pdl_wait();
    pdl_launch_dependents();                             // behind the wait: the clearing kernel does not wait, and may write what an earlier kernel read
    uint32_t* hist = sort_smem;
    uint32_t *total = hist + kSortWarps * kSortBins, *base = total + kSortBins, *warp_sum = base + kSortBins;
    for (int pass = 0; pass < a.passes; ++pass) sort_digit(a, pass, hist, total, base, warp_sum);
}

// Clears [p, p + bytes) while the sort is running.  Its last thread block ends after the sort has: what waits for this kernel finds both done.
__global__ void __launch_bounds__(1024)
embed_clear_kernel(uint8_t* p, uint64_t bytes)
{
    pdl_launch_dependents();
    const uint64_t head = min((uint64_t)((16u - ((uint32_t)reinterpret_cast<uintptr_t>(p) & 15u)) & 15u), bytes);      // up to the first 16-byte boundary
    const uint64_t words = (bytes - head) / 16, tail = bytes - head - words * 16;
    uint4* w = reinterpret_cast<uint4*>(p + head);
    const uint64_t first = (uint64_t)blockIdx.x * (kClearBytes / 16) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kClearBytes / 16 / 1024; ++i)
        if (first + i * 1024 < words) w[first + i * 1024] = make_uint4(0u, 0u, 0u, 0u);
    if (blockIdx.x == 0) {
        if (threadIdx.x < head) p[threadIdx.x] = 0;
        if (threadIdx.x < tail) p[head + words * 16 + threadIdx.x] = 0;
    }
    if (blockIdx.x == gridDim.x - 1) pdl_wait();
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T rounded(float x);
template <> __device__ __forceinline__ float rounded(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half rounded(float x) { return __float2half_rn(x); }

// The column of element j of a lane, counted from the warp's first: eight neighbours where rows allow 16-byte accesses, else 32 apart.
template <bool kWide>
__device__ __forceinline__ int span_col(int lane, int j) { return kWide ? lane * 8 + j : j * 32 + lane; }

// Raw elements of a row of dy, as loaded: several rows of them are in flight at a time.
template <typename T, bool kWide> struct Span { T v[8]; };
template <> struct __align__(16) Span<float, true> { float v[8]; };
template <> struct __align__(16) Span<__nv_bfloat16, true> { __nv_bfloat16 v[8]; };
template <> struct __align__(16) Span<__half, true> { __half v[8]; };

template <typename T, bool kWide>
__device__ __forceinline__ void load_span(Span<T, kWide>& s, const T* row, int64_t col0, int lane, int64_t dim)
{
    if (kWide && col0 + lane * 8 + 8 <= dim) {
        const uint4* p = reinterpret_cast<const uint4*>(row + col0 + lane * 8);
        uint4* d = reinterpret_cast<uint4*>(s.v);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) d[i] = __ldcs(p + i);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t c = col0 + span_col<kWide>(lane, j);
            s.v[j] = c < dim ? row[c] : rounded<T>(0.0f);
        }
    }
}

template <typename G, bool kWide>
__device__ __forceinline__ void store_grad(const EmbedGrad& a, uint32_t key, int64_t col0, int lane, const float sum[8])
{
    G* row = static_cast<G*>(a.grad) + (int64_t)key * a.dim;
    if (kWide && col0 + lane * 8 + 8 <= a.dim) {
        __align__(16) G v[8];
        uint4* p = reinterpret_cast<uint4*>(row + col0 + lane * 8);
        if (a.accumulate) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(G) / 2; ++i) reinterpret_cast<uint4*>(v)[i] = p[i];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = rounded<G>(a.accumulate ? to_f(v[j]) + a.scale * sum[j] : a.scale * sum[j]);
#pragma unroll
        for (int i = 0; i < (int)sizeof(G) / 2; ++i) p[i] = reinterpret_cast<const uint4*>(v)[i];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t c = col0 + span_col<kWide>(lane, j);
            if (c < a.dim) row[c] = rounded<G>(a.accumulate ? to_f(row[c]) + a.scale * sum[j] : a.scale * sum[j]);
        }
    }
}

__device__ __forceinline__ float* part_of(const EmbedGrad& a, int64_t piece, int slot, int64_t col0, int lane)
{
    const int64_t padded = (a.dim + kSpan - 1) / kSpan * kSpan;
    return a.part + (piece * 2 + slot) * padded + col0 + lane * 8;
}

// A warp: a.piece sorted positions, kSpan columns.  Sums of tokens that begin and end inside the piece are final; the one that reaches in
// from the piece before goes to slot 0 of the piece, the one that begins here and reaches into the next to slot 1.
template <typename T, typename G, bool kWide>
__global__ void __launch_bounds__(kSumWarps * 32)
embed_sum_kernel(EmbedGrad a, int64_t pieces, uint32_t spans)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const uint32_t unit = blockIdx.x * kSumWarps + (threadIdx.x >> 5), piece = unit / spans;
    if (piece >= pieces) return;
    const int64_t col0 = (int64_t)(unit - piece * spans) * kSpan, first = (int64_t)piece * a.piece;
    const int count = (int)min((int64_t)a.piece, a.n - first);
    const uint32_t *keys = a.key[a.sorted], *poss = a.pos[a.sorted], none = (uint32_t)a.vocab;
    const uint32_t key = lane < count ? keys[first + lane] : none, pos = lane < count ? poss[first + lane] : 0u;
    const uint32_t key_before = first > 0 ? keys[first - 1] : none, key_after = first + count < a.n ? keys[first + count] : none;
    const int used = __popc(__ballot_sync(0xffffffffu, key != none));      // what has no row sorts last
    if (used == 0) return;
    uint32_t cur = __shfl_sync(0xffffffffu, key, 0);
    bool from_before = cur == key_before;
    float sum[8] = {};
    auto flush = [&](bool goes_on) {
        if (from_before || goes_on) {
            float* p = part_of(a, piece, from_before ? 0 : 1, col0, lane);
            *reinterpret_cast<float4*>(p) = make_float4(sum[0], sum[1], sum[2], sum[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(sum[4], sum[5], sum[6], sum[7]);
        } else {
            store_grad<G, kWide>(a, cur, col0, lane, sum);
        }
        from_before = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
    };
    constexpr int kAhead = sizeof(T) == 4 ? 4 : 8;       // rows in flight
    for (int i0 = 0; i0 < used; i0 += kAhead) {
        Span<T, kWide> s[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t p = __shfl_sync(0xffffffffu, pos, (i0 + i) & 31);
            if (i0 + i < used) load_span<T, kWide>(s[i], static_cast<const T*>(a.dy) + (int64_t)p * a.dim, col0, lane, a.dim);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (i0 + i < used) {
                const uint32_t k = __shfl_sync(0xffffffffu, key, (i0 + i) & 31);
                if (k != cur) {
                    flush(false);
                    cur = k;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += to_f(s[i].v[j]);
            }
        }
    }
    flush(cur == key_after);
}

// Sums that reach across pieces: a thread block takes those that begin in its piece (there is one at most), for kSpan columns, and its
// warps take contiguous runs of the pieces that follow.
template <typename G, bool kWide>
__global__ void __launch_bounds__(kSumWarps * 32)
embed_join_kernel(EmbedGrad a, int64_t pieces, uint32_t spans)
{
    __shared__ __align__(16) float sums[kSumWarps][kSpan];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t piece = blockIdx.x / spans, col0 = (int64_t)(blockIdx.x % spans) * kSpan, last = (piece + 1) * a.piece - 1;
    const uint32_t* keys = a.key[a.sorted];
    if (last + 1 >= a.n) return;
    const uint32_t key = keys[last];
    if (key == (uint32_t)a.vocab || keys[last + 1] != key) return;                        // nothing reaches out of the piece
    if (piece > 0 && keys[piece * a.piece] == key && keys[piece * a.piece - 1] == key) return;   // it began in an earlier one
    int64_t lo = piece + 1, hi = pieces;                // the first piece that does not begin with the token is in [lo, hi]: 32 of them looked at together
    while (lo < hi) {
        const int64_t step = (hi - lo + 31) / 32, at = lo + lane * step;
        const uint32_t same = __ballot_sync(0xffffffffu, at < hi && keys[at * a.piece] == key);
        const int t = __popc(same);                      // the first t of them do
        const int64_t end = lo + t * step;
        if (t > 0) lo = end - step + 1;
        hi = min(hi, end);
    }
    const int64_t more = lo - (piece + 1), run = (more + kSumWarps - 1) / kSumWarps;
    float sum[8] = {};
    auto add = [&](int64_t p, int slot) {
        const float* q = part_of(a, p, slot, col0, lane);
        const float4 u = *reinterpret_cast<const float4*>(q), v = *reinterpret_cast<const float4*>(q + 4);
        sum[0] += u.x; sum[1] += u.y; sum[2] += u.z; sum[3] += u.w; sum[4] += v.x; sum[5] += v.y; sum[6] += v.z; sum[7] += v.w;
    };
    if (warp == 0) add(piece, 1);
    const int64_t p1 = min(piece + 1 + (warp + 1) * run, lo);
#pragma unroll 4
    for (int64_t p = piece + 1 + warp * run; p < p1; ++p) add(p, 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[warp][j * 32 + lane] = sum[j];
    __syncthreads();
    if (warp != 0) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float s = sums[0][j * 32 + lane];
        for (int w = 1; w < kSumWarps; ++w) s += sums[w][j * 32 + lane];
        sum[j] = s;
    }
    store_grad<G, kWide>(a, key, col0, lane, sum);
}

int bits_of(uint64_t v)
{
    int b = 0;
    while (v) { ++b; v >>= 1; }
    return b;
}

// Positions per warp of the sums: as many as leave a warp to every slot of 148 SMs with 24 each, 32 at most and 8 at least.  The same on every device: the
// order of the additions and the size of the workspace follow from it.
int piece_of(int64_t n, int64_t dim)
{
    int piece = 32;
    while (piece > 8 && (n + piece - 1) / piece * ((dim + kSpan - 1) / kSpan) < 148 * 24) piece /= 2;
    return piece;
}

uint64_t round256(uint64_t v) { return (v + 255) / 256 * 256; }

template <typename T, typename G, bool kWide>
int launch_sums(const EmbedGrad& a, int64_t pieces, uint32_t spans, cudaStream_t st)
{
    const int64_t ctas = (pieces * (int64_t)spans + kSumWarps - 1) / kSumWarps;
    if (launch_pdl(embed_sum_kernel<T, G, kWide>, (unsigned)ctas, kSumWarps * 32, 0, st, a, pieces, spans) != cudaSuccess) return LLVQ_ECUDA;
    if (pieces > 1 && launch_pdl(embed_join_kernel<G, kWide>, (unsigned)(pieces * spans), kSumWarps * 32, 0, st, a, pieces, spans) != cudaSuccess) return LLVQ_ECUDA;
    return launch_status();
}

template <typename T, typename G>
int launch_sums(const EmbedGrad& a, int64_t pieces, uint32_t spans, cudaStream_t st)
{
    return a.wide ? launch_sums<T, G, true>(a, pieces, spans, st) : launch_sums<T, G, false>(a, pieces, spans, st);
}

template <typename T>
int launch_sums(const EmbedGrad& a, int grad_dtype, int64_t pieces, uint32_t spans, cudaStream_t st)
{
    return grad_dtype == LLVQ_F32 ? launch_sums<T, float>(a, pieces, spans, st)
           : grad_dtype == LLVQ_BF16 ? launch_sums<T, __nv_bfloat16>(a, pieces, spans, st)
                                     : launch_sums<T, __half>(a, pieces, spans, st);
}

bool dtype_ok(int t) { return t == LLVQ_F32 || t == LLVQ_BF16 || t == LLVQ_F16; }
int size_of(int t) { return t == LLVQ_F32 ? 4 : 2; }

}  // namespace

extern "C" {

int llvq_mx_dequant_matrix(const llvq_ctx* ctx, const uint8_t* d_codes, const uint8_t* d_scales, int64_t rows, int64_t cols, uint16_t* d_w_bf16, int64_t ld,
                           void* stream)
{
    if (ctx && ctx->device >= 0 && (rows == 0 || cols == 0)) return LLVQ_OK;      // nothing to do: pointers may be null
    if (!ctx || ctx->device < 0 || !d_codes || !d_scales || !d_w_bf16 || rows < 0 || cols < 0 || ld < cols) return LLVQ_EINVAL;
    if (!aligned(d_codes, 16) || !aligned(d_scales, 16) || !aligned(d_w_bf16, 2)) return LLVQ_EALIGN;
    if (rows > 0x7fffffffll || cols > (1ll << 30)) return LLVQ_EUNSUPPORTED;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return LLVQ_ECUDA;
    Rows a{};
    a.src = d_codes; a.scales = d_scales; a.src_pitch = mx_code_pitch(cols); a.scale_pitch = mx_scale_pitch(cols);
    a.vocab = rows; a.n = rows; a.dim = cols; a.ld = ld; a.out = reinterpret_cast<uint8_t*>(d_w_bf16); a.scale = 1.0f; a.bad_index = ctx->dev.bad_index;
    return launch_rows<__nv_bfloat16, true>(a, (cudaStream_t)stream);
}

int llvq_embed(const llvq_ctx* ctx, const void* d_table, int dtype, int64_t vocab, int64_t dim, const void* d_tokens, int token_bytes, int64_t n, float scale,
               void* d_out, void* stream)
{
    if (ctx && ctx->device >= 0 && (n == 0 || dim == 0)) return LLVQ_OK;
    if (!ctx || ctx->device < 0 || !d_table || !d_tokens || !d_out || vocab <= 0 || dim < 0 || n < 0) return LLVQ_EINVAL;
    if (!dtype_ok(dtype) || (token_bytes != 4 && token_bytes != 8)) return LLVQ_EINVAL;
    const int es = size_of(dtype);
    if (!aligned(d_table, es) || !aligned(d_out, es) || !aligned(d_tokens, token_bytes)) return LLVQ_EALIGN;
    if (vocab > 0x7fffffffll || dim > (1ll << 30) || n > 0x7fffffffll) return LLVQ_EUNSUPPORTED;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return LLVQ_ECUDA;
    Rows a{};
    a.src = static_cast<const uint8_t*>(d_table); a.src_pitch = dim * es; a.src_end = a.src + vocab * a.src_pitch;
    a.vocab = vocab; a.n = n; a.dim = dim; a.ld = dim; a.tokens = d_tokens; a.token_bytes = token_bytes; a.out = static_cast<uint8_t*>(d_out); a.scale = scale;
    a.bad_index = ctx->dev.bad_index;
    cudaStream_t st = (cudaStream_t)stream;
    return dtype == LLVQ_F32 ? launch_rows<float, false>(a, st) : dtype == LLVQ_BF16 ? launch_rows<__nv_bfloat16, false>(a, st) : launch_rows<__half, false>(a, st);
}

int llvq_mx_embed(const llvq_ctx* ctx, const uint8_t* d_codes, const uint8_t* d_scales, int64_t vocab, int64_t dim, const void* d_tokens, int token_bytes,
                  int64_t n, float scale, uint16_t* d_out_bf16, void* stream)
{
    if (ctx && ctx->device >= 0 && (n == 0 || dim == 0)) return LLVQ_OK;
    if (!ctx || ctx->device < 0 || !d_codes || !d_scales || !d_tokens || !d_out_bf16 || vocab <= 0 || dim < 0 || n < 0) return LLVQ_EINVAL;
    if (token_bytes != 4 && token_bytes != 8) return LLVQ_EINVAL;
    if (!aligned(d_codes, 16) || !aligned(d_scales, 16) || !aligned(d_out_bf16, 2) || !aligned(d_tokens, token_bytes)) return LLVQ_EALIGN;
    if (vocab > 0x7fffffffll || dim > (1ll << 30) || n > 0x7fffffffll) return LLVQ_EUNSUPPORTED;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return LLVQ_ECUDA;
    Rows a{};
    a.src = d_codes; a.scales = d_scales; a.src_pitch = mx_code_pitch(dim); a.scale_pitch = mx_scale_pitch(dim);
    a.vocab = vocab; a.n = n; a.dim = dim; a.ld = dim; a.tokens = d_tokens; a.token_bytes = token_bytes; a.out = reinterpret_cast<uint8_t*>(d_out_bf16);
    a.scale = scale; a.bad_index = ctx->dev.bad_index;
    return launch_rows<__nv_bfloat16, true>(a, (cudaStream_t)stream);
}

size_t llvq_embed_grad_bytes(int64_t n, int64_t dim)
{
    if (n <= 0 || dim <= 0 || n >= (1ll << 31) || dim > (1ll << 31)) return 0;
    const uint64_t piece = (uint64_t)piece_of(n, dim), pieces = ((uint64_t)n + piece - 1) / piece, padded = ((uint64_t)dim + kSpan - 1) / kSpan * kSpan;
    const unsigned __int128 all = (unsigned __int128)4 * round256((uint64_t)n * 4) + (unsigned __int128)pieces * 2 * padded * 4;
    return all > ((unsigned __int128)1 << 62) ? 0 : (size_t)all;
}

int llvq_embed_grad(const llvq_ctx* ctx, const void* d_dy, int dy_dtype, const void* d_tokens, int token_bytes, int64_t n, int64_t vocab, int64_t dim, float scale,
                    int64_t padding_idx, int accumulate, void* d_grad, int grad_dtype, void* d_work, void* stream)
{
    if (ctx && ctx->device >= 0 && (vocab == 0 || dim == 0)) return LLVQ_OK;
    if (!ctx || ctx->device < 0 || !d_grad || vocab < 0 || dim < 0 || n < 0 || !dtype_ok(dy_dtype) || !dtype_ok(grad_dtype)) return LLVQ_EINVAL;
    if (n > 0 && (!d_dy || !d_tokens || !d_work || (token_bytes != 4 && token_bytes != 8))) return LLVQ_EINVAL;
    const int es = size_of(dy_dtype), gs = size_of(grad_dtype);
    if (!aligned(d_grad, gs) || (n > 0 && (!aligned(d_dy, es) || !aligned(d_tokens, token_bytes) || !aligned(d_work, 256)))) return LLVQ_EALIGN;
    if (vocab >= (1ll << 31) || dim > (1ll << 31) || n >= (1ll << 31) || (n > 0 && llvq_embed_grad_bytes(n, dim) == 0)) return LLVQ_EUNSUPPORTED;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return LLVQ_ECUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if (n == 0) {
        if (accumulate) return LLVQ_OK;
        return cudaMemsetAsync(d_grad, 0, (size_t)vocab * dim * gs, st) == cudaSuccess ? LLVQ_OK : LLVQ_ECUDA;
    }
    EmbedGrad a{};
    a.tokens = d_tokens; a.token_bytes = token_bytes; a.n = n; a.vocab = vocab; a.dim = dim; a.padding = padding_idx;
    uint8_t* w = static_cast<uint8_t*>(d_work);
    const uint64_t list = round256((uint64_t)n * 4);
    a.key[0] = reinterpret_cast<uint32_t*>(w); a.key[1] = reinterpret_cast<uint32_t*>(w + list);
    a.pos[0] = reinterpret_cast<uint32_t*>(w + 2 * list); a.pos[1] = reinterpret_cast<uint32_t*>(w + 3 * list);
    a.part = reinterpret_cast<float*>(w + 4 * list);
    const int bits = bits_of((uint64_t)vocab);           // keys 0 .. vocab: the last for positions that have no row
    a.passes = (bits + kSortBits - 1) / kSortBits;
    a.bits = (bits + a.passes - 1) / a.passes;
    a.sorted = a.passes & 1;
    a.dy = d_dy; a.grad = d_grad; a.accumulate = accumulate != 0; a.scale = scale; a.bad_index = ctx->dev.bad_index;
    a.wide = aligned(d_dy, 16) && aligned(d_grad, 16) && dim * es % 16 == 0 && dim * gs % 16 == 0;
    a.piece = piece_of(n, dim);
    const uint64_t clear = accumulate ? 0 : (uint64_t)vocab * (uint64_t)dim * gs, clearing = (clear + 15 + kClearBytes - 1) / kClearBytes;
    const int64_t pieces = (n + a.piece - 1) / a.piece;
    const uint32_t spans = (uint32_t)((dim + kSpan - 1) / kSpan);
    if (clearing > 0x7fffffff || pieces * (int64_t)spans > 0x7fffffff) return LLVQ_EUNSUPPORTED;
    const size_t smem = (size_t)(kSortWarps * kSortBins + 2 * kSortBins + kSortWarps) * 4;
    if (!set_smem<embed_sort_kernel>(ctx, smem)) return LLVQ_ECUDA;
    const unsigned groups = (unsigned)((n + 31) / 32);
    const cudaError_t r = n <= kRankTokens ? launch_pdl(embed_rank_kernel, groups, kRankWarps * 32, groups * 128, st, a)
                                           : launch_pdl(embed_sort_kernel, (unsigned)kSortCtas, kSortWarps * 32, smem, st, a);
    if (r != cudaSuccess) return LLVQ_ECUDA;
    if (!accumulate && launch_pdl(embed_clear_kernel, (unsigned)clearing, 1024, 0, st, static_cast<uint8_t*>(d_grad), clear) != cudaSuccess) return LLVQ_ECUDA;
    return dy_dtype == LLVQ_F32    ? launch_sums<float>(a, grad_dtype, pieces, spans, st)
           : dy_dtype == LLVQ_BF16 ? launch_sums<__nv_bfloat16>(a, grad_dtype, pieces, spans, st)
                                   : launch_sums<__half>(a, grad_dtype, pieces, spans, st);
}

}  // extern "C"
