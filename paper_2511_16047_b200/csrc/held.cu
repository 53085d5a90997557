// A cache held in 8 bits: the append that quantises, and the copy of a segment out of a cache of either kind.
//
// A block is 16 tokens of one (row, head); its power of two is the least 2^e with no |x| above 448 * 2^e (the largest e4m3), at
// least 2^-100.  Powers of two cost a float code nothing but the headroom of one binade, and make code * 2^e exact in bf16, so that
// attention over the cache is attention over bf16 values, and x * 2^-e exact in fp32, so that a value is rounded once.  Both are
// bound by memory: the append reads two bytes a channel and writes one.
#include <cuda_fp8.h>

#include "keys.cuh"

namespace amskv {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

__device__ __forceinline__ uint32_t abs_max2(uint32_t a, uint32_t b)   // of two bf16 pairs without their signs, lane by lane
{
    return __vmaxu2(a & 0x7fff7fffu, b & 0x7fff7fffu);                 // (their bits are ordered as their values are)
}
// four bf16 pairs -> eight codes
__device__ __forceinline__ uint2 codes_of(const uint4& x, float inv)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = make_float2(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xffff0000u) * inv);
        c[i] = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
    }
    return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}

// A warp takes the block of K, then that of V.
template <int D>
__global__ void __launch_bounds__(kThreads)
append_held_kernel(const __nv_bfloat16* K, const __nv_bfloat16* V, int64_t k_row, int64_t k_head, int64_t k_tok, int64_t v_row,
                   int64_t v_head, int64_t v_tok, uint8_t* codes, uint32_t* scales, int32_t capacity, int32_t offset, int32_t T,
                   int32_t heads, int64_t items)
{
    constexpr int kPieces = D / 8, kN = kBlock * kPieces / 32;   // 16-byte pieces of a token; of a lane
    const int lane = threadIdx.x & 31;
    const int32_t blocks = (T + kBlock - 1) / kBlock;
    overlap_with_previous();
    const int64_t total = items * blocks, step = (int64_t)gridDim.x * kWarps;
    for (int64_t at = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); at < total; at += step) {
        const int64_t item = at / blocks;
        const int32_t b = (int32_t)(at - item * blocks), row = (int32_t)(item / heads), head = (int32_t)(item - (int64_t)row * heads);
        uint4 x[2][kN];
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            const __nv_bfloat16* src = kv ? V + row * v_row + head * v_head : K + row * k_row + head * k_head;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const int p = i * 32 + lane, tok = b * kBlock + p / kPieces;
                x[kv][i] = tok < T ? load_16B_once(src + tok * (kv ? v_tok : k_tok) + p % kPieces * 8) : make_uint4(0, 0, 0, 0);
            }
        }
        int32_t power[2];
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < kN; ++i) top = abs_max2(abs_max2(abs_max2(top, x[kv][i].x), abs_max2(x[kv][i].y, x[kv][i].z)), x[kv][i].w);
            const uint32_t amax = __reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16));   // bits of a bf16
            // amax = (1 + f / 128) 2^(E - 127) <= 1.75 * 2^8 * 2^e
            const int32_t e = amax == 0 ? 0 : max((int32_t)(amax >> 7) - 135 + ((amax & 127u) > 96u ? 1 : 0), -100);
            const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
            uint8_t* dst = codes + (item * 2 + kv) * (int64_t)capacity * D + (int64_t)(offset + b * kBlock) * D;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const int p = i * 32 + lane;
                if (b * kBlock + p / kPieces < T) *reinterpret_cast<uint2*>(dst + p * 8) = codes_of(x[kv][i], inv);
            }
            power[kv] = e;
        }
        if (lane == 0) scales[item * (capacity / kBlock) + offset / kBlock + b] = scale_word(power[0], power[1]);
    }
}

// 16 codes, or 8 bf16 values, a thread: K, then V.
template <bool kHeld>
__global__ void __launch_bounds__(kThreads)
read_segment_kernel(const void* region, const uint32_t* scales, int32_t capacity, int32_t offset, int32_t T, int32_t D, int32_t heads,
                    int64_t items, __nv_bfloat16* K, __nv_bfloat16* V, int64_t row_stride, int64_t head_stride, int64_t tok_stride)
{
    constexpr int kValues = kHeld ? 16 : 8;
    overlap_with_previous();
    const int32_t pieces = D / kValues, per_item = T * pieces;
    const int64_t total = items * 2 * per_item, step = (int64_t)gridDim.x * kThreads;
    for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x; at < total; at += step) {
        const int64_t half = at / per_item, item = half >> 1;
        const int32_t rest = (int32_t)(at - half * per_item), tok = rest / pieces, piece = rest - tok * pieces;
        const int kv = (int)(half & 1);
        const int32_t row = (int32_t)(item / heads), head = (int32_t)(item - (int64_t)row * heads);
        const uint4 x = load_16B(static_cast<const uint4*>(region) + (half * capacity + offset + tok) * pieces + piece);
        uint4* dst = reinterpret_cast<uint4*>((kv ? V : K) + row * row_stride + head * head_stride + tok * tok_stride + piece * kValues);
        if (kHeld) {
            uint4 lo, hi;
            widen16_by(x, load_word(scales + item * (capacity / kBlock) + (offset + tok) / kBlock), kv != 0, lo, hi);
            dst[0] = lo;
            dst[1] = hi;
        } else {
            dst[0] = x;
        }
    }
}

}  // namespace

cudaError_t launch_append_held(const Strided& K, const Strided& V, const HeldRegion& region, int32_t offset, int32_t T, int32_t rows,
                               int32_t heads, int32_t D, int sm_count, cudaStream_t stream)
{
    const int64_t items = (int64_t)rows * heads, total = items * ((T + kBlock - 1) / kBlock);
    const int64_t blocks = std::min<int64_t>((total + kWarps - 1) / kWarps, 64ll * sm_count);
    auto* kernel = D == 64 ? append_held_kernel<64> : append_held_kernel<128>;
    return launch_kernel(true, kernel, dim3((unsigned)blocks), dim3(kThreads), KernelMemory(0), stream, (const __nv_bfloat16*)K.ptr,
                         (const __nv_bfloat16*)V.ptr, K.row, K.head, K.token, V.row, V.head, V.token, region.codes, region.scales,
                         region.capacity, offset, T, heads, items);
}

cudaError_t launch_read_segment(const void* region, const uint32_t* scales, int32_t capacity, int32_t offset, int32_t T, int32_t rows,
                                int32_t heads, int32_t D, const Strided& K, const Strided& V, int sm_count, cudaStream_t stream)
{
    const int64_t items = (int64_t)rows * heads, total = items * 2 * T * (D / (scales ? 16 : 8));
    const int64_t blocks = std::min<int64_t>((total + kThreads - 1) / kThreads, 64ll * sm_count);
    auto* kernel = scales ? read_segment_kernel<true> : read_segment_kernel<false>;
    return launch_kernel(true, kernel, dim3((unsigned)blocks), dim3(kThreads), KernelMemory(0), stream, region, scales, capacity, offset, T, D,
                         heads, items, (__nv_bfloat16*)K.ptr, (__nv_bfloat16*)V.ptr, K.row, K.head, K.token);
}

}  // namespace amskv
