// A cache held in 8 bits: the append that quantises, and the copy of a segment out of a cache of either kind.
//
// A block is 16 tokens of one (row, head); its power of two is the least 2^e with no |x| above 448 * 2^e (the largest e4m3), at
// least 2^-100.  Powers of two cost a float code nothing but the headroom of one binade, and make code * 2^e exact in bf16, so that
// attention over the cache is attention over bf16 values, and x * 2^-e exact too (or a zero in any case), so that a value is rounded once.
// A block with an infinity or what is no number gets codes of 0 and an infinite power, whose products are NaN: nothing that reads the cache
// has to look for it.  Both are bound by memory: the append reads two bytes a channel and writes one.
#include <cuda_fp8.h>

#include "keys.cuh"

namespace amskv {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

__device__ __forceinline__ __nv_bfloat162 as_pair(uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); }
__device__ __forceinline__ __nv_bfloat162 abs_max2(__nv_bfloat162 a, uint32_t b) { return __hmax2_nan(a, __habs2(as_pair(b))); }   // (one instruction; keeps a NaN)
// four bf16 pairs -> eight codes.  (The product with a power of two is exact, or so small that its code is a zero.)
__device__ __forceinline__ uint2 codes_of(const uint4& x, __nv_bfloat162 inv)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 y = __hmul2(as_pair(w[i]), inv);
        const uint32_t bits = *reinterpret_cast<const uint32_t*>(&y);
        c[i] = __nv_cvt_float2_to_fp8x2(make_float2(__uint_as_float(bits << 16), __uint_as_float(bits & 0xffff0000u)), __NV_SATFINITE, __NV_E4M3);
    }
    return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}

// A warp per block of K or of V, which needs half the registers of one for both and leaves twice the warps to wait for memory (256 items,
// 1 024 tokens, 128 channels: 37.7 us, 29.1; 30.8 at the rate of a copy).  Divisions by launch constants are multiplications.
template <int D>
__global__ void __launch_bounds__(kThreads)
append_held_kernel(const __nv_bfloat16* K, const __nv_bfloat16* V, int64_t k_row, int64_t k_head, int64_t k_tok, int64_t v_row,
                   int64_t v_head, int64_t v_tok, uint8_t* codes, uint32_t* scales, int32_t capacity, int32_t offset, int32_t T,
                   Divisor blocks, Divisor heads, int32_t total)
{
    constexpr int kPieces = D / 8, kN = kBlock * kPieces / 32;   // 16-byte pieces of a token; of a lane
    const int lane = threadIdx.x & 31, piece = lane % kPieces, sub = lane / kPieces;
    overlap_with_previous();
    const int32_t step = (int32_t)gridDim.x * kWarps;
    for (int32_t at = (int32_t)blockIdx.x * kWarps + (int32_t)(threadIdx.x >> 5); at < total; at += step) {
        const int kv = at & 1;
        const int32_t item = blocks(at >> 1), b = (at >> 1) - item * (int32_t)blocks.d, row = heads(item), head = item - row * (int32_t)heads.d;
        const int64_t tok_stride = kv ? v_tok : k_tok;
        const __nv_bfloat16* src = (kv ? V + row * v_row + head * v_head : K + row * k_row + head * k_head) + (b * kBlock + sub) * tok_stride + piece * 8;
        const int32_t left = T - b * kBlock - sub;
        uint4 x[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) x[i] = i * (32 / kPieces) < left ? load_16B_once(src + i * (32 / kPieces) * tok_stride) : make_uint4(0, 0, 0, 0);
        __nv_bfloat162 most = as_pair(0);
#pragma unroll
        for (int i = 0; i < kN; ++i) most = abs_max2(abs_max2(abs_max2(abs_max2(most, x[i].x), x[i].y), x[i].z), x[i].w);
        const uint32_t top = *reinterpret_cast<const uint32_t*>(&most);   // (bits of numbers without a sign are ordered as the numbers are)
        const uint32_t amax = __reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16));   // bits of a bf16
        const bool none = amax >= 0x7f80u;
        // amax = (1 + f / 128) 2^(E - 127) <= 1.75 * 2^8 * 2^e
        const int32_t e = amax == 0 ? 0 : max((int32_t)(amax >> 7) - 135 + ((amax & 127u) > 96u ? 1 : 0), -100);
        const uint32_t inv = (uint32_t)(127 - e) * 0x00800080u;
        uint8_t* dst = codes + ((int64_t)item * 2 + kv) * ((int64_t)capacity * D) + (int64_t)(offset + b * kBlock) * D + lane * 8;
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (i * (32 / kPieces) < left) *reinterpret_cast<uint2*>(dst + i * 256) = none ? make_uint2(0, 0) : codes_of(x[i], as_pair(inv));
        if (lane == 0) {
            const uint32_t word = none ? kNoNumber : scale_word(e, e);
            uint8_t* bytes = reinterpret_cast<uint8_t*>(scales + (int64_t)item * (capacity / kBlock) + offset / kBlock + b) + kv;
            bytes[0] = (uint8_t)word;
            bytes[2] = (uint8_t)(word >> 16);
        }
    }
}

// 16 codes, or 8 bf16 values, a thread: K, then V.
template <bool kHeld>
__global__ void __launch_bounds__(kThreads)
read_segment_kernel(const void* region, const uint32_t* scales, int32_t capacity, int32_t offset, int32_t log_pieces, Divisor per_item,
                    Divisor heads, int64_t total, __nv_bfloat16* K, __nv_bfloat16* V, int64_t row_stride, int64_t head_stride, int64_t tok_stride)
{
    constexpr int kValues = kHeld ? 16 : 8;
    overlap_with_previous();
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x; at < total; at += step) {
        const int32_t half = total <= 0x7fffffff ? per_item((int32_t)at) : (int32_t)(at / per_item.d), item = half >> 1;
        const int32_t rest = (int32_t)(at - (int64_t)half * per_item.d), tok = rest >> log_pieces, piece = rest & ((1 << log_pieces) - 1);
        const int kv = half & 1;
        const int32_t row = heads(item), head = item - row * (int32_t)heads.d;
        const uint4 x = load_16B(static_cast<const uint4*>(region) + ((((int64_t)half * capacity + offset + tok) << log_pieces) + piece));
        uint4* dst = reinterpret_cast<uint4*>((kv ? V : K) + row * row_stride + head * head_stride + tok * tok_stride + piece * kValues);
        if (kHeld) {
            uint4 lo, hi;
            widen16_by(x, load_word(scales + (int64_t)item * (capacity / kBlock) + (offset + tok) / kBlock), kv != 0, lo, hi);
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
    const int64_t items = (int64_t)rows * heads, total = items * ((T + kBlock - 1) / kBlock) * 2;
    const int64_t grid = std::min<int64_t>((total + kWarps - 1) / kWarps, 64ll * sm_count);
    if (total + grid * kWarps > 0x7fffffffll) return cudaErrorInvalidValue;   // (2^31 blocks are more than a TB of codes)
    Divisor by_blocks, by_heads;
    by_blocks.set((T + kBlock - 1) / kBlock);
    by_heads.set(heads);
    auto* kernel = D == 64 ? append_held_kernel<64> : append_held_kernel<128>;
    return launch_kernel(true, kernel, dim3((unsigned)grid), dim3(kThreads), KernelMemory(0), stream, (const __nv_bfloat16*)K.ptr,
                         (const __nv_bfloat16*)V.ptr, K.row, K.head, K.token, V.row, V.head, V.token, region.codes, region.scales,
                         region.capacity, offset, T, by_blocks, by_heads, (int32_t)total);
}

cudaError_t launch_read_segment(const void* region, const uint32_t* scales, int32_t capacity, int32_t offset, int32_t T, int32_t rows,
                                int32_t heads, int32_t D, const Strided& K, const Strided& V, int sm_count, cudaStream_t stream)
{
    const int32_t pieces = D / (scales ? 16 : 8);   // 4, 8 or 16
    const int64_t items = (int64_t)rows * heads, per_item = (int64_t)T * pieces, total = items * 2 * per_item;
    if (per_item > 0x7fffffffll || items > 0x3fffffffll) return cudaErrorInvalidValue;
    const int64_t blocks = std::min<int64_t>((total + kThreads - 1) / kThreads, 64ll * sm_count);
    Divisor by_item, by_heads;
    by_item.set((int32_t)per_item);
    by_heads.set(heads);
    auto* kernel = scales ? read_segment_kernel<true> : read_segment_kernel<false>;
    return launch_kernel(true, kernel, dim3((unsigned)blocks), dim3(kThreads), KernelMemory(0), stream, region, scales, capacity, offset,
                         pieces == 4 ? 2 : pieces == 8 ? 3 : 4, by_item, by_heads, total, (__nv_bfloat16*)K.ptr, (__nv_bfloat16*)V.ptr, K.row,
                         K.head, K.token);
}

}  // namespace amskv
