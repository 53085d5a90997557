// Keys and values that are not bf16 tokens of a layer's region: an encoder's states, of another length for every row, and a region
// held in 8 bits.  Shared by the two kernels that attend to them.  Keys come in blocks of 16 slots, of which the first `valid`
// hold a key.
#pragma once

#include "kernels.cuh"

namespace amskv {

constexpr int kBlock = 16;   // slots of a block

#ifdef __CUDACC__
// The keys of one (row, key/value head) of an encoder.
struct EncoderView {
    const __nv_bfloat16 *k, *v;
    int64_t tok;
    int32_t len;

    __device__ __forceinline__ EncoderView(const EncoderKeys& e, int32_t row, int32_t kv_head)
    {
        int32_t first = 0, end = e.keys;
        if (e.offsets) {   // (whatever is found there, nothing outside the tensor is read)
            first = min(max(load_int(e.offsets + row), 0), e.keys);
            end = min(max(load_int(e.offsets + row + 1), first), e.keys);
        } else if (e.lengths) {
            end = min(max(load_int(e.lengths + row), 0), e.keys);
        }
        len = min(end - first, e.max_keys);
        tok = e.tok;
        const int64_t at = (e.offsets ? 0 : row * e.row) + kv_head * e.head + first * e.tok;
        k = e.K + at;
        v = e.V + at;
    }
    __device__ __forceinline__ int32_t blocks() const { return (len + kBlock - 1) / kBlock; }
    __device__ __forceinline__ int32_t valid(int32_t b) { return min(max(len - b * kBlock, 0), kBlock); }
};

// The keys of one item of a region held in 8 bits, in the order of its ranges; walks forward only.
struct HeldView {
    const RangeList& ranges;
    const uint8_t* codes;      // [capacity][D] keys, values behind them
    const int8_t* exps;        // [capacity / 16] of the keys, of the values behind them
    int32_t capacity, total;
    int32_t range = 0, first = 0, n = 0;   // the range the walk is in, the number of its first block, and its blocks

    __device__ __forceinline__ HeldView(const HeldKeys& h, int64_t item, int32_t D)
        : ranges(h.ranges), codes(h.codes + item * 2 * h.capacity * D), exps(h.exps + item * 2 * (h.capacity / kBlock)),
          capacity(h.capacity), total(h.blocks)
    {
        n = (ranges.r[0].len + kBlock - 1) / kBlock;
    }
    __device__ __forceinline__ int32_t blocks() const { return total; }
    __device__ __forceinline__ void walk(int32_t b)
    {
        while (b - first >= n) {
            first += n;
            ++range;
            n = (ranges.r[range].len + kBlock - 1) / kBlock;
        }
    }
    __device__ __forceinline__ int32_t valid(int32_t b)
    {
        if (b >= total) return 0;
        walk(b);
        return min(ranges.r[range].len - (b - first) * kBlock, kBlock);
    }
    __device__ __forceinline__ int32_t position(int32_t b)   // first slot of block b < total
    {
        walk(b);
        return ranges.r[range].start + (b - first) * kBlock;
    }
};

// Four e4m3 codes times a power of two, exactly, as bf16: the code's exponent and fraction are moved to their places (a bf16
// 2^120 too small, which also holds for the codes without a leading one), then scaled twice, as 2^120 and the block's power of two
// may be more than one bf16.
__device__ __forceinline__ void widen4(uint32_t codes, __nv_bfloat162 scale, uint32_t& a, uint32_t& b)
{
    constexpr uint32_t k2p120 = 0x7b807b80u;
    const uint32_t c[2] = {__byte_perm(codes, 0u, 0x1404), __byte_perm(codes, 0u, 0x3424)};
    uint32_t out[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t w = ((c[i] >> 4) & 0x07f007f0u) | (c[i] & 0x80008000u);
        const __nv_bfloat162 x = __hmul2(__hmul2(*reinterpret_cast<const __nv_bfloat162*>(&w), *reinterpret_cast<const __nv_bfloat162*>(&k2p120)), scale);
        out[i] = *reinterpret_cast<const uint32_t*>(&x);
    }
    a = out[0];
    b = out[1];
}
__device__ __forceinline__ void widen16(const uint4& codes, __nv_bfloat162 scale, uint4& lo, uint4& hi)
{
    widen4(codes.x, scale, lo.x, lo.y);
    widen4(codes.y, scale, lo.z, lo.w);
    widen4(codes.z, scale, hi.x, hi.y);
    widen4(codes.w, scale, hi.z, hi.w);
}
// 2^e for -126 <= e <= 127, twice
__device__ __forceinline__ __nv_bfloat162 power_of_two(int32_t e)
{
    const uint32_t w = (uint32_t)(e + 127) * 0x00800080u;
    return *reinterpret_cast<const __nv_bfloat162*>(&w);
}
__device__ __forceinline__ int32_t load_exponent(const int8_t* p)
{
    int32_t v;
    asm volatile("ld.global.s8 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
// 16 bytes global -> shared, zeros where !real (src must be readable-looking but is not read then)
__device__ __forceinline__ void copy16_or_zero(uint32_t dst, const void* src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
#endif

}  // namespace amskv
