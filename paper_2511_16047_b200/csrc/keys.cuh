// Keys and values that are not bf16 tokens of a layer's region: an encoder's states, of another length for every row, and a region
// held in 8 bits.  Shared by the two kernels that attend to them.  Keys come in blocks of 16 slots, of which the first `valid`
// hold a key.
#pragma once

#include "kernels.cuh"

namespace amskv {

// Division of numbers below 2^31 by a launch constant: three instructions where the compiler, not knowing it, takes about twenty.
struct Divisor {
    uint32_t d, mul, shift;
    __host__ void set(int32_t by)
    {
        d = (uint32_t)by;
        for (shift = 0; (1u << shift) < d; ++shift) {}
        mul = (uint32_t)((((1ull << shift) - d) << 32) / d + 1);
    }
    __device__ __forceinline__ int32_t operator()(int32_t n) const { return (int32_t)((__umulhi((uint32_t)n, mul) + (uint32_t)n) >> shift); }
};
constexpr int kBlock = 16;   // slots of a block

#ifdef __CUDACC__
// What the device knows of a row's keys, as loaded; made use of later, so that the loads can run ahead of it.
struct EncoderBounds {
    int32_t a = 0, b = 0;

    __device__ __forceinline__ EncoderBounds(const EncoderKeys& e, int32_t row)
    {
        if (e.offsets) {
            a = load_int(e.offsets + row);
            b = load_int(e.offsets + row + 1);
        } else if (e.lengths) {
            b = load_int(e.lengths + row);
        } else {
            b = e.keys;
        }
    }
    // (whatever is found there, nothing outside the tensor is read)
    __device__ __forceinline__ int32_t first(const EncoderKeys& e) const { return min(max(a, 0), e.keys); }
    __device__ __forceinline__ int32_t len(const EncoderKeys& e) const { return min(min(max(b, first(e)), e.keys) - first(e), e.max_keys); }
};
// The keys of one (row, key/value head) of an encoder.
struct EncoderView {
    const __nv_bfloat16 *k, *v;
    int64_t tok;
    int32_t len;

    __device__ __forceinline__ EncoderView(const EncoderKeys& e, int32_t row, int32_t kv_head, const EncoderBounds& bounds)
    {
        len = bounds.len(e);
        tok = e.tok;
        const int64_t at = (e.offsets ? 0 : row * e.row) + kv_head * e.head + bounds.first(e) * e.tok;
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
    const uint32_t* scales;    // [capacity / 16]
    int32_t capacity, total;
    int32_t range = 0, first = 0, n = 0;   // the range the walk is in, the number of its first block, and its blocks

    __device__ __forceinline__ HeldView(const HeldKeys& h, int64_t item, int32_t D)
        : ranges(h.ranges), codes(h.codes + item * 2 * h.capacity * D), scales(h.scales + item * (h.capacity / kBlock)),
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

// The powers of two of a block's keys and values, in one word: the exponent fields of bf16 factors 2^(120 + e), or of 2^127 where
// that is less, in bytes 0 (keys) and 1 (values), and what is then left of e in bytes 2 and 3.
__device__ __forceinline__ uint32_t scale_word(int32_t ke, int32_t ve)
{
    return (uint32_t)(min(ke, 7) + 247) | (uint32_t)(min(ve, 7) + 247) << 8 | (uint32_t)max(ke - 7, 0) << 16 | (uint32_t)max(ve - 7, 0) << 24;
}
// The word of a block that is no number: infinite factors, and nothing left (codes of 0 go with it).
constexpr uint32_t kNoNumber = 0x0000ffffu;
// of a word, for keys or values: the factor twice, and what is left of e
__device__ __forceinline__ uint32_t scale_factor(uint32_t word, bool values) { return ((values ? word >> 8 : word) & 0xffu) * 0x00800080u; }
__device__ __forceinline__ uint32_t scale_rest(uint32_t word, bool values) { return (values ? word >> 24 : word >> 16) & 0xffu; }
// 16 e4m3 codes times their power of two, exactly, as bf16.  With its sign spread over the byte above it a code is four bits short of
// its place in a bf16 that is 2^120 too small (which also holds for codes without a leading one), so that a shift, a mask and a
// product with the word's factor are all it takes; only magnitudes above 57 344 need a second product.
__device__ __forceinline__ void widen16(const uint4& codes, uint32_t f, uint32_t left, uint4& lo, uint4& hi)
{
    const uint32_t c[4] = {codes.x, codes.y, codes.z, codes.w};
    uint32_t out[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t w;
        if (i & 1) asm("prmt.b32 %0, %1, 0, 0xB3A2;" : "=r"(w) : "r"(c[i / 2]));
        else asm("prmt.b32 %0, %1, 0, 0x9180;" : "=r"(w) : "r"(c[i / 2]));
        w = (w << 4) & 0x87f087f0u;
        const __nv_bfloat162 x = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&w), *reinterpret_cast<const __nv_bfloat162*>(&f));
        out[i] = *reinterpret_cast<const uint32_t*>(&x);
    }
    if (left) {
        const uint32_t f2 = (left + 127u) * 0x00800080u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __nv_bfloat162 x = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&out[i]), *reinterpret_cast<const __nv_bfloat162*>(&f2));
            out[i] = *reinterpret_cast<const uint32_t*>(&x);
        }
    }
    lo = make_uint4(out[0], out[1], out[2], out[3]);
    hi = make_uint4(out[4], out[5], out[6], out[7]);
}
__device__ __forceinline__ void widen16_by(const uint4& codes, uint32_t word, bool values, uint4& lo, uint4& hi)
{
    widen16(codes, scale_factor(word, values), scale_rest(word, values), lo, hi);
}
// 16 bytes global -> shared, zeros where !real (src is not read then)
__device__ __forceinline__ void copy16_or_zero(uint32_t dst, const void* src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
#endif

}  // namespace amskv
