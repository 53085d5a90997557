// Rotary positions: a table of cosines and sines from positions, and the rotation of Q and K by its rows.
//
// A pair (u, w) of channels turns by the angle of its axis and frequency: (u c - w s, w c + u s), in fp32 with one rounding to
// bf16.  Both kernels are bound by memory: the rotation reads and writes Q and K once (a token's table row is shared by its heads),
// the table is written once.
#include "kernels.cuh"

namespace amskv {

namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- the table
// Entry (n, column) = (cos, sin) of positions[n][axis] * frequency, times the amplitude.  An fp32 angle would be off by 0.06 at position
// 10^6.  Here the frequency is a fraction of a turn in 64 bits, the position 24 bits and an exponent, and the 64 low bits of their product
// lose whole turns by wrapping around, which is all the range reduction there is.  The top 32 bits of that, within an eighth of a turn
// of a quarter, become an fp32 angle (off by 2^-23 of at most pi / 4) for the Taylor sums of sine (to the 9th power: 2e-9 is left) and
// cosine (to the 10th: 1e-10).  What bounds it is the instructions: 131 071 x 64 entries 22.0 us, against 10.3 for the table's bytes;
// with fp64 angles 27.4, with 88-bit products and sincospif 31.2 (95 instructions an entry).
struct TableRow {   // what a position is, for all its columns
    uint32_t m, sign;
    int32_t shift;      // position = +-m * 2^shift
    bool none;          // not a number or infinite: no angle
    bool fixed;         // a multiple of 1 / 256 below 2^23, as token numbers are, and then `parts` of them
    int32_t parts;
    __device__ __forceinline__ explicit TableRow(float position)
    {
        const uint32_t bits = __float_as_uint(position), exponent = (bits >> 23) & 0xffu;
        m = exponent ? (bits & 0x7fffffu) | 0x800000u : bits & 0x7fffffu;
        sign = (uint32_t)((int32_t)bits >> 31);
        shift = (int32_t)max(exponent, 1u) - 150;
        none = exponent == 255;
        const float scaled = position * 256.f;
        fixed = fabsf(scaled) < 2147483648.f && scaled == rintf(scaled);
        parts = fixed ? (int32_t)scaled : 0;
    }
};
__device__ __forceinline__ float2 table_entry(const TableRow& p, uint64_t turns, float amplitude)
{
    // (a right shift leaves out bits of the frequency that the product would bring to less than 2^-32 turns)
    uint32_t x;   // 2^-32 turns
    if (p.fixed) {
        const uint64_t f = turns >> 8;
        const uint32_t q = (uint32_t)abs(p.parts);
        x = __umulhi(q, (uint32_t)f) + q * (uint32_t)(f >> 32);
    } else {
        const uint64_t f = p.shift >= 0 ? (p.shift < 64 ? turns << p.shift : 0ull) : (p.shift > -64 ? turns >> -p.shift : 0ull);
        x = __umulhi(p.m, (uint32_t)f) + p.m * (uint32_t)(f >> 32);
    }
    x = (x ^ p.sign) - p.sign;
    const uint32_t quarter = (x + 0x20000000u) >> 30;
    const float r = (float)(int32_t)(x - (quarter << 30)) * 1.4629180792671596e-09f /* 2 pi / 2^32 */, r2 = r * r;
    float s = fmaf(r2, 2.7557319e-6f /* 1 / 9! */, -1.9841270e-4f /* 1 / 7! */);
    s = fmaf(r2, s, 8.3333333e-3f /* 1 / 5! */);
    s = fmaf(r2, s, -1.6666667e-1f /* 1 / 3! */);
    s = fmaf(r * r2, s, r);
    float c = fmaf(r2, -2.7557319e-7f /* 1 / 10! */, 2.4801587e-5f /* 1 / 8! */);
    c = fmaf(r2, c, -1.3888889e-3f /* 1 / 6! */);
    c = fmaf(r2, c, 4.1666667e-2f /* 1 / 4! */);
    c = fmaf(r2, c, -0.5f);
    c = fmaf(r2, c, 1.f);
    const float a = p.none ? __uint_as_float(0x7fc00000u) : amplitude;
    const float cosine = (quarter & 1u ? s : c) * a, sine = (quarter & 1u ? c : s) * a;
    return make_float2(__uint_as_float(__float_as_uint(cosine) ^ ((quarter + 1u) >> 1 << 31)), __uint_as_float(__float_as_uint(sine) ^ (quarter >> 1 << 31)));
}

constexpr int kTableRows = 4;   // rows of a thread on their way at a time
// kCols neighbouring columns a thread (two where an axis has an even number of them: 16-byte stores).
template <int kCols>
__global__ void __launch_bounds__(kThreads)
rotary_table_kernel(const float* positions, const __grid_constant__ RotaryFrequencies freq, int64_t count, float2* table)
{
    const int32_t cols = freq.axes * freq.n, groups = cols / kCols, per_pass = kThreads / groups;
    const int32_t row0 = (int32_t)threadIdx.x / groups, col = ((int32_t)threadIdx.x - row0 * groups) * kCols;
    overlap_with_previous();
    if (row0 >= per_pass) return;
    const int32_t axis = col / freq.n;
    uint64_t turns[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) turns[c] = freq.turns[col - axis * freq.n + c];
    const int64_t step = (int64_t)gridDim.x * per_pass;
    for (int64_t row = (int64_t)blockIdx.x * per_pass + row0; row < count; row += kTableRows * step) {
        float pos[kTableRows];
#pragma unroll
        for (int i = 0; i < kTableRows; ++i) pos[i] = row + i * step < count ? load_float(positions + (row + i * step) * freq.axes + axis) : 0.f;
#pragma unroll
        for (int i = 0; i < kTableRows; ++i) {
            if (row + i * step >= count) break;
            const TableRow p(pos[i]);
            float2 e[kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c) e[c] = table_entry(p, turns[c], freq.amplitude);
            float2* dst = table + (row + i * step) * cols + col;
            if constexpr (kCols == 2) *reinterpret_cast<float4*>(dst) = make_float4(e[0].x, e[0].y, e[1].x, e[1].y);
            else dst[0] = e[0];
        }
    }
}

// ---------------------------------------------------------------- the rotation
// A thread turns two 16-byte pieces of the same token in kHeads heads, which share its 64 bytes of the table.  Half layout: a piece
// and its partner, half a part away (P a multiple of 16); interleaved: pieces u and u + units, each complete in itself (rotary_dim a
// multiple of 8).  What is not rotated is copied, two pieces a thread, unless the output is the input.
template <bool kInterleaved, int kHeads>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const __grid_constant__ RotaryArgs a, int32_t units)
{
    const uint32_t at = blockIdx.x * (uint32_t)kThreads + threadIdx.x, rt = at / (uint32_t)units;
    const int32_t unit = (int32_t)(at - rt * (uint32_t)units);
    const int64_t row = rt / (uint32_t)a.T;
    const int32_t t = (int32_t)(rt - (uint32_t)row * (uint32_t)a.T);
    if (row >= a.rows) return;
    const int32_t chunks = a.D / 8, cols = a.rotary_dim / 2;
    int32_t first, second, col_first, col_second;   // pieces (second may be behind the head's end), and their columns
    bool turn_first, turn_second;
    if (kInterleaved) {
        first = unit, second = unit + units;
        turn_first = first * 8 < a.rotary_dim, turn_second = second * 8 < a.rotary_dim;
        col_first = first * 4, col_second = second * 4;
    } else {
        const int32_t part = a.rotary_dim / a.axes / 16, pairs = part * a.axes;   // pieces in half a part; in half of all
        turn_first = turn_second = unit < pairs;
        const int32_t axis = unit / part, j = unit - axis * part, rest = 2 * pairs + 2 * (unit - pairs);
        first = turn_first ? axis * 2 * part + j : rest;
        second = turn_first ? first + part : rest + 1;
        col_first = unit * 8, col_second = col_first + 4;
    }
    overlap_with_previous();
    float4 cs[4];   // (cos, sin) of two pairs each
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = make_float4(1.f, 0.f, 1.f, 0.f);
    const int64_t n = a.index ? (int64_t)load_int(a.index + row * a.index_row + t) : a.first + t;
    if (n >= 0 && n < a.table_rows) {
        const float2* e = a.table + n * cols;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < 2 ? turn_first : turn_second)
                cs[i] = load_float4(e + (i < 2 ? col_first : col_second) + 2 * (i & 1));
    } else {
        // A token without a position keeps its channels, bit for bit: turned by an angle of 0 an infinity would make its partner not a
        // number, and a -0 would lose its sign.
        turn_first = turn_second = false;
    }
    const int32_t head0 = blockIdx.y * kHeads;
    uint4 x[kHeads][2];
    __nv_bfloat16* dst[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
        int32_t head = head0 + h;
        dst[h] = nullptr;
        const int which = head >= a.heads[0];
        if (which) head -= a.heads[0];
        if (head >= a.heads[which]) continue;
        const __nv_bfloat16* src = a.x[which] + row * a.x_row[which] + head * a.x_head[which] + t * a.x_tok[which];
        dst[h] = a.y[which] + row * a.y_row[which] + head * a.y_head[which] + t * a.y_tok[which];
        x[h][0] = load_16B(src + first * 8);
        if (second < chunks) x[h][1] = load_16B(src + second * 8);
    }
    auto turn = [&](uint32_t& u, uint32_t& w, const float4& v) {   // the pairs (u.lo, w.lo) and (u.hi, w.hi)
        const float u0 = __uint_as_float(u << 16), u1 = __uint_as_float(u & 0xffff0000u);
        const float w0 = __uint_as_float(w << 16), w1 = __uint_as_float(w & 0xffff0000u);
        const float s0 = a.direction * v.y, s1 = a.direction * v.w;
        const __nv_bfloat162 nu = __floats2bfloat162_rn(fmaf(u0, v.x, -(w0 * s0)), fmaf(u1, v.z, -(w1 * s1)));
        const __nv_bfloat162 nw = __floats2bfloat162_rn(fmaf(w0, v.x, u0 * s0), fmaf(w1, v.z, u1 * s1));
        u = *reinterpret_cast<const uint32_t*>(&nu);
        w = *reinterpret_cast<const uint32_t*>(&nw);
    };
    auto turn_inside = [&](uint32_t& p, const float c, const float sin) {   // the pair (p.lo, p.hi)
        const float u = __uint_as_float(p << 16), w = __uint_as_float(p & 0xffff0000u), s = a.direction * sin;
        const __nv_bfloat162 r = __floats2bfloat162_rn(fmaf(u, c, -(w * s)), fmaf(w, c, u * s));
        p = *reinterpret_cast<const uint32_t*>(&r);
    };
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
        if (!dst[h]) continue;
        uint4 &u = x[h][0], &w = x[h][1];
        if (kInterleaved) {
            if (turn_first) {
                turn_inside(u.x, cs[0].x, cs[0].y);
                turn_inside(u.y, cs[0].z, cs[0].w);
                turn_inside(u.z, cs[1].x, cs[1].y);
                turn_inside(u.w, cs[1].z, cs[1].w);
            }
            if (turn_second) {
                turn_inside(w.x, cs[2].x, cs[2].y);
                turn_inside(w.y, cs[2].z, cs[2].w);
                turn_inside(w.z, cs[3].x, cs[3].y);
                turn_inside(w.w, cs[3].z, cs[3].w);
            }
        } else if (turn_first) {
            turn(u.x, w.x, cs[0]);
            turn(u.y, w.y, cs[1]);
            turn(u.z, w.z, cs[2]);
            turn(u.w, w.w, cs[3]);
        }
        *reinterpret_cast<uint4*>(dst[h] + first * 8) = u;
        if (second < chunks) *reinterpret_cast<uint4*>(dst[h] + second * 8) = w;
    }
}

// Any shape: tokens go through shared memory, so that a thread, which writes eight channels, finds their partners wherever they are.
// Everything a block writes it has read before, so that the output may be the input.  What bounds it: an 8-byte load of the table per channel,
// which heads do not share, and two barriers per 4 KB.  16 rows x 32 heads x 4 096 x 128: 616 us with 120 channels turned by halves or
// 124 interleaved, where the kernel above takes 158 with 112, 120 (interleaved) or 128.
__global__ void __launch_bounds__(kThreads)
rotary_any_kernel(const __grid_constant__ RotaryArgs a)
{
    extern __shared__ __align__(16) __nv_bfloat16 held[];   // [tokens of a pass][D]
    const int32_t chunks = a.D / 8, per_pass = kThreads / chunks;
    const int32_t slot = (int32_t)threadIdx.x / chunks, chunk = (int32_t)threadIdx.x - slot * chunks;
    const int32_t P = a.rotary_dim / a.axes, cols = a.rotary_dim / 2;
    int32_t partner[8], column[8];
    float sign[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int32_t c = chunk * 8 + i, axis = c / P, r = c - axis * P;
        const bool second = a.interleaved ? (r & 1) != 0 : r >= P / 2;
        const int32_t away = a.interleaved ? 1 : P / 2;
        partner[i] = second ? c - away : c + away;
        column[i] = axis * (P / 2) + (a.interleaved ? r / 2 : (second ? r - P / 2 : r));
        sign[i] = second ? a.direction : -a.direction;
    }
    overlap_with_previous();
    const int64_t total = (int64_t)a.rows * (a.heads[0] + a.heads[1]) * a.T;
    for (int64_t base = (int64_t)blockIdx.x * per_pass; base < total; base += (int64_t)gridDim.x * per_pass) {
        const int64_t at = base + slot;
        const bool mine = slot < per_pass && at < total;
        const __nv_bfloat16* src = nullptr;
        __nv_bfloat16* dst = nullptr;
        int64_t row = 0;
        int32_t t = 0;
        __nv_bfloat16* own = held + slot * a.D + chunk * 8;
        if (mine) {
            const int64_t rh = at / a.T;
            t = (int32_t)(at - rh * a.T);
            row = rh / (a.heads[0] + a.heads[1]);
            int32_t head = (int32_t)(rh - row * (a.heads[0] + a.heads[1]));
            const int which = head >= a.heads[0];
            if (which) head -= a.heads[0];
            src = a.x[which] + row * a.x_row[which] + head * a.x_head[which] + t * a.x_tok[which] + chunk * 8;
            dst = a.y[which] + row * a.y_row[which] + head * a.y_head[which] + t * a.y_tok[which] + chunk * 8;
            *reinterpret_cast<uint4*>(own) = load_16B(src);
        }
        __syncthreads();
        if (mine) {
            const int64_t n = a.index ? (int64_t)load_int(a.index + row * a.index_row + t) : a.first + t;
            const bool turned = n >= 0 && n < a.table_rows;   // (a token without a position keeps its channels)
            const float2* cs = a.table + n * cols;
            __align__(16) __nv_bfloat162 out[4];   // (stored as one piece)
            __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(out);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                o[i] = own[i];
                if (turned && chunk * 8 + i < a.rotary_dim) {
                    const float2 v = load_float2(cs + column[i]);
                    o[i] = __float2bfloat16_rn(fmaf(__bfloat162float(own[i]), v.x, sign[i] * (__bfloat162float(held[slot * a.D + partner[i]]) * v.y)));
                }
            }
            *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<uint4*>(out);
        }
        __syncthreads();
    }
}

}  // namespace

cudaError_t launch_rotary_table(const float* positions, const RotaryFrequencies& freq, int64_t count, float2* table, int sm_count,
                                cudaStream_t stream)
{
    const int32_t wide = freq.n % 2 == 0 ? 2 : 1, per_pass = kThreads / (freq.axes * freq.n / wide);
    const int64_t blocks = std::min<int64_t>((count + per_pass - 1) / per_pass, 8ll * sm_count);
    return launch_kernel(true, wide == 2 ? rotary_table_kernel<2> : rotary_table_kernel<1>, dim3((unsigned)blocks), dim3(kThreads), KernelMemory(0),
                         stream, positions, freq, count, table);
}

cudaError_t launch_rotary(const RotaryArgs& a, int sm_count, cudaStream_t stream)
{
    const int32_t heads = a.heads[0] + a.heads[1], P = a.rotary_dim / a.axes;
    const bool in_place = a.x[0] == a.y[0] && (a.heads[1] == 0 || a.x[1] == a.y[1]);
    if (a.interleaved ? a.rotary_dim % 8 == 0 : P % 16 == 0) {
        const int32_t moved = in_place ? a.rotary_dim / 8 : a.D / 8, units = (moved + 1) / 2;   // pieces, two a thread
        const int64_t threads = (int64_t)a.rows * a.T * units, blocks = (threads + kThreads - 1) / kThreads;
        // Four heads a thread share their part of the table; one, where that would leave SMs with less than half of their threads.
        const bool four = threads * ((heads + 3) / 4) >= 1024ll * sm_count;
        const int32_t groups = four ? (heads + 3) / 4 : heads;
        if (threads <= 0xffffffffll - kThreads && groups <= 65535) {
            const dim3 grid((unsigned)blocks, (unsigned)groups);
            auto* kernel = a.interleaved ? (four ? rotary_kernel<true, 4> : rotary_kernel<true, 1>)
                                         : (four ? rotary_kernel<false, 4> : rotary_kernel<false, 1>);
            return launch_kernel(true, kernel, grid, dim3(kThreads), KernelMemory(0), stream, a, units);
        }
    }
    const int32_t per_pass = kThreads / (a.D / 8);
    const int64_t total = (int64_t)a.rows * heads * a.T;
    const int64_t blocks = std::min<int64_t>((total + per_pass - 1) / per_pass, 8ll * sm_count);
    return launch_kernel(true, rotary_any_kernel, dim3((unsigned)blocks), dim3(kThreads), KernelMemory((size_t)kThreads * 16), stream, a);
}

}  // namespace amskv
