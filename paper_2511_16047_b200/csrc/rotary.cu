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
// Entry (n, column) = (cos, sin) of positions[n][axis] * frequency, times the amplitude.  The angle is formed and reduced in 64 bits,
// in half turns (the host divides the frequencies by pi): at position 10^6 an fp32 angle would be off by 0.06.  What is left,
// within a quarter turn either way, is rounded to fp32 once (an angle error of 2^-26 pi) and goes through sincospif.
__global__ void __launch_bounds__(kThreads)
rotary_table_kernel(const float* positions, const __grid_constant__ RotaryFrequencies freq, int64_t count, float2* table)
{
    const int32_t cols = freq.axes * freq.n, per_pass = kThreads / cols;
    const int32_t row0 = (int32_t)threadIdx.x / cols, col = (int32_t)threadIdx.x - row0 * cols;
    overlap_with_previous();
    if (row0 >= per_pass) return;
    const int32_t axis = col / freq.n;
    const double half_turns = freq.half_turns[col - axis * freq.n];
    for (int64_t row = (int64_t)blockIdx.x * per_pass + row0; row < count; row += (int64_t)gridDim.x * per_pass) {
        const double t = (double)load_float(positions + row * freq.axes + axis) * half_turns;
        const double f = fma(-2.0, rint(0.5 * t), t), n = rint(f);   // f in [-1, 1]
        float s, c;
        sincospif((float)(f - n), &s, &c);
        const float a = n != 0.0 ? -freq.amplitude : freq.amplitude;
        table[row * cols + col] = make_float2(c * a, s * a);
    }
}

// ---------------------------------------------------------------- the rotation
// Any shape: tokens go through shared memory, so that a thread, which writes eight channels, finds their partners wherever they are.
// Everything a block writes it has read before, so that the output may be the input.
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
            __nv_bfloat162 out[4];
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
    const int32_t per_pass = kThreads / (freq.axes * freq.n);
    const int64_t blocks = std::min<int64_t>((count + per_pass - 1) / per_pass, 8ll * sm_count);
    return launch_kernel(true, rotary_table_kernel, dim3((unsigned)blocks), dim3(kThreads), KernelMemory(0), stream, positions, freq,
                         count, table);
}

cudaError_t launch_rotary(const RotaryArgs& a, int sm_count, cudaStream_t stream)
{
    const int32_t per_pass = kThreads / (a.D / 8);
    const int64_t total = (int64_t)a.rows * (a.heads[0] + a.heads[1]) * a.T;
    const int64_t blocks = std::min<int64_t>((total + per_pass - 1) / per_pass, 8ll * sm_count);
    return launch_kernel(true, rotary_any_kernel, dim3((unsigned)blocks), dim3(kThreads), KernelMemory((size_t)kThreads * 16), stream, a);
}

}  // namespace amskv
