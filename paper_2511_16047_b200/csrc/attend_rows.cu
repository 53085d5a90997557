// Attention with warp-level matrix instructions over an encoder's states or a region held in 8 bits: calls of few queries, or of few
// items, where a 128-row tile of the tensor-memory kernel (attend_tiles.cu) would be mostly empty.
//
// The query rows of a key/value head are those of all query heads that share it, one head behind the other: a few queries in each
// of four heads fill one 16-row block and read the keys once.  A CTA of four warps (eight) takes kQB (1, 2, 4) such blocks and gives each
// kWarps / kQB warps, which share a chunk's 64 keys; a cluster of up to eight CTAs shares the keys of a call with few rows and many keys.
// Every warp keeps its own reference maximum, sum and products; they are put together once at the end, through (distributed) shared
// memory, without atomics, so that results are the same each time.
//
// An encoder's chunks come by 16-byte asynchronous copies, kStages - 1 ahead, with zeros behind a row's last key (what lies there
// in memory may be anything and is not read).  Codes of 8 bits are fetched into registers a chunk ahead and widened to bf16, which
// holds them and their powers of two exactly, on the way to shared memory.  From there on both are the same.
#include <cstring>

#include "keys.cuh"
#include "sm100_ptx.cuh"

namespace amskv {

namespace {

constexpr int kChunk = 64;                 // keys of a stage
constexpr float kRescaleLog2 = 8.f;        // a reference maximum moves when a chunk exceeds it by 2^8

template <int D, bool kHeld, int kWarps>
struct RowsCfg {
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kStages = kHeld ? 2 : 3;
    static constexpr int kRowBytes = D * 2;
    static constexpr int kTileBytes = kChunk * kRowBytes;
    static constexpr int kStageBytes = 2 * kTileBytes;
    static constexpr int kPartRow = D + 8;                                  // floats; shifts the banks of a row by 8
    static constexpr int kPartBytes = 16 * kPartRow * 4;                    // products of a warp's 16 rows
    static constexpr int kStatsAt = kWarps * kPartBytes;                    // maxima and sums of the rows behind them
    static constexpr int kPartsEnd = kStatsAt + 2 * kWarps * 16 * 8;        // the parts take the place of the stages
    static constexpr int kSmemBytes = kStages * kStageBytes > kPartsEnd ? kStages * kStageBytes : kPartsEnd;
};

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float4 ld_cluster_16B(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 ld_cluster_8B(uint32_t addr)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

// Codes of one chunk on their way: a thread's 16-byte pieces of K and V, and the scale words of their blocks.
template <int D, int kThreads>
struct HeldPieces {
    static constexpr int kPieces = D / 16, kRows = kThreads / kPieces, kN = kChunk / kRows;   // pieces of a row, rows of a pass, passes
    uint4 k[kN], v[kN];
    uint32_t scale[kN];
};

template <int D, int kQB, bool kHeld, int kWarps>
__global__ void __launch_bounds__(kWarps * 32, (D == 64 ? 16 : 8) / kWarps)
attend_rows_kernel(const __nv_bfloat16* Q, int64_t q_row, int64_t q_head, int64_t q_tok, __nv_bfloat16* O, int64_t o_row, int64_t o_head,
                   int64_t o_tok, const __grid_constant__ EncoderKeys enc, const __grid_constant__ HeldKeys held, int32_t T,
                   int32_t kv_heads, int32_t group, int32_t parts, int32_t splits, float scale_log2)
{
    using C = RowsCfg<D, kHeld, kWarps>;
    constexpr int kThreads = C::kThreads;
    constexpr int kKS = kWarps / kQB;                       // warps that share a chunk's keys
    constexpr int kWarpKeys = kChunk / kKS, kTiles = kWarpKeys / 8, kBlocks = kWarpKeys / kBlock;
    constexpr int kPieces = D / 32;                         // 16-byte pieces of a row per lane, in fragment order
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t smem0 = ptx::smem_u32(smem);
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int g = lane >> 2, q = lane & 3, ks = warp % kKS, qb = warp / kKS;
    const int32_t rank = (int32_t)blockIdx.x % splits;
    int32_t item = (int32_t)blockIdx.x / splits;
    const int32_t part = item % parts;
    item /= parts;
    const int32_t row = item / kv_heads, kv_head = item - row * kv_heads;
    const int32_t M = T * group;                            // query rows of this key/value head
    const int32_t m0 = (part * kQB + qb) * 16;
    const bool live = m0 < M;
    // query row m: token m % T of head m / T of the group
    auto row_offset = [&](int32_t m, int64_t head_stride, int64_t tok_stride) -> int64_t {
        const int32_t h = m / T;
        return (int64_t)(kv_head * group + h) * head_stride + (int64_t)(m - h * T) * tok_stride;
    };
    const __nv_bfloat16* qbase = Q + row * q_row;
    const uint4* q0 = reinterpret_cast<const uint4*>(qbase + row_offset(min(m0 + g, M - 1), q_head, q_tok) + 8 * q);
    const uint4* q1 = reinterpret_cast<const uint4*>(qbase + row_offset(min(m0 + g + 8, M - 1), q_head, q_tok) + 8 * q);
    overlap_with_previous();
    EncoderView ev(enc, row, kv_head, EncoderBounds(enc, row));
    HeldView hv(held, item, D);
    const int32_t blocks = kHeld ? hv.blocks() : ev.blocks();
    // this CTA's chunks
    const int32_t all = (blocks + kChunk / kBlock - 1) / (kChunk / kBlock), share = (all + splits - 1) / splits;
    const int32_t c0 = min(rank * share, all), c1 = min(c0 + share, all);

    uint4 qa0[kPieces], qa1[kPieces];
#pragma unroll
    for (int h = 0; h < kPieces; ++h) {
        qa0[h] = load_16B(q0 + 4 * h);
        qa1[h] = load_16B(q1 + 4 * h);
    }

    // ---- an encoder's keys: copies
    constexpr int kTokPieces = D / 8, kStep = kThreads / kTokPieces;   // 16-byte pieces of a token; tokens a pass of all threads covers
    const int cp_piece = (int)threadIdx.x % kTokPieces, cp_row = (int)threadIdx.x / kTokPieces;
    static_assert(kStep % 8 == 0, "a thread's rows share their swizzle");
    auto copy_chunk = [&](int32_t c) {
        const uint32_t st = smem0 + (uint32_t)(c % C::kStages) * C::kStageBytes;
#pragma unroll
        for (int i = 0; i < kChunk / kStep; ++i) {
            const int r = cp_row + i * kStep;
            const int32_t key = c * kChunk + r;
            const bool real = key < ev.len;
            const int64_t at = (real ? (int64_t)key * ev.tok : 0) + cp_piece * 8;
            copy16_or_zero(st + r * C::kRowBytes + ((cp_piece ^ ((r & 1) << 2)) << 4), ev.k + at, real);
            copy16_or_zero(st + C::kTileBytes + r * C::kRowBytes + ((cp_piece ^ (r & 7)) << 4), ev.v + at, real);
        }
    };
    // ---- codes: fetch, then widen into a stage
    using Pieces = HeldPieces<D, kThreads>;
    Pieces next;
    const int w_piece = (int)threadIdx.x % Pieces::kPieces, w_row = (int)threadIdx.x / Pieces::kPieces;
    HeldView fetch = hv;
    auto fetch_chunk = [&](int32_t c) {
#pragma unroll
        for (int i = 0; i < Pieces::kN; ++i) {
            const int r = w_row + i * Pieces::kRows;
            const int32_t b = c * (kChunk / kBlock) + r / kBlock, slot = r % kBlock;
            next.k[i] = next.v[i] = make_uint4(0, 0, 0, 0);
            next.scale[i] = 0;
            if (slot < fetch.valid(b)) {
                const int32_t pos = fetch.position(b);
                const uint8_t* src = fetch.codes + (int64_t)(pos + slot) * D + w_piece * 16;
                next.k[i] = load_16B(src);
                next.v[i] = load_16B(src + (int64_t)fetch.capacity * D);
                next.scale[i] = load_word(fetch.scales + pos / kBlock);
            }
        }
    };
    auto widen_chunk = [&](int32_t c) {
        uint8_t* st = smem + (c % C::kStages) * C::kStageBytes;
#pragma unroll
        for (int i = 0; i < Pieces::kN; ++i) {
            const int r = w_row + i * Pieces::kRows;
            uint4 lo, hi;
            widen16_by(next.k[i], next.scale[i], false, lo, hi);
            uint8_t* kt = st + r * C::kRowBytes;
            *reinterpret_cast<uint4*>(kt + (((2 * w_piece) ^ ((r & 1) << 2)) << 4)) = lo;
            *reinterpret_cast<uint4*>(kt + (((2 * w_piece + 1) ^ ((r & 1) << 2)) << 4)) = hi;
            widen16_by(next.v[i], next.scale[i], true, lo, hi);
            uint8_t* vt = st + C::kTileBytes + r * C::kRowBytes;
            *reinterpret_cast<uint4*>(vt + (((2 * w_piece) ^ (r & 7)) << 4)) = lo;
            *reinterpret_cast<uint4*>(vt + (((2 * w_piece + 1) ^ (r & 7)) << 4)) = hi;
        }
    };

    if (kHeld) {
        if (c0 < c1) fetch_chunk(c0);
    } else {
#pragma unroll 1
        for (int i = 0; i < C::kStages - 1; ++i) {
            if (c0 + i < c1) copy_chunk(c0 + i);
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    }

    float o[D / 8][4];
#pragma unroll
    for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    float m_a = -INFINITY, m_b = -INFINITY, nb_a = 0.f, nb_b = 0.f, l_a = 0.f, l_b = 0.f;

#pragma unroll 1
    for (int32_t c = c0; c < c1; ++c) {
        if (kHeld) {
            // (the stage was read two chunks ago, before the barrier of the chunk between)
            widen_chunk(c);
            if (c + 1 < c1) fetch_chunk(c + 1);
        } else {
            asm volatile("cp.async.wait_group %0;" ::"n"(C::kStages - 2) : "memory");
        }
        __syncthreads();
        if (!kHeld) {
            if (c + C::kStages - 1 < c1) copy_chunk(c + C::kStages - 1);   // into the stage of the chunk before, which all have left
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        const int32_t block0 = c * (kChunk / kBlock) + ks * kBlocks;
        if (!live || block0 >= blocks) continue;
        const uint32_t stage = (uint32_t)(c % C::kStages) * C::kStageBytes;
        const uint8_t* kt = smem + stage + (ks * kWarpKeys + g) * C::kRowBytes;
        const int kx = (q ^ ((g & 1) << 2)) << 4;
        float s[kTiles][4];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
#pragma unroll
            for (int h = 0; h < kPieces; ++h) {
                const uint4 kk = *reinterpret_cast<const uint4*>(kt + t * 8 * C::kRowBytes + (kx ^ (h << 6)));
                mma_16816(s[t], qa0[h].x, qa1[h].x, qa0[h].y, qa1[h].y, kk.x, kk.y);
                mma_16816(s[t], qa0[h].z, qa1[h].z, qa0[h].w, qa1[h].w, kk.z, kk.w);
            }
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const int32_t valid = kHeld ? hv.valid(block0 + b) : ev.valid(block0 + b);
            if (valid == kBlock) continue;
#pragma unroll
            for (int t = 2 * b; t < 2 * b + 2; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if ((t & 1) * 8 + 2 * q + e >= valid) s[t][e] = s[t][2 + e] = -INFINITY;
        }
        float mx_a = fmaxf(s[0][0], s[0][1]), mx_b = fmaxf(s[0][2], s[0][3]);
#pragma unroll
        for (int t = 1; t < kTiles; ++t) {
            mx_a = ptx::max3(mx_a, s[t][0], s[t][1]);
            mx_b = ptx::max3(mx_b, s[t][2], s[t][3]);
        }
        mx_a = fmaxf(mx_a, __shfl_xor_sync(0xffffffffu, mx_a, 1));
        mx_b = fmaxf(mx_b, __shfl_xor_sync(0xffffffffu, mx_b, 1));
        mx_a = fmaxf(mx_a, __shfl_xor_sync(0xffffffffu, mx_a, 2));
        mx_b = fmaxf(mx_b, __shfl_xor_sync(0xffffffffu, mx_b, 2));
        // (the first block of the chunk holds a key, so that the first chunk always moves the reference from minus infinity)
        const bool grow_a = (mx_a - m_a) * scale_log2 > kRescaleLog2, grow_b = (mx_b - m_b) * scale_log2 > kRescaleLog2;
        if (__any_sync(0xffffffffu, grow_a || grow_b)) {
            const float f_a = grow_a ? fast_exp2((m_a - mx_a) * scale_log2) : 1.f, f_b = grow_b ? fast_exp2((m_b - mx_b) * scale_log2) : 1.f;
            if (grow_a) { m_a = mx_a; nb_a = -mx_a * scale_log2; }
            if (grow_b) { m_b = mx_b; nb_b = -mx_b * scale_log2; }
            l_a *= f_a;
            l_b *= f_b;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) {
                o[n][0] *= f_a;
                o[n][1] *= f_a;
                o[n][2] *= f_b;
                o[n][3] *= f_b;
            }
        }
        const int vkey = ks * kWarpKeys + (lane & 15);
        const uint32_t vt = smem0 + stage + C::kTileBytes + (uint32_t)vkey * C::kRowBytes;
        const uint32_t vx = (uint32_t)(((lane >> 4) ^ (vkey & 7)) << 4);
#pragma unroll
        for (int step = 0; step < kTiles / 2; ++step) {
            uint32_t p[4];   // rounded to bf16 for the product, the type of V; the sums take them as they are
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float (&x)[4] = s[2 * step + u];
                x[0] = fast_exp2(fmaf(x[0], scale_log2, nb_a));
                x[1] = fast_exp2(fmaf(x[1], scale_log2, nb_a));
                x[2] = fast_exp2(fmaf(x[2], scale_log2, nb_b));
                x[3] = fast_exp2(fmaf(x[3], scale_log2, nb_b));
                l_a += x[0] + x[1];
                l_b += x[2] + x[3];
                p[2 * u] = pack_bf16(x[0], x[1]);
                p[2 * u + 1] = pack_bf16(x[2], x[3]);
            }
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                uint32_t v[4];
                ldmatrix_x4_trans(v, vt + step * 16 * C::kRowBytes + ((uint32_t)(j << 5) ^ vx));
                mma_16816(o[2 * j], p[0], p[1], p[2], p[3], v[0], v[1]);
                mma_16816(o[2 * j + 1], p[0], p[1], p[2], p[3], v[2], v[3]);
            }
        }
    }
    l_a += __shfl_xor_sync(0xffffffffu, l_a, 1);
    l_b += __shfl_xor_sync(0xffffffffu, l_b, 1);
    l_a += __shfl_xor_sync(0xffffffffu, l_a, 2);
    l_b += __shfl_xor_sync(0xffffffffu, l_b, 2);

    // ---- the parts of all warps of the cluster that had some of a block's keys
    if (!kHeld) asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();   // the stages are free
    float* own = reinterpret_cast<float*>(smem + warp * C::kPartBytes);
    float2* stats = reinterpret_cast<float2*>(smem + C::kStatsAt) + warp * 16;
#pragma unroll
    for (int n = 0; n < D / 8; ++n) {
        *reinterpret_cast<float2*>(own + g * C::kPartRow + 8 * n + 2 * q) = make_float2(o[n][0], o[n][1]);
        *reinterpret_cast<float2*>(own + (g + 8) * C::kPartRow + 8 * n + 2 * q) = make_float2(o[n][2], o[n][3]);
    }
    if (q == 0) {
        stats[g] = make_float2(m_a, l_a);
        stats[g + 8] = make_float2(m_b, l_b);
    }
    __syncthreads();
    // the parts of this CTA's warps, eight channels of a row at a time, into the place of the first (or out)
    const float2* all_stats = reinterpret_cast<const float2*>(smem + C::kStatsAt);
    constexpr int32_t kPieceRounds = kQB * 16 * (D / 8) / kThreads;
#pragma unroll
    for (int32_t i = 0; i < kPieceRounds; ++i) {
        if (kKS == 1 && splits > 1) break;   // (a row has one part already)
        const int32_t at = i * kThreads + threadIdx.x, r = at / (D / 8), c = at % (D / 8) * 8, w0 = r / 16 * kKS;   // row among the CTA's kQB x 16
        float2 ml[kKS];
        float top = -INFINITY;
#pragma unroll
        for (int n = 0; n < kKS; ++n) {
            ml[n] = all_stats[(w0 + n) * 16 + r % 16];
            top = fmaxf(top, ml[n].x);
        }
        float l = 0.f, acc[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.f;
        float* first = reinterpret_cast<float*>(smem + w0 * C::kPartBytes) + r % 16 * C::kPartRow + c;
#pragma unroll
        for (int n = 0; n < kKS; ++n) {
            const float f = top == -INFINITY ? 0.f : fast_exp2((ml[n].x - top) * scale_log2);   // (a row without a key: zeros)
            l = fmaf(ml[n].y, f, l);
            const float4 x = *reinterpret_cast<const float4*>(first + n * (C::kPartBytes / 4)), y = *reinterpret_cast<const float4*>(first + n * (C::kPartBytes / 4) + 4);
            acc[0] = fmaf(x.x, f, acc[0]);
            acc[1] = fmaf(x.y, f, acc[1]);
            acc[2] = fmaf(x.z, f, acc[2]);
            acc[3] = fmaf(x.w, f, acc[3]);
            acc[4] = fmaf(y.x, f, acc[4]);
            acc[5] = fmaf(y.y, f, acc[5]);
            acc[6] = fmaf(y.z, f, acc[6]);
            acc[7] = fmaf(y.w, f, acc[7]);
        }
        if (splits == 1) {
            const int32_t m = part * kQB * 16 + r;
            if (m < M) {
                const float inv = l > 0.f ? 1.f / l : 0.f;
                *reinterpret_cast<uint4*>(O + row * o_row + row_offset(m, o_head, o_tok) + c) =
                    make_uint4(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv),
                               pack_bf16(acc[4] * inv, acc[5] * inv), pack_bf16(acc[6] * inv, acc[7] * inv));
            }
        } else {
            *reinterpret_cast<float4*>(first) = make_float4(acc[0], acc[1], acc[2], acc[3]);
            *reinterpret_cast<float4*>(first + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
            // the row's maximum and sum, beside the parts' (which other threads may still read)
            if (c == 0) reinterpret_cast<float2*>(smem + C::kStatsAt)[kWarps * 16 + r] = make_float2(top, l);
        }
    }
    if (splits == 1) return;
    // the parts of the cluster's CTAs: each finishes its share of the channels, kWide at a time, and asks for all parts before it uses one
    ptx::cluster_sync();
    constexpr int kMaxSplits = 8, kWide = kQB == 4 ? 8 : 4;
    const uint32_t stats_at = smem0 + C::kStatsAt + (kKS == 1 ? 0 : kWarps * 16 * 8);
    const int32_t pieces = D / kWide / splits;
    for (int32_t i = threadIdx.x; i < kQB * 16 * pieces; i += kThreads) {
        const int32_t r = i / pieces, c = (rank * pieces + i - r * pieces) * kWide, m = part * kQB * 16 + r;
        if (m >= M) continue;
        float2 ml[kMaxSplits];
        float4 x[kMaxSplits][kWide / 4];
        float top = -INFINITY;
#pragma unroll
        for (int n = 0; n < kMaxSplits; ++n)
            if (n < splits) {
                ml[n] = ld_cluster_8B(ptx::map_to_rank(stats_at + r * 8, n));
                const uint32_t from = ptx::map_to_rank(smem0 + r / 16 * kKS * C::kPartBytes + (r % 16 * C::kPartRow + c) * 4, n);
#pragma unroll
                for (int e = 0; e < kWide / 4; ++e) x[n][e] = ld_cluster_16B(from + 16 * e);
            }
#pragma unroll
        for (int n = 0; n < kMaxSplits; ++n)
            if (n < splits) top = fmaxf(top, ml[n].x);
        float l = 0.f, acc[kWide];
#pragma unroll
        for (int e = 0; e < kWide; ++e) acc[e] = 0.f;
#pragma unroll
        for (int n = 0; n < kMaxSplits; ++n)
            if (n < splits) {
                const float f = top == -INFINITY ? 0.f : fast_exp2((ml[n].x - top) * scale_log2);
                l = fmaf(ml[n].y, f, l);
#pragma unroll
                for (int e = 0; e < kWide / 4; ++e) {
                    acc[4 * e] = fmaf(x[n][e].x, f, acc[4 * e]);
                    acc[4 * e + 1] = fmaf(x[n][e].y, f, acc[4 * e + 1]);
                    acc[4 * e + 2] = fmaf(x[n][e].z, f, acc[4 * e + 2]);
                    acc[4 * e + 3] = fmaf(x[n][e].w, f, acc[4 * e + 3]);
                }
            }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        uint2* dst = reinterpret_cast<uint2*>(O + row * o_row + row_offset(m, o_head, o_tok) + c);
#pragma unroll
        for (int e = 0; e < kWide / 4; ++e)
            dst[e] = make_uint2(pack_bf16(acc[4 * e] * inv, acc[4 * e + 1] * inv), pack_bf16(acc[4 * e + 2] * inv, acc[4 * e + 3] * inv));
    }
    ptx::cluster_sync();   // nobody's parts go while another reads them
}

template <int D, int kQB, bool kHeld, int kWarps = 4>
cudaError_t launch(const Strided& Q, const Strided& O, const EncoderKeys& enc, const HeldKeys& held, int32_t T, int32_t rows,
                   int32_t kv_heads, int32_t group, int64_t max_keys, float scale_log2, int sm_count, bool fixed_form, cudaStream_t stream)
{
    using C = RowsCfg<D, kHeld, kWarps>;
    static SharedMemoryOptIn opt_in;
    const cudaError_t oe = opt_in.ensure(attend_rows_kernel<D, kQB, kHeld, kWarps>, C::kSmemBytes);
    if (oe != cudaSuccess) return oe;
    const int64_t blocks = ((int64_t)T * group + 15) / 16, parts = (blocks + kQB - 1) / kQB, ctas = parts * rows * kv_heads;
    // Few CTAs and several chunks of keys: clusters share them.  What a merge costs is about four chunks of an encoder's keys or
    // two of codes (256 keys in four chunks, shared by two CTAs / not: 64 channels 5.4 / 4.6, 128 channels 7.5 / 6.7 us;
    // 484 keys 6.2 / 6.7 and 9.0 / 9.8; 8 bits, 64 channels, 256 keys 6.2 / 7.6).
    constexpr int kFirst = kHeld ? 4 : 8, kMore = 4;
    const int64_t chunks = (max_keys + kChunk - 1) / kChunk;
    int32_t splits = 1;
    const int64_t slots = kWarps == 8 && D == 128 ? sm_count : 2ll * sm_count;   // (a CTA of eight warps of 128 channels has an SM's registers)
    while (!fixed_form && splits < 8 && ctas * splits * 2 <= slots && chunks >= (splits == 1 ? kFirst : splits * kMore)) splits *= 2;
    if (ctas * splits > 0x7fffffffll) return cudaErrorInvalidValue;
    // Behind an append, CTAs that are more than the SMs but do not fill them spread evenly over an idle chip, not over SMs that come free one
    // by one: not overlapped with the launch before (64 channels: 128 items, T = 100 22 us, 19; 32 items, T = 400 43, 37).  An encoder's
    // calls have no append before them and keep the 0.2 to 0.5 us of the overlap.
    const int64_t grid = ctas * splits;
    const bool uneven = kHeld && grid > sm_count && grid < (D == 64 ? 16 : 8) / kWarps * (int64_t)sm_count;
    return launch_kernel(!uneven, attend_rows_kernel<D, kQB, kHeld, kWarps>, dim3((unsigned)grid), dim3(C::kThreads),
                         KernelMemory(C::kSmemBytes, (unsigned)splits), stream, (const __nv_bfloat16*)Q.ptr, Q.row, Q.head, Q.token,
                         (__nv_bfloat16*)O.ptr, O.row, O.head, O.token, enc, held, T, kv_heads, group, (int32_t)parts, splits, scale_log2);
}

template <bool kHeld>
cudaError_t launch_any(const Strided& Q, const Strided& O, const EncoderKeys& enc, const HeldKeys& held, int32_t T, int32_t rows,
                       int32_t kv_heads, int32_t group, int32_t D, int64_t max_keys, float softmax_scale, int sm_count, bool fixed_form,
                       cudaStream_t stream)
{
    const int64_t M = (int64_t)T * group;
    if (T < 1 || M > 0x7fffffff - 128 || (int64_t)rows * kv_heads > 0x7fffffffll) return cudaErrorInvalidValue;
    const float scale_log2 = softmax_scale * 1.4426950408889634f;
#define AMSKV_ROWS_LAUNCH(DD, QB) \
    return launch<DD, QB, kHeld>(Q, O, enc, held, T, rows, kv_heads, group, max_keys, scale_log2, sm_count, fixed_form, stream)
    // 16-row blocks of a CTA: one while all CTAs run at once (with codes, which every CTA widens for itself, fewer of them the more keys
    // there are), two likewise, else four.
    // us per call with one / two / four: 16 items, T = 36, 64 keys: 64 channels 2.6 / 3.1 / 3.6, 128 channels 3.4 / 3.9 / 4.6;
    // 32 items, T = 144, 484 keys: 6.7 / 8.2 / 10.0, 9.7 / 12.8 / 14.2;  64 items, T = 100, 256 keys: 6.5 / 5.7 / 6.4, 11.7 / 8.5 / 9.0;
    // 128 items, T = 144, 256 keys: 11.8 / 11.1 / 12.3.
    // 8 bits, with one / four blocks and eight warps: 16 items, T = 100, 164 keys 4.9 / 5.9 and 6.9 / 8.6, 584 keys 9.5 / 9.6 and 14.5 / 12.6;
    // 32 items, T = 36, 520 keys 9.6 / 8.9 and 14.4 / 11.3, 1 060 keys 13.6 / 12.1 and 21.2 / 14.4.
    // A fixed form does without all that depends on the number of items, which decides in what order keys are summed up.
    const int64_t blocks = (M + 15) / 16, items = (int64_t)rows * kv_heads;
    const int64_t ones = !kHeld ? 2ll * sm_count : D == 64 ? (max_keys <= 512 ? 2ll : 1ll) * sm_count : max_keys <= 448 ? sm_count : sm_count / 2;
    const int qb = blocks == 1 || (!fixed_form && items * blocks <= ones) ? 1 : blocks == 2 || (!kHeld && !fixed_form && items * ((blocks + 1) / 2) <= 2ll * sm_count) ? 2 : 4;
    // Codes: twice the warps, which widen them twice as fast, where all CTAs have an SM of their own (64 items, T = 100, 64 keys 7.2 us with
    // four warps, 5.9 with eight, 128 channels 10.8, 8.7; 128 items, T = 64, 1 088 keys 21.5, 19.5, 128 channels, 484 keys 21.2, 18.7).
    const bool eight = kHeld && !fixed_form && qb == 4 && items * ((blocks + 3) / 4) <= sm_count;
    if (D == 64) {
        if constexpr (kHeld)
            if (eight) return launch<64, 4, kHeld, 8>(Q, O, enc, held, T, rows, kv_heads, group, max_keys, scale_log2, sm_count, fixed_form, stream);
        if (qb == 1) AMSKV_ROWS_LAUNCH(64, 1);
        if (qb == 2) AMSKV_ROWS_LAUNCH(64, 2);
        AMSKV_ROWS_LAUNCH(64, 4);
    }
    if constexpr (kHeld)
        if (eight) return launch<128, 4, kHeld, 8>(Q, O, enc, held, T, rows, kv_heads, group, max_keys, scale_log2, sm_count, fixed_form, stream);
    if (qb == 1) AMSKV_ROWS_LAUNCH(128, 1);
    if (qb == 2) AMSKV_ROWS_LAUNCH(128, 2);
    AMSKV_ROWS_LAUNCH(128, 4);
#undef AMSKV_ROWS_LAUNCH
}

}  // namespace

cudaError_t launch_attend_rows(const Strided& Q, const Strided& O, const EncoderKeys& enc, int32_t T, int32_t rows, int32_t kv_heads,
                               int32_t group, int32_t D, float softmax_scale, int sm_count, bool fixed_form, cudaStream_t stream)
{
    HeldKeys none;
    memset(&none, 0, sizeof(none));
    return launch_any<false>(Q, O, enc, none, T, rows, kv_heads, group, D, enc.max_keys, softmax_scale, sm_count, fixed_form, stream);
}

cudaError_t launch_attend_rows(const Strided& Q, const Strided& O, const HeldKeys& held, int32_t T, int32_t rows, int32_t heads,
                               int32_t D, float softmax_scale, int sm_count, bool fixed_form, cudaStream_t stream)
{
    EncoderKeys none;
    memset(&none, 0, sizeof(none));
    if (held.ranges.n < 1 || held.blocks < 1) return cudaErrorInvalidValue;
    return launch_any<true>(Q, O, none, held, T, rows, heads, 1, D, (int64_t)held.blocks * kBlock, softmax_scale, sm_count, fixed_form,
                            stream);
}

}  // namespace amskv
