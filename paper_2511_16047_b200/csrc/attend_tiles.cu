// Attention over an encoder's states or a region held in 8 bits on the tensor cores: both products are tcgen05 instructions with their
// accumulators in tensor memory.  Calls of few queries or items take the warp-matrix kernel (attend_rows.cu).
//
// A CTA per SM walks units of two streams, each a (query head, tile of 128 queries) of the same row, and so with as many keys.  Two
// streams of one key/value head (two tiles of a head, or heads of a group) share every tile of 64 keys in shared memory; others
// have tiles of their own, which alternate.
//   warps 0-3, 4-7   softmax of stream A, of stream B: a query row per thread (row = TMEM lane)
//   warps 8, 9       issue the products of stream A, of stream B
//   warps 10-13      fill the ring of key/value stages
// Per tile: S = Q K^T (128 x 64 fp32, two buffers per stream, so that S of the next tile is formed while the softmax of this one
// runs); the softmax warps exponentiate in base 2 against a reference maximum and write P as bf16 over S; O += P V with P from tensor
// memory.  The reference is the maximum of the first tile; O and the sums are rescaled only when a later one exceeds it by 2^8.
// Why not the bulk copies of the paired kernel (attend_pair.cu): keys behind a row's last one may be anything, NaN among them, and
// a product with a zero probability would spread it, so that the tail has to arrive as zeros, at an end that only the device
// knows; and codes of 8 bits have to pass through registers to become bf16.  Four warps with 16-byte asynchronous copies (zeros
// where there is no key), or with loads a tile ahead, have room beside eight softmax warps, which is what binds a unit.
// Every wait is bounded: one that gives up records a status code and sets a flag, its role stops, and so do the others at their
// next wait.  Copies and products still under way are then awaited, and the tensor memory is freed.
#include <algorithm>
#include <cstring>

#include "keys.cuh"
#include "sm100_ptx.cuh"

namespace amskv {

namespace {

using namespace ptx;

constexpr int kQRows = 128;       // query rows per tile = TMEM lanes
constexpr int kQBoxRows = 32;     // query rows per bulk copy
constexpr int kKT = 64;           // keys per tile
constexpr int kTileBlocks = kKT / kBlock;
constexpr int kStages = 4;
constexpr int kGroupWarps = 4;
constexpr int kMmaWarp = 8, kLoadWarp = 10, kLoadWarps = 4, kLoadThreads = kLoadWarps * 32;
constexpr int kThreads = (kLoadWarp + kLoadWarps) * 32;
constexpr float kRescaleLog2 = 8.f;
constexpr int kPolyEvery = 6;     // every 6th pair of exponentials from the FMA pipe, as in the paired kernel

template <int D>
struct TilesCfg {
    static constexpr int kHalves = D / 64;                      // 128-byte swizzle atoms per row
    static constexpr uint32_t kQBytes = kQRows * D * 2, kQHalfBytes = kQRows * 128;
    static constexpr uint32_t kKVBytes = kKT * D * 2, kKVHalfBytes = kKT * 128;
    static constexpr uint32_t kStageBytes = 2 * kKVBytes;
    static constexpr uint32_t kTileBytes = 2 * kQBytes + kStages * kStageBytes;
    static constexpr uint32_t kSmemBytes = 2048 + kTileBytes;   // barriers and alignment slack in front
    static constexpr uint32_t kTmemCols = 512, kSCol = 0, kOCol = 4 * kKT;   // two S buffers of both streams, then O of both
    static_assert(kOCol + 2 * D <= kTmemCols, "tensor memory");
    static_assert(kSmemBytes <= 227 * 1024, "shared memory");
    static_assert(kKVHalfBytes % 1024 == 0 && kQHalfBytes % 1024 == 0, "swizzle atoms stay 1024-byte aligned");
};

struct Barriers {
    uint64_t q_full[2], kv_full[kStages], kv_empty[kStages], s_full[2][2], p_full[2][2], pv_done[2], o_full[2], drained[2];
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(Barriers) + 1024 <= 2048, "barriers fit in front of the aligned tiles");

struct TilePlan {
    int32_t nqt, heads, group, units_per_row;   // query tiles per head; query heads; of them per key/value head; ceil(nqt * heads / 2)
    int64_t units;
};
// Unit n: streams 2 u and 2 u + 1 of its row's nqt * heads.
struct Unit {
    int32_t row, head[2], qt[2];
    bool two, shared;

    __device__ __forceinline__ Unit(const TilePlan& p, int64_t n)
    {
        row = (int32_t)(n / p.units_per_row);
        const int32_t s = 2 * (int32_t)(n - (int64_t)row * p.units_per_row);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            head[g] = (s + g) / p.nqt;
            qt[g] = s + g - head[g] * p.nqt;
        }
        two = head[1] < p.heads;
        shared = two && head[0] / p.group == head[1] / p.group;
    }
};

template <int D, bool kHeld>
__global__ void __launch_bounds__(kThreads, 1)
attend_tiles_kernel(const __grid_constant__ CUtensorMap q_map, int3 qpos, __nv_bfloat16* O, int64_t o_row, int64_t o_head, int64_t o_tok,
                    const __grid_constant__ EncoderKeys enc, const __grid_constant__ HeldKeys held, int32_t T,
                    const __grid_constant__ TilePlan plan, float scale_log2, int* status)
{
    using C = TilesCfg<D>;
    extern __shared__ uint8_t smem_raw[];
    Barriers* bars = reinterpret_cast<Barriers*>(smem_raw);
    volatile int* abort_flag = &bars->abort_flag;
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t q_smem = (raw + (uint32_t)sizeof(Barriers) + 1023u) & ~1023u, kv_smem = q_smem + 2 * C::kQBytes;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        bars->abort_flag = 0;
        for (int g = 0; g < 2; ++g) {
            mbar_init(smem_u32(&bars->q_full[g]), 1);
            for (int b = 0; b < 2; ++b) {
                mbar_init(smem_u32(&bars->s_full[g][b]), 1);
                mbar_init(smem_u32(&bars->p_full[g][b]), kGroupWarps);
            }
            mbar_init(smem_u32(&bars->pv_done[g]), 1);
            mbar_init(smem_u32(&bars->o_full[g]), 1);
            mbar_init(smem_u32(&bars->drained[g]), 1);
        }
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&bars->kv_full[s]), kLoadWarps);
            mbar_init(smem_u32(&bars->kv_empty[s]), 2);   // one arrival per issuing warp, or two of the one whose tile it is
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    {
        // query rows that a tile does not cover keep whatever the slot held before; start them at zero
        uint4* qz = reinterpret_cast<uint4*>(smem_raw + (q_smem - raw));
        for (uint32_t i = threadIdx.x; i < 2 * C::kQBytes / 16; i += kThreads) qz[i] = make_uint4(0, 0, 0, 0);
        fence_async_smem();
    }
    if (warp == kMmaWarp) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)), "r"(C::kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
    overlap_with_previous();

    const uint32_t q_full0 = smem_u32(&bars->q_full[0]), kv_full0 = smem_u32(&bars->kv_full[0]), kv_empty0 = smem_u32(&bars->kv_empty[0]);
    const uint32_t s_full0 = smem_u32(&bars->s_full[0][0]), p_full0 = smem_u32(&bars->p_full[0][0]);   // + 16 g + 8 buffer
    const uint32_t pv_done0 = smem_u32(&bars->pv_done[0]), o_full0 = smem_u32(&bars->o_full[0]);
    const int64_t n_units = plan.units > blockIdx.x ? (plan.units - 1 - blockIdx.x) / gridDim.x + 1 : 0;   // of this CTA
    auto unit_at = [&](int64_t n) -> Unit { return Unit(plan, (int64_t)blockIdx.x + n * gridDim.x); };
    // blocks of keys of a row; a row without any is left out by every role (but for the zeros it gets)
    auto blocks_of = [&](const Unit& u) -> int32_t { return kHeld ? held.blocks : EncoderView(enc, u.row, 0).blocks(); };

    if (warp >= kLoadWarp) {
        // ------------------------------------------------------------ key/value stages
        const int tid = (int)threadIdx.x - kLoadWarp * 32;
        uint32_t sq = 0;                 // stages begun
        bool ok = true;
        auto announce = [&](uint32_t seq) {
            fence_async_smem();          // what this thread wrote is for the tensor cores to read
            __syncwarp();
            if (lane == 0) mbar_arrive(kv_full0 + 8 * (seq % kStages));
        };
        auto free_stage = [&](uint32_t seq) -> bool {
            return warp_wait(kv_empty0 + 8 * (seq % kStages), ((seq / kStages) & 1u) ^ 1u, abort_flag);
        };
        if constexpr (!kHeld) {
            constexpr int kPieces = D / 8, kStep = kLoadThreads / kPieces, kN = kKT / kStep;
            const int piece = tid % kPieces, row0 = tid / kPieces;
            static_assert(kStep % 8 == 0, "a thread's rows share their swizzle");
            const uint32_t slot = (uint32_t)(piece >> 3) * C::kKVHalfBytes + row0 * 128 + (((piece & 7) ^ (row0 & 7)) << 4);
            for (int64_t n = 0; ok && n < n_units; ++n) {
                const Unit u = unit_at(n);
                const EncoderView va(enc, u.row, u.head[0] / plan.group), vb(enc, u.row, u.two ? u.head[1] / plan.group : 0);
                const int n_tiles = (va.blocks() + kTileBlocks - 1) / kTileBlocks, per_tile = u.two && !u.shared ? 2 : 1;
                for (int j = 0; ok && j < n_tiles; ++j) {
                    const int rows = min(kTileBlocks, va.blocks() - j * kTileBlocks) * kBlock;   // (the products read no others)
                    for (int g = 0; g < per_tile; ++g, ++sq) {
                        if (!free_stage(sq)) {
                            ok = false;
                            break;
                        }
                        const __nv_bfloat16 *kp = (g ? vb.k : va.k) + piece * 8, *vp = (g ? vb.v : va.v) + piece * 8;
                        const uint32_t dst = kv_smem + sq % kStages * C::kStageBytes + slot;
#pragma unroll
                        for (int i = 0; i < kN; ++i) {
                            const int r = row0 + i * kStep;
                            if (r < rows) {
                                const int32_t key = j * kKT + r;
                                const int64_t at = key < va.len ? (int64_t)key * va.tok : 0;
                                copy16_or_zero(dst + i * kStep * 128, kp + at, key < va.len);
                                copy16_or_zero(dst + C::kKVBytes + i * kStep * 128, vp + at, key < va.len);
                            }
                        }
                        asm volatile("cp.async.commit_group;" ::: "memory");
                        // the stage before has landed; announced one late, it never holds up what frees the next stage
                        if (sq > 0) {
                            asm volatile("cp.async.wait_group 1;" ::: "memory");
                            announce(sq - 1);
                        }
                    }
                }
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            if (ok && sq > 0) announce(sq - 1);
        } else {
            constexpr int kPieces = D / 16, kStep = kLoadThreads / kPieces, kN = kKT / kStep;
            const int piece = tid % kPieces, row0 = tid / kPieces;
            static_assert(kStep % kBlock == 0, "a pass is whole blocks");
            const uint32_t swz = row0 & 7, half = (uint32_t)(2 * piece) >> 3, p0 = (2 * piece) & 7;
            const uint32_t lo_at = half * C::kKVHalfBytes + row0 * 128 + ((p0 ^ swz) << 4), hi_at = half * C::kKVHalfBytes + row0 * 128 + (((p0 + 1) ^ swz) << 4);
            uint4 k[kN], v[kN];
            int32_t ke[kN], ve[kN];
            auto fetch = [&](HeldView& view, int j) {
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    const int r = row0 + i * kStep;
                    const int32_t b = j * kTileBlocks + r / kBlock;
                    k[i] = v[i] = make_uint4(0, 0, 0, 0);
                    ke[i] = ve[i] = 0;
                    if (r % kBlock < view.valid(b)) {
                        const int32_t pos = view.position(b);
                        const uint8_t* src = view.codes + (int64_t)(pos + r % kBlock) * D + piece * 16;
                        k[i] = load_16B(src);
                        v[i] = load_16B(src + (int64_t)view.capacity * D);
                        ke[i] = load_exponent(view.exps + pos / kBlock);
                        ve[i] = load_exponent(view.exps + (view.capacity + pos) / kBlock);
                    }
                }
            };
            const int n_tiles = (held.blocks + kTileBlocks - 1) / kTileBlocks;
            for (int64_t n = 0; ok && n < n_units; ++n) {
                const Unit u = unit_at(n);
                HeldView va(held, (int64_t)u.row * plan.heads + u.head[0], D), vb(held, (int64_t)u.row * plan.heads + (u.two ? u.head[1] : u.head[0]), D);
                const int per_tile = u.two && !u.shared ? 2 : 1;
                fetch(va, 0);
                for (int j = 0; ok && j < n_tiles; ++j) {
                    const int rows = min(kTileBlocks, held.blocks - j * kTileBlocks) * kBlock;
                    for (int g = 0; g < per_tile; ++g, ++sq) {
                        if (!free_stage(sq)) {
                            ok = false;
                            break;
                        }
                        uint8_t* dst = smem_raw + (kv_smem - raw) + sq % kStages * C::kStageBytes;
#pragma unroll
                        for (int i = 0; i < kN; ++i) {
                            if (row0 + i * kStep < rows) {
                                uint4 lo, hi;
                                widen16(k[i], power_of_two(ke[i]), lo, hi);
                                *reinterpret_cast<uint4*>(dst + lo_at + i * kStep * 128) = lo;
                                *reinterpret_cast<uint4*>(dst + hi_at + i * kStep * 128) = hi;
                                widen16(v[i], power_of_two(ve[i]), lo, hi);
                                *reinterpret_cast<uint4*>(dst + C::kKVBytes + lo_at + i * kStep * 128) = lo;
                                *reinterpret_cast<uint4*>(dst + C::kKVBytes + hi_at + i * kStep * 128) = hi;
                            }
                        }
                        if (per_tile == 2 && g == 0) fetch(vb, j);
                        else if (j + 1 < n_tiles) fetch(va, j + 1);
                        announce(sq);
                    }
                }
            }
        }
        if (!ok && lane == 0) report(status, kStatusTmaTimeout, abort_flag);
    } else if (warp >= kMmaWarp) {
        // ------------------------------------------------------------ products of stream g
        const int g = warp - kMmaWarp;
        const uint32_t idesc_pv = make_idesc(kQRows, D, 1);
        const uint32_t k_lo0 = desc_lo(kv_smem, 16), v_lo0 = desc_lo(kv_smem + C::kKVBytes, C::kKVHalfBytes);
        const uint32_t q_lo = desc_lo(q_smem + g * C::kQBytes, 16);
        constexpr uint32_t kStageLo = C::kStageBytes >> 4;
        auto await = [&](uint32_t bar, uint32_t parity) -> bool {
            return warp_wait_lean(bar, parity, status, kStatusMmaTimeout, abort_flag);
        };
        uint32_t pv_stage = 0, pv_nch = 0, pv_first = 0, pv_last = 0, pv_twice = 0, t = 0, un = 0, sq = 0;   // t: tiles, un: units begun
        bool live = false;                                                                                  // a P V is due
        auto issue_pv = [&]() -> bool {
            const uint32_t last = t - 1u, buf = last & 1u;
            if (!await(p_full0 + 16 * g + 8 * buf, (last >> 1) & 1u)) return false;
            tc_fence_after();
            const uint32_t empty = kv_empty0 + 8 * pv_stage;
            umma_pv(tmem + C::kOCol + g * D, tmem + C::kSCol + (g * 2 + buf) * kKT, v_lo0 + pv_stage * kStageLo, kDescHi, idesc_pv, pv_first ^ 1u,
                    pv_nch, 1u, empty, pv_last, o_full0 + 8 * g);
            if (pv_twice) umma_commit_elected(empty);
            umma_commit_elected(pv_done0 + 8 * g);
            live = false;
            return true;
        };
        for (int64_t n = 0; n < n_units; ++n) {
            const Unit u = unit_at(n);
            const int32_t blocks = blocks_of(u);
            const int n_tiles = (blocks + kTileBlocks - 1) / kTileBlocks;
            const uint32_t per_tile = u.two && !u.shared ? 2u : 1u;
            if (g == 1 && !u.two) {
                // the last P V must not wait for a next S that is not coming soon: it holds a stage
                if (live && !issue_pv()) goto stopped;
                sq += (uint32_t)n_tiles;
                continue;
            }
            for (int j = 0; j < n_tiles; ++j, sq += per_tile) {
                const uint32_t nch = (uint32_t)min(kTileBlocks, blocks - j * kTileBlocks);
                const uint32_t seq = per_tile == 2u ? sq + g : sq, stage = seq % kStages;
                if (j == 0) {
                    if (!await(q_full0 + 8 * g, un & 1u)) goto stopped;
                    ++un;
                }
                // Shared tiles: S first, to run while the softmax of the tile before finishes.  Tiles of one stream: P V first, as
                // the stage it frees is what the tile behind this one waits for.
                if (per_tile == 2u && live && !issue_pv()) goto stopped;
                if (!await(kv_full0 + 8 * stage, (seq / kStages) & 1u)) goto stopped;
                tc_fence_after();
                const uint32_t buf = t & 1u;
                umma_s<D, C::kQHalfBytes, C::kKVHalfBytes>(tmem + C::kSCol + (g * 2 + buf) * kKT, q_lo, k_lo0 + stage * kStageLo, kDescHi,
                                                          make_idesc(kQRows, nch * 16, 0), s_full0 + 16 * g + 8 * buf);
                if (live && !issue_pv()) goto stopped;
                live = true;
                pv_stage = stage;
                pv_nch = nch;
                pv_first = j == 0;
                pv_last = j == n_tiles - 1;
                pv_twice = !u.shared;
                ++t;
            }
        }
        if (live) (void)issue_pv();
    stopped:;
    } else {
        // ------------------------------------------------------------ softmax and output (warps 0-7)
        const int g = warp >> 2, wq = warp & 3, r = wq * 32 + lane;
        const uint32_t lane_base = ((uint32_t)(wq * 32)) << 16;
        const uint32_t s_tmem0 = tmem + C::kSCol + g * 2 * kKT + lane_base, o_tmem = tmem + C::kOCol + g * D + lane_base;
        const bool q_loader = wq == 0 && lane == 0;
        const bool o_sectors = ((reinterpret_cast<uintptr_t>(O) | (uintptr_t)(2 * o_row) | (uintptr_t)(2 * o_head) | (uintptr_t)(2 * o_tok)) & 31u) == 0;
        uint32_t q_asked = 0;     // query tiles requested
        int64_t q_next = 0;       // first unit not yet searched for one
        auto load_next_q = [&]() {
            for (; q_next < n_units; ++q_next) {
                const Unit u = unit_at(q_next);
                if ((g == 1 && !u.two) || blocks_of(u) == 0) continue;
                const int32_t q0 = u.qt[g] * kQRows, boxes = (min(kQRows, T - q0) + kQBoxRows - 1) / kQBoxRows;
                const uint32_t bar = q_full0 + 8 * g, dst = q_smem + g * C::kQBytes;
                mbar_expect_tx(bar, (uint32_t)boxes * kQBoxRows * D * 2);
                int c[4] = {0, 0, 0, 0};
                c[qpos.y] = u.head[g];
                c[qpos.z] = u.row;
                for (int bx = 0; bx < boxes; ++bx) {
                    c[qpos.x] = q0 + bx * kQBoxRows;
#pragma unroll
                    for (int h = 0; h < C::kHalves; ++h)
                        tma_load_4d(dst + h * C::kQHalfBytes + bx * kQBoxRows * 128, &q_map, bar, h * 64, c[1], c[2], c[3]);
                }
                ++q_asked;
                ++q_next;
                return;
            }
        };
        if (q_loader) {
            prefetch_tensormap(&q_map);
            load_next_q();
        }
        __syncwarp();
        uint32_t t = 0, un = 0;   // tiles and units of this stream
        bool ok = true;
        for (int64_t n = 0; ok && n < n_units; ++n) {
            const Unit u = unit_at(n);
            if (g == 1 && !u.two) continue;
            EncoderView ev(enc, u.row, 0);
            HeldView hv(held, 0, D);
            const int32_t blocks = kHeld ? held.blocks : ev.blocks();
            const int n_tiles = (blocks + kTileBlocks - 1) / kTileBlocks;
            const int32_t valid_rows = min(kQRows, T - u.qt[g] * kQRows);
            const bool warp_live = wq * 32 < valid_rows;
            float m_ref = 0.f, l = 0.f, nb = 0.f;
            for (int j = 0; j < n_tiles; ++j, ++t) {
                const uint32_t buf = t & 1u, s_tmem = s_tmem0 + buf * kKT;
                if (!__all_sync(0xffffffffu, mbar_wait(s_full0 + 16 * g + 8 * buf, (t >> 1) & 1u, abort_flag))) {
                    report(status, kStatusSyncTimeout, abort_flag);
                    ok = false;
                    break;
                }
                tc_fence_after();
                if (j == n_tiles - 1 && q_loader) load_next_q();   // the last S has landed: its queries are no longer read
                if (warp_live) {
                    uint32_t sr[kKT];
                    tmem_ld64(s_tmem, sr);
                    const int groups = min(kTileBlocks, blocks - j * kTileBlocks);
                    uint64_t keep = 0;   // a bit per column that holds a key
                    if (kHeld) {
#pragma unroll
                        for (int b = 0; b < kTileBlocks; ++b) keep |= ((1ull << hv.valid(j * kTileBlocks + b)) - 1ull) << (b * kBlock);
                    } else {
                        const int32_t left = ev.len - j * kKT;
                        keep = left >= kKT ? ~0ull : (1ull << left) - 1ull;
                    }
                    if (keep != ~0ull) {
                        const uint32_t lo = (uint32_t)keep, hi = (uint32_t)(keep >> 32);
#pragma unroll
                        for (int i = 0; i < kKT; ++i)
                            if ((((i < 32 ? lo : hi) >> (i & 31)) & 1u) == 0u) sr[i] = 0xff800000u;  // -inf
                    }
                    float mx[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) mx[c] = max3(__uint_as_float(sr[c]), __uint_as_float(sr[4 + c]), __uint_as_float(sr[8 + c]));
#pragma unroll
                    for (int i = 12; i < kKT - 4; i += 8)
#pragma unroll
                        for (int c = 0; c < 4; ++c) mx[c] = max3(mx[c], __uint_as_float(sr[i + c]), __uint_as_float(sr[i + 4 + c]));
#pragma unroll
                    for (int c = 0; c < 4; ++c) mx[c] = fmaxf(mx[c], __uint_as_float(sr[kKT - 4 + c]));
                    const float mt = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
                    if (j == 0) {
                        m_ref = mt;
                        nb = -mt * scale_log2;
                    } else {
                        const bool grow = fmaf(mt, scale_log2, nb) > kRescaleLog2;
                        if (__any_sync(0xffffffffu, grow)) {
                            // rare: O and the sums to a new reference, once the P V before is done (the next one needs the P that
                            // this tile has not written yet)
                            if (!__all_sync(0xffffffffu, mbar_wait(pv_done0 + 8 * g, (t - 1u) & 1u, abort_flag))) {
                                report(status, kStatusSyncTimeout, abort_flag);
                                ok = false;
                                break;
                            }
                            tc_fence_after();
                            float alpha = 1.f;
                            if (grow) {
                                alpha = fast_exp2((m_ref - mt) * scale_log2);
                                m_ref = mt;
                                nb = -mt * scale_log2;
                                l *= alpha;
                            }
#pragma unroll 1
                            for (int cb = 0; cb < D / 8; ++cb) {
                                uint32_t o[8];
                                tmem_ld8(o_tmem + cb * 8, o);
#pragma unroll
                                for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                tmem_st8(o_tmem + cb * 8, o);
                            }
                        }
                    }
                    // P over S, bf16 (the type of V) for the product; the sums take the probabilities as they are.  Blocks behind the last
                    // one are not read by the product and keep stale bits.
                    float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
                    for (int grp = 0; grp < kTileBlocks; ++grp) {
                        if (grp < groups) {
                            uint32_t pk[8];
#pragma unroll
                            for (int ii = 0; ii < 8; ++ii) {
                                const int i = (grp & 1) * 8 + ii, c = grp * 16 + 2 * ii;
                                float x0, x1, p0, p1;
                                fma2(x0, x1, __uint_as_float(sr[c]), __uint_as_float(sr[c + 1]), scale_log2, scale_log2, nb, nb);
                                if (i % kPolyEvery == 0) {
                                    exp2_poly2(p0, p1, x0, x1);
                                } else {
                                    p0 = fast_exp2(x0);
                                    p1 = fast_exp2(x1);
                                }
                                add2(sum0, sum1, sum0, sum1, p0, p1);
                                const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
                                pk[ii] = *reinterpret_cast<const uint32_t*>(&h);
                            }
                            tmem_st8_nowait(s_tmem + grp * 8, pk);
                        }
                    }
                    l += sum0 + sum1;
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full0 + 16 * g + 8 * buf);
            }
            if (!ok) break;
            if (n_tiles > 0) {
                if (!__all_sync(0xffffffffu, mbar_wait(o_full0 + 8 * g, un & 1u, abort_flag))) {
                    report(status, kStatusSyncTimeout, abort_flag);
                    ok = false;
                    break;
                }
                ++un;
                tc_fence_after();
            }
            if (warp_live) {
                const float inv = n_tiles > 0 ? 1.f / l : 0.f;
                __nv_bfloat16* dst = O + u.row * o_row + u.head[g] * o_head + (int64_t)(u.qt[g] * kQRows + r) * o_tok;
#pragma unroll
                for (int cb = 0; cb < D / 32; ++cb) {
                    uint32_t o[32];
                    if (n_tiles > 0) {
                        tmem_ld32(o_tmem + cb * 32, o);
                    } else {   // a row without keys: zeros
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0u;
                    }
                    if (r < valid_rows) {
                        uint32_t w[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
                            w[i] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                        if (o_sectors) {
                            st_global_32B(dst + cb * 32, w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]);
                            st_global_32B(dst + cb * 32 + 16, w[8], w[9], w[10], w[11], w[12], w[13], w[14], w[15]);
                        } else {
#pragma unroll
                            for (int c = 0; c < 4; ++c)
                                reinterpret_cast<uint4*>(dst + cb * 32)[c] = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
                        }
                    }
                }
            }
            tc_fence_before();   // the reads of O come before the arrival on p_full for the next unit's first tile
        }
        // query tiles requested but never used must land before the CTA ends
        if (q_loader)
            for (uint32_t q = un; q < q_asked; ++q)
                for (uint32_t i = 0; i < kSpinLimit; ++i)
                    if (mbar_try_wait(q_full0 + 8 * g, q & 1u)) break;
    }

    // ---------------------------------------------------------------- teardown
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {   // (the same for all threads) a launch that gave up: its products end before tensor memory is given back
        if (warp >= kMmaWarp && warp < kLoadWarp) {
            const uint32_t drained = smem_u32(&bars->drained[warp - kMmaWarp]);
            umma_commit_elected(drained);
            for (uint32_t i = 0; i < kSpinLimit; ++i)
                if (mbar_try_wait(drained, 0u)) break;
        }
        __syncthreads();
    }
    if (warp == kMmaWarp) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
    }
}

template <int D, bool kHeld>
cudaError_t launch(const Strided& Q, const Strided& O, const EncoderKeys& enc, const HeldKeys& held, int32_t T, int32_t rows,
                   int32_t kv_heads, int32_t group, float softmax_scale, int* status, int sm_count, cudaStream_t stream)
{
    using C = TilesCfg<D>;
    TilePlan plan;
    plan.heads = kv_heads * group;
    plan.group = group;
    plan.nqt = (T + kQRows - 1) / kQRows;
    const int64_t streams = (int64_t)plan.nqt * plan.heads;
    if (T < 1 || streams > 0x7ffffffell) return cudaErrorInvalidValue;
    plan.units_per_row = (int32_t)((streams + 1) / 2);
    plan.units = (int64_t)rows * plan.units_per_row;
    CUtensorMap qm;
    int pos[3];
    if (!tc_encode_q_map(Q, T, rows, plan.heads, D, kQBoxRows, &qm, pos)) return cudaErrorNotSupported;
    static SharedMemoryOptIn opt_in;
    const cudaError_t oe = opt_in.ensure(attend_tiles_kernel<D, kHeld>, (int)C::kSmemBytes);
    if (oe != cudaSuccess) return oe;
    const int64_t grid = std::min<int64_t>(plan.units, sm_count);
    return launch_kernel(true, attend_tiles_kernel<D, kHeld>, dim3((unsigned)grid), dim3(kThreads), KernelMemory(C::kSmemBytes), stream, qm,
                         make_int3(pos[0], pos[1], pos[2]), (__nv_bfloat16*)O.ptr, O.row, O.head, O.token, enc, held, T, plan,
                         softmax_scale * 1.4426950408889634f, status);
}

}  // namespace

cudaError_t launch_attend_tiles(const Strided& Q, const Strided& O, const EncoderKeys& enc, int32_t T, int32_t rows, int32_t kv_heads,
                                int32_t group, int32_t D, float softmax_scale, int* status, int sm_count, cudaStream_t stream)
{
    HeldKeys none;
    memset(&none, 0, sizeof(none));
    if (D == 64) return launch<64, false>(Q, O, enc, none, T, rows, kv_heads, group, softmax_scale, status, sm_count, stream);
    return launch<128, false>(Q, O, enc, none, T, rows, kv_heads, group, softmax_scale, status, sm_count, stream);
}

cudaError_t launch_attend_tiles(const Strided& Q, const Strided& O, const HeldKeys& held, int32_t T, int32_t rows, int32_t heads,
                                int32_t D, float softmax_scale, int* status, int sm_count, cudaStream_t stream)
{
    EncoderKeys none;
    memset(&none, 0, sizeof(none));
    if (held.ranges.n < 1 || held.blocks < 1) return cudaErrorInvalidValue;
    if (D == 64) return launch<64, true>(Q, O, none, held, T, rows, heads, 1, softmax_scale, status, sm_count, stream);
    return launch<128, true>(Q, O, none, held, T, rows, heads, 1, softmax_scale, status, sm_count, stream);
}

}  // namespace amskv
