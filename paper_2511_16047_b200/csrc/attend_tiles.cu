// Attention over an encoder's states or a region held in 8 bits on the tensor cores: both products are tcgen05 instructions with their
// accumulators in tensor memory.  Calls of few queries or items take the warp-matrix kernel (attend_rows.cu).
//
// CTAs walk units of two streams, each a (query head, tile of 128 queries) of the same row, and so with as many keys.  Two
// streams of one key/value head (two tiles of a head, or heads of a group) share every tile of 64 keys in shared memory; others
// have tiles of their own, which alternate.
//   warps 0-3, 4-7   softmax of stream A, of stream B: a query row per thread (row = TMEM lane)
//   then kMmaWarps   issue the products: one warp for both streams, or one for each
//   then kLoadWarps  fill the stages of keys and values: with bulk copies, or by widening codes
//   then kFetchWarps ask for codes (else the first loading warp does)
// Per tile: S = Q K^T (128 x 64 fp32); the softmax warps exponentiate in base 2 against a reference maximum and write P as bf16 over S;
// O += P V with P from tensor memory.  The reference is the maximum of the first tile; later tiles' maxima are not even taken: a row
// that outgrows it (by 2^64 in the sum over a tile, or to what is not a number) makes its warp take the true maxima, rescale O and the
// sums, and form the tile again.
//   64 channels: two CTAs per SM, so that 16 softmax warps keep the special-function unit busy.
//   128 channels: one CTA per SM with two S buffers per stream (S of the next tile is formed while the softmax of this one runs), two
//     issuing warps and, over an encoder, two query tiles per stream, so that a unit's queries are there when it begins.
// Keys behind a row's last one may be anything, NaN among them, and a product with a zero probability would spread it: the block
// that a row's values do not fill comes in 16-byte asynchronous copies, with zeros behind the last key; all else in bulk copies.  Codes
// come in bulk copies into a ring of tiles, from which warps widen them to bf16; where a tile's codes lie, and which of its slots
// hold a key, is tabulated once per launch.
// What bounds it: the exponentials, 64 channels (a tile's 8 192 take 512 cycles of an SM's special-function unit, the products 256), and
// the products, 128 channels; with codes no unit by itself (64 channels: special-function unit 46 %, issue slots 44 % busy at 425 keys), but the
// chain of widening, S, softmax and P V, whose waits for tensor memory lead.  4 096 queries x 10 521 keys x 64
// heads: 64 channels 910 us (0.73 PFLOP/s of products), 128 channels 1 050 (1.26); from codes 1 040 to 1 270 and 1 250 (0.9 and 1.06).
// 256 queries x 430 keys: 64 channels, 3 840 heads 176, codes 225; 128 channels, 2 048 heads 141, codes 176.
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
constexpr int kOutRows = 32;      // output rows per bulk copy: those of a warp
constexpr int kKT = 64;           // keys per tile
constexpr int kTileBlocks = kKT / kBlock;
constexpr int kGroupWarps = 4;
constexpr int kMmaWarp = 8;
constexpr int kMaxStages = 4;
constexpr float kRescaleLog2 = 8.f;
// Probabilities are formed 2^kLowered below what the reference makes of them, so that a row may outgrow it by 2^64 while its sums stay below
// 2^24: values are multiplied by no more, and fp32 holds their sums as long as (keys / 64) * |V| stays below 2^104.  (Formed as they
// are, with a limit of 2^64, values of 2^64 were infinities in O; a limit of 2^14 instead costs 20 to 50 % where logits spread by 10.)
constexpr float kLowered = 40.f;
constexpr float kSumLimit = 16777216.f;      // 2^24
constexpr int kHeldTab = 192;                // tiles of a cache that are tabulated in shared memory

template <int D, bool kHeld>
struct TilesCfg {
    static constexpr bool kWide = D == 128;
    static constexpr int kCtasPerSm = kWide ? 1 : 2, kStages = kWide || kHeld ? 3 : 4;
    static constexpr int kSBufs = kWide ? 2 : 1, kQBufs = kWide && !kHeld ? 2 : 1;     // per stream
    // Every so many pairs of exponentials come from the FMA pipe (0: none), where the special-function unit is what a tile waits for.  Not
    // beside warps that widen codes with two CTAs' softmax warps, which leave no room for more instructions.
    static constexpr int kPolyEvery = kWide ? 6 : kHeld ? 0 : 12;
    // Outputs go through the place of their unit's queries (below): with one such place that holds the next unit's queries up, which with
    // 64 channels costs more than scattered stores do.
    static constexpr bool kBulkOut = kWide;
    static constexpr int kMmaWarps = kWide ? 2 : 1, kLoadWarps = kWide && kHeld ? 4 : 1;
    static constexpr int kFetchWarps = kWide && kHeld ? 1 : 0;  // a warp that only asks for codes, else the first loading warp does
    static constexpr int kWarps = kMmaWarp + kMmaWarps + kLoadWarps + kFetchWarps, kThreads = kWarps * 32;
    static constexpr bool kLoaderQ = kQBufs == 2;               // the loading warp fetches the queries, else a lane of each softmax group does
    static constexpr int kHalves = D / 64;                      // 128-byte swizzle atoms per row
    static constexpr uint32_t kQBytes = kQRows * D * 2, kQHalfBytes = kQRows * 128;
    static constexpr uint32_t kKVBytes = kKT * D * 2, kKVHalfBytes = kKT * 128;
    static constexpr uint32_t kStageBytes = 2 * kKVBytes;
    static constexpr int kRing = kHeld ? 2 : 0;                 // tiles of codes on their way, each with 32 bytes behind it
    static constexpr uint32_t kCodeBytes = 2 * kKT * D, kRingBytes = kCodeBytes + 32;
    static constexpr uint32_t kSmemBytes = 2048 + 2 * kQBufs * kQBytes + kStages * kStageBytes + kRing * kRingBytes +
                                           (kHeld ? kHeldTab * 24 : 0);   // barriers and slack in front
    static constexpr uint32_t kTmemCols = kWide ? 512 : 256, kSCol = 0, kOCol = 2 * kSBufs * kKT;   // S of both streams, then O of both
    static_assert(kOCol + 2 * D <= kTmemCols && kCtasPerSm * kTmemCols <= 512, "tensor memory");
    static_assert(kCtasPerSm * (kSmemBytes + 1024) <= 228 * 1024, "shared memory");
    static_assert(kKVHalfBytes % 1024 == 0 && kQHalfBytes % 1024 == 0 && kStages <= kMaxStages, "swizzle atoms stay 1024-byte aligned");
};

struct Barriers {
    uint64_t q_full[2][2], q_free[2][2], ring_full[2], ring_empty[2], kv_full[kMaxStages], kv_empty[kMaxStages], s_full[2][2], p_full[2][2], pv_done[2], o_full[2], drained[2];
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(Barriers) + 1024 <= 2048, "barriers fit in front of the aligned tiles");

struct TilePlan {
    Divisor nqt, group, units_per_row;   // query tiles per head; query heads per key/value head; ceil(nqt * heads / 2)
    int32_t heads;
    int32_t units;
    uint32_t sms;
};
// Unit n: streams 2 u and 2 u + 1 of its row's nqt * heads.
struct Unit {
    int32_t row, head0, head1, qt0, qt1, kv0, kv1;
    bool two, shared;

    __device__ __forceinline__ Unit(const TilePlan& p, int32_t n)
    {
        row = p.units_per_row(n);
        const int32_t s = 2 * (n - row * (int32_t)p.units_per_row.d), nqt = (int32_t)p.nqt.d;
        head0 = p.nqt(s);
        qt0 = s - head0 * nqt;
        head1 = head0 + (qt0 + 1 == nqt ? 1 : 0);
        qt1 = qt0 + 1 == nqt ? 0 : qt0 + 1;
        two = head1 < p.heads;
        kv0 = p.group(head0);
        kv1 = two ? p.group(head1) : kv0;
        shared = two && kv0 == kv1;
    }
    __device__ __forceinline__ int32_t head(int g) const { return g ? head1 : head0; }
    __device__ __forceinline__ int32_t qt(int g) const { return g ? qt1 : qt0; }
};

// Which 16-byte pieces of a tile of codes a loading warp moves: of the tile's 128 rows, 64 of K and 64 of V behind them, the kRows of every
// kLoadWarps-th pass, a row kPieces lanes wide.
template <int D>
struct CodeShare {
    static constexpr int kPieces = D / 16, kRows = 32 / kPieces, kWarps = TilesCfg<D, true>::kLoadWarps, kN = 2 * kKT / kRows / kWarps;
    static constexpr int kBatch = 4;
    static_assert(2 * kKT % (kRows * kWarps) == 0 && kBlock % (kRows * kWarps) == 0 && kN % kBatch == 0, "a block is whole rounds of the warps");
};

// Coordinates 1 to 3 of a rank-4 map whose token, head and row dimensions are at `pos`.
__device__ __forceinline__ int3 coords(const int3& pos, int tok, int head, int row)
{
    auto at = [&](int i) { return pos.x == i ? tok : pos.y == i ? head : row; };
    return make_int3(at(1), at(2), at(3));
}

// Tile j of a cache: a bit per slot that holds a key, and the first slots of the blocks.  (Not inlined: beyond the table it is hardly ever
// called, and the registers are the softmax warps'.)
__device__ __noinline__ uint64_t held_tile(const HeldKeys& held, int j, int4* pos)
{
    HeldView view(held, 0, 0);
    uint64_t keep = 0;
    int32_t p[kTileBlocks];
#pragma unroll
    for (int b = 0; b < kTileBlocks; ++b) {
        const int32_t n = view.valid(j * kTileBlocks + b);
        keep |= ((1ull << n) - 1ull) << (b * kBlock);
        p[b] = n > 0 ? view.position(j * kTileBlocks + b) : p[0];   // (the first block is there)
    }
    if (pos) *pos = make_int4(p[0], p[1], p[2], p[3]);
    return keep;
}

template <int D, bool kHeld>
__global__ void __launch_bounds__(TilesCfg<D, kHeld>::kThreads, TilesCfg<D, kHeld>::kCtasPerSm)
attend_tiles_kernel(const __grid_constant__ CUtensorMap q_map, int3 qpos, const __grid_constant__ CUtensorMap o_map, int3 opos,
                    const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                    const __grid_constant__ CUtensorMap v_map16, int3 kpos, __nv_bfloat16* O, int64_t o_row, int64_t o_head, int64_t o_tok,
                    const __grid_constant__ EncoderKeys enc, const __grid_constant__ HeldKeys held, int32_t T,
                    const __grid_constant__ TilePlan plan, float scale_log2, int* status)
{
    using C = TilesCfg<D, kHeld>;
    extern __shared__ uint8_t smem_raw[];
    Barriers* bars = reinterpret_cast<Barriers*>(smem_raw);
    volatile int* abort_flag = &bars->abort_flag;
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t q_smem = (raw + (uint32_t)sizeof(Barriers) + 1023u) & ~1023u, kv_smem = q_smem + 2 * C::kQBufs * C::kQBytes;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    // Two CTAs on an SM: the loading warp of one is beside the issuing warp of the other on an SM sub-partition (as far as CTAs a whole
    // round of SMs apart share one).
    const bool swapped = C::kCtasPerSm == 2 && ((uint32_t)blockIdx.x / plan.sms & 1u) != 0;
    const int mma_warp = swapped ? kMmaWarp + C::kLoadWarps : kMmaWarp, load_warp = swapped ? kMmaWarp : kMmaWarp + C::kMmaWarps;

    if (threadIdx.x == 0) {
        bars->abort_flag = 0;
        for (int g = 0; g < 2; ++g) {
            for (int b = 0; b < 2; ++b) {
                mbar_init(smem_u32(&bars->q_full[g][b]), 1);
                mbar_init(smem_u32(&bars->q_free[g][b]), kGroupWarps);
                mbar_init(smem_u32(&bars->s_full[g][b]), 1);
                mbar_init(smem_u32(&bars->p_full[g][b]), kGroupWarps);
            }
            mbar_init(smem_u32(&bars->pv_done[g]), 1);
            mbar_init(smem_u32(&bars->o_full[g]), 1);
            mbar_init(smem_u32(&bars->drained[g]), 1);
        }
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(smem_u32(&bars->kv_full[s]), kHeld ? C::kLoadWarps : 33);   // (the lanes of the one loading warp, and its bulk copies)
            mbar_init(smem_u32(&bars->kv_empty[s]), C::kMmaWarps);   // one arrival per issuing warp, whether it uses the tile or passes it
        }
        for (int s = 0; s < C::kRing; ++s) {
            mbar_init(smem_u32(&bars->ring_full[s]), 1 + kTileBlocks);   // the bulk copies, and a scale word each
            mbar_init(smem_u32(&bars->ring_empty[s]), C::kLoadWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // A cache's tiles, the same for all units, are tabulated: worked out tile by tile the softmax and the loading warps would pay for it (430 keys x
    // 256 queries x 3 840 heads of 64: 311 us, 246 with the masks in a table, 232 with the positions, too).
    int4* pos_tab = reinterpret_cast<int4*>(smem_raw + (kv_smem - raw) + C::kStages * C::kStageBytes + C::kRing * C::kRingBytes);
    uint64_t* mask_tab = reinterpret_cast<uint64_t*>(pos_tab + kHeldTab);
    if (kHeld)
        for (int j = threadIdx.x; j < kHeldTab && j * kTileBlocks < held.blocks; j += C::kThreads) mask_tab[j] = held_tile(held, j, pos_tab + j);
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

    const uint32_t q_full0 = smem_u32(&bars->q_full[0][0]), kv_full0 = smem_u32(&bars->kv_full[0]), kv_empty0 = smem_u32(&bars->kv_empty[0]);
    const uint32_t s_full0 = smem_u32(&bars->s_full[0][0]), p_full0 = smem_u32(&bars->p_full[0][0]);   // + 16 g + 8 buffer (q_full0 too)
    const uint32_t pv_done0 = smem_u32(&bars->pv_done[0]), o_full0 = smem_u32(&bars->o_full[0]);
    const int32_t n_units = plan.units > (int32_t)blockIdx.x ? (plan.units - 1 - (int32_t)blockIdx.x) / (int32_t)gridDim.x + 1 : 0;   // of this CTA
    auto unit_at = [&](int32_t n) -> Unit { return Unit(plan, (int32_t)(blockIdx.x + n * gridDim.x)); };
    // the bounds of unit n's row, asked for a unit ahead (those of the last unit once more behind it)
    auto bounds_at = [&](int32_t n) -> EncoderBounds {
        return EncoderBounds(enc, plan.units_per_row((int32_t)(blockIdx.x + min(n, n_units - 1) * gridDim.x)));
    };
    // S buffer and phase of a stream's tile t; query buffer and phase of its unit n
    auto buf_of = [](uint32_t t) -> uint32_t { return C::kSBufs == 2 ? t & 1u : 0u; };
    auto par_of = [](uint32_t t) -> uint32_t { return C::kSBufs == 2 ? (t >> 1) & 1u : t & 1u; };
    auto qbuf_of = [](uint32_t n) -> uint32_t { return C::kQBufs == 2 ? n & 1u : 0u; };
    auto qpar_of = [](uint32_t n) -> uint32_t { return C::kQBufs == 2 ? (n >> 1) & 1u : n & 1u; };
    // blocks of keys of a row; a row without any is left out by every role (but for the zeros it gets)
    auto blocks_of = [&](const EncoderBounds& b) -> int32_t { return kHeld ? held.blocks : (b.len(enc) + kBlock - 1) / kBlock; };

    const uint32_t q_free0 = smem_u32(&bars->q_free[0][0]);
    // (one lane) the query tile of stream g in unit u, the q-th of the stream
    auto load_q = [&](const Unit& u, int g, uint32_t q) {
        const uint32_t qb = qbuf_of(q), bar = q_full0 + 16 * g + 8 * qb, dst = q_smem + (g * C::kQBufs + qb) * C::kQBytes;
        mbar_expect_tx(bar, C::kQBytes);
        const int3 c = coords(qpos, u.qt(g) * kQRows, u.head(g), u.row);
#pragma unroll
        for (int h = 0; h < C::kHalves; ++h) tma_load_4d(dst + h * C::kQHalfBytes, &q_map, bar, h * 64, c.x, c.y, c.z);
    };
    // the output that went through the place of query tile q has left it
    auto q_place_free = [&](int g, uint32_t q) -> bool {
        return q < (uint32_t)C::kQBufs || mbar_wait(q_free0 + 16 * g + 8 * qbuf_of(q), (q / C::kQBufs - 1u) & 1u, abort_flag);
    };
    auto await_q = [&](int g, uint32_t q) {   // whatever becomes of the launch, a copy into shared memory ends before the CTA does
        for (uint32_t i = 0; i < kSpinLimit; ++i)
            if (mbar_try_wait(q_full0 + 16 * g + 8 * qbuf_of(q), qpar_of(q))) break;
    };

    if (warp >= load_warp && warp < load_warp + C::kLoadWarps + C::kFetchWarps) {
        // ------------------------------------------------------------ key/value stages
        uint32_t stage = 0, phase = 0;   // of the next tile
        bool ok = true;
        auto next_stage = [&]() {
            if (++stage == C::kStages) {
                stage = 0;
                phase ^= 1u;
            }
        };
        // What warps wrote themselves is announced by their arrivals alone; the fence that orders these writes before the tensor cores' reads
        // is the issuing warps'.  Here it would wait for all copies in flight, so that no tile could be fetched ahead.
        auto free_stage = [&]() -> bool { return warp_wait(kv_empty0 + 8 * stage, phase ^ 1u, abort_flag); };
        // place in a stage of channels 8 c .. 8 c + 7 of row r of its 128
        auto place = [](int r, int c) -> uint32_t {
            return (uint32_t)((r / kKT) * (int)C::kKVBytes + (c >> 3) * (int)C::kKVHalfBytes + (r % kKT) * 128 + (((c & 7) ^ (r & 7)) << 4));
        };
        if constexpr (!kHeld) {
            // Bulk copies, but for the last block of values of a row that it does not fill: these come piece by piece, with zeros behind the last
            // one, as a probability of zero does not take away what a product makes of a NaN.  (Scores of keys behind the last one
            // are overwritten, whatever they are.)
            if (lane == 0) {
                prefetch_tensormap(&k_map);
                prefetch_tensormap(&v_map);
                prefetch_tensormap(&v_map16);
            }
            constexpr int kPieces = D / 8, kRows = 32 / kPieces;
            const int piece = lane % kPieces, row = lane / kPieces;
            uint32_t q_asked[2] = {0, 0}, issued = 0;
            EncoderBounds ahead = bounds_at(0);
            for (int32_t n = 0; ok && n < n_units; ++n) {
                const Unit u = unit_at(n);
                const EncoderView view(enc, u.row, u.kv0, ahead);
                const int32_t first_key = ahead.first(enc);
                ahead = bounds_at(n + 1);
                const int32_t blocks = view.blocks();
                const int n_tiles = (blocks + kTileBlocks - 1) / kTileBlocks, per_tile = u.two && !u.shared ? 2 : 1;
                if (C::kLoaderQ && n_tiles > 0) {
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        if (g == 1 && !u.two) break;
                        if (!__all_sync(0xffffffffu, q_place_free(g, q_asked[g]))) {
                            ok = false;
                            break;
                        }
                        if (elect_one()) load_q(u, g, q_asked[g]);
                        __syncwarp();
                        ++q_asked[g];
                    }
                }
                for (int j = 0; ok && j < n_tiles; ++j) {
                    const int32_t left = view.len - j * kKT;
                    for (int g = 0; g < per_tile; ++g) {
                        if (!free_stage()) {
                            ok = false;
                            break;
                        }
                        const uint32_t dst = kv_smem + stage * C::kStageBytes, bar = kv_full0 + 8 * stage;
                        const int whole = min(left / kBlock, kTileBlocks), over = left - whole * kBlock;   // blocks of values; values over (>= 16: none)
                        if (elect_one()) {
                            mbar_expect_tx(bar, C::kKVBytes + (uint32_t)whole * kBlock * D * 2);
                            const int tok = first_key + j * kKT, head = g ? u.kv1 : u.kv0, from = enc.row_maps ? u.row : 0;
                            const int3 c = coords(kpos, tok, head, from);
#pragma unroll
                            for (int h = 0; h < C::kHalves; ++h) tma_load_4d(dst + h * C::kKVHalfBytes, &k_map, bar, h * 64, c.x, c.y, c.z);
                            if (whole == kTileBlocks) {
#pragma unroll
                                for (int h = 0; h < C::kHalves; ++h)
                                    tma_load_4d(dst + C::kKVBytes + h * C::kKVHalfBytes, &v_map, bar, h * 64, c.x, c.y, c.z);
                            } else {
#pragma unroll 1
                                for (int b = 0; b < whole; ++b) {
                                    const int3 cb = coords(kpos, tok + b * kBlock, head, from);
#pragma unroll
                                    for (int h = 0; h < C::kHalves; ++h)
                                        tma_load_4d(dst + C::kKVBytes + h * C::kKVHalfBytes + b * kBlock * 128, &v_map16, bar, h * 64, cb.x, cb.y, cb.z);
                                }
                            }
                        }
                        __syncwarp();
                        if (whole < kTileBlocks && over > 0) {
                            const __nv_bfloat16* src = view.v + (int64_t)(j * kKT + whole * kBlock) * view.tok + (g ? (int64_t)(u.kv1 - u.kv0) * enc.head : 0) + piece * 8;
#pragma unroll
                            for (int i = 0; i < kBlock / kRows; ++i) {
                                const int r = i * kRows + row;
                                copy16_or_zero(dst + place(kKT + whole * kBlock + r, piece), r < over ? src + r * view.tok : view.v, r < over);
                            }
                            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");   // once they have landed
                        } else if (lane == 0) {
                            mbar_arrive_n(bar, 32);
                        }
                        __syncwarp();
                        ++issued;
                        next_stage();
                    }

                }
            }
            // whatever becomes of the launch, copies into shared memory end before the CTA does
            asm volatile("cp.async.wait_all;" ::: "memory");
            for (uint32_t q = issued > (uint32_t)C::kStages ? issued - C::kStages : 0u; q < issued; ++q)
                for (uint32_t i = 0; i < kSpinLimit; ++i)
                    if (mbar_try_wait(kv_full0 + 8 * (q % C::kStages), (q / C::kStages) & 1u)) break;
            if (C::kLoaderQ) {
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    for (uint32_t q = q_asked[g] > 2u ? q_asked[g] - 2u : 0u; q < q_asked[g]; ++q) await_q(g, q);
            }
        } else {
            // Codes land in a ring of their own by bulk copies of whole blocks, and with them the scale words of the
            // four blocks and the number of slots that the products read (0: there is no further tile).  Slots without a key keep what
            // they held: any code times a block's power is a finite number, and its probability is zero (but in a block that is no number, whose
            // row is none either).  (Fetched into registers instead, a wait for a tile's codes
            // waits for all younger ones too, as loads are counted, not named; with 16-byte copies of every lane the copies took as
            // many instructions as the widening.)
            using Share = CodeShare<D>;
            // A lane's piece and row of a pass.  The row's lowest bit is bit 2 of the lane, so that eight lanes that store together, four pieces of two
            // rows, meet all banks.
            const int w = warp - load_warp, piece = (lane & 3) + (Share::kPieces == 8 ? (lane >> 1) & 4 : 0);
            const int row = ((lane >> 2) & 1) + (Share::kPieces == 8 ? (lane >> 3) & 2 : (lane >> 2) & 6);
            // (a pass's first row is a multiple of kRows, which divides 8, so that the swizzle of a row is that of the pass and that of the lane)
            const uint32_t part_lo = place(row, 2 * piece), part_hi = place(row, 2 * piece + 1);
            auto at_pass = [](uint32_t part, int p) -> uint32_t {
                const int r = p * Share::kRows;
                return (part ^ (uint32_t)((r & 7) << 4)) + (uint32_t)((r / kKT) * (int)C::kKVBytes + (r % kKT) * 128);
            };
            const int n_tiles = (held.blocks + kTileBlocks - 1) / kTileBlocks;
            uint8_t* ring = smem_raw + (kv_smem - raw) + C::kStages * C::kStageBytes;
            const uint32_t ring_at = kv_smem + C::kStages * C::kStageBytes;
            const uint32_t ring_full0 = smem_u32(&bars->ring_full[0]), ring_empty0 = smem_u32(&bars->ring_empty[0]);
            int32_t f_n = 0;   // the walk of the copies: unit, tile, stream
            int f_j = 0, f_g = 0;
            Unit f_u = unit_at(0);
            const int64_t values_at = (int64_t)held.capacity * D, scales_of_item = held.capacity / kBlock;
            uint32_t f_slot = 0, f_phase = 0, asked = 0;
            bool ended = false;
            static_assert(C::kRing <= 2, "barriers");
            static_assert(C::kFetchWarps == 1 || C::kLoadWarps == 1, "one warp asks for codes");
            auto fetch = [&]() -> bool {   // the next tile into the ring
                if (ended) return true;
                if (!warp_wait(ring_empty0 + 8 * f_slot, f_phase ^ 1u, abort_flag)) return false;
                const uint32_t at = f_slot * C::kRingBytes, bar = ring_full0 + 8 * f_slot;
                int* slots = reinterpret_cast<int*>(ring + at + C::kCodeBytes + 16);
                if (f_n >= n_units) {
                    ended = true;
                    if (lane == 0) {
                        *slots = 0;
                        mbar_arrive_n(bar, 1 + kTileBlocks);
                    }
                    __syncwarp();
                    ++asked;   // (it takes a phase of its place, as a tile does)
                    return true;
                }
                int4 pos;
                uint64_t keep;
                if (f_j < kHeldTab) {
                    pos = pos_tab[f_j];
                    keep = mask_tab[f_j];
                } else {
                    keep = held_tile(held, f_j, &pos);
                }
                const int64_t item = (int64_t)f_u.row * plan.heads + f_u.head0 + f_g;   // (the other stream's is the item behind the first one's)
                const uint8_t* codes = held.codes + item * 2 * values_at;
                const uint32_t to = ring_at + at;
                if (lane == 0) {
                    *slots = min(kTileBlocks, held.blocks - f_j * kTileBlocks) * kBlock;
                    mbar_expect_tx(bar, 2u * (uint32_t)__popcll(keep) * D);
                }
                __syncwarp();
                if (lane < kTileBlocks) {   // a lane per block (one that is not there: the first one's word)
                    const int32_t p = lane == 0 ? pos.x : lane == 1 ? pos.y : lane == 2 ? pos.z : pos.w;
                    copy4(to + C::kCodeBytes + lane * 4, held.scales + item * scales_of_item + p / kBlock);
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
                    const bool whole = keep == ~0ull && pos.w == pos.x + 3 * kBlock;   // one piece of the region (blocks are in its order)
                    const uint32_t n = whole ? (lane == 0 ? (uint32_t)kKT : 0u) : (uint32_t)__popcll((keep >> (lane * kBlock)) & 0xffffull);
                    if (n > 0) {
                        bulk_load(to + lane * kBlock * D, codes + (int64_t)p * D, n * D, bar);
                        bulk_load(to + (kKT + lane * kBlock) * D, codes + values_at + (int64_t)p * D, n * D, bar);
                    }
                }
                __syncwarp();
                ++asked;
                if (++f_slot == C::kRing) {
                    f_slot = 0;
                    f_phase ^= 1u;
                }
                // next: the other stream's tile (the item behind this one), the next tile, the next unit
                if (f_u.two && !f_u.shared && f_g == 0) {
                    f_g = 1;
                } else {
                    f_g = 0;
                    if (++f_j == n_tiles) {
                        f_j = 0;
                        if (++f_n < n_units) f_u = unit_at(f_n);
                    }
                }
                return true;
            };
            uint32_t slot = 0, ring_phase = 0;   // of the next tile
            if (C::kFetchWarps > 0 && w == C::kLoadWarps)
                while (ok && !ended) ok = fetch();
            if (C::kFetchWarps == 0)
                for (int i = 0; ok && i < C::kRing; ++i) ok = fetch();
            while (ok && w < C::kLoadWarps) {
                if (!warp_wait(ring_full0 + 8 * slot, ring_phase, abort_flag)) {
                    ok = false;
                    break;
                }
                const uint8_t* from = ring + slot * C::kRingBytes;
                const int rows = *reinterpret_cast<const int*>(from + C::kCodeBytes + 16);
                if (rows == 0) break;
                const uint4 words = *reinterpret_cast<const uint4*>(from + C::kCodeBytes);
                if (!free_stage()) {
                    ok = false;
                    break;
                }
                uint8_t* dst = smem_raw + (kv_smem - raw) + stage * C::kStageBytes;
                const uint8_t* mine = from + (w * Share::kRows + row) * D + piece * 16;
                auto put = [&](int i, const uint4& codes, uint32_t factor, uint32_t rest) {
                    const int p = w + i * Share::kWarps;
                    uint4 lo, hi;
                    widen16(codes, factor, rest, lo, hi);
                    *reinterpret_cast<uint4*>(dst + at_pass(part_lo, p)) = lo;
                    *reinterpret_cast<uint4*>(dst + at_pass(part_hi, p)) = hi;
                };
                auto codes_at = [&](int i) -> uint4 { return *reinterpret_cast<const uint4*>(mine + i * Share::kWarps * Share::kRows * D); };
                if (rows == kKT && ((words.x | words.y | words.z | words.w) >> 16) == 0u) {
                    // (nearly always) several passes' codes before the first is stored: no load can move above a store for the compiler
#pragma unroll
                    for (int i0 = 0; i0 < Share::kN; i0 += Share::kBatch) {
                        uint4 x[Share::kBatch];
#pragma unroll
                        for (int i = 0; i < Share::kBatch; ++i) x[i] = codes_at(i0 + i);
#pragma unroll
                        for (int i = 0; i < Share::kBatch; ++i) {
                            const int b = (i0 + i) * Share::kWarps * Share::kRows % kKT / kBlock;
                            put(i0 + i, x[i], scale_factor(b == 0 ? words.x : b == 1 ? words.y : b == 2 ? words.z : words.w, i0 + i >= Share::kN / 2), 0u);
                        }
                    }
                } else {
#pragma unroll 1
                    for (int i = 0; i < Share::kN; ++i) {
                        const int b = i * Share::kWarps * Share::kRows % kKT / kBlock;
                        const uint32_t v = b == 0 ? words.x : b == 1 ? words.y : b == 2 ? words.z : words.w;
                        if (b * kBlock < rows) put(i, codes_at(i), scale_factor(v, i >= Share::kN / 2), scale_rest(v, i >= Share::kN / 2));
                    }
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(kv_full0 + 8 * stage);
                    mbar_arrive(ring_empty0 + 8 * slot);
                }
                next_stage();
                if (++slot == C::kRing) {
                    slot = 0;
                    ring_phase ^= 1u;
                }
                if (C::kFetchWarps == 0) ok = fetch();   // into the place of this tile
            }
            // whatever becomes of the launch, copies into shared memory end before the CTA does
            asm volatile("cp.async.wait_all;" ::: "memory");
            for (uint32_t q = asked > (uint32_t)C::kRing ? asked - C::kRing : 0u; q < asked; ++q)
                for (uint32_t i = 0; i < kSpinLimit; ++i)
                    if (mbar_try_wait(ring_full0 + 8 * (q % C::kRing), (q / C::kRing) & 1u)) break;
        }
        if (!ok && lane == 0) report(status, kStatusTmaTimeout, abort_flag);
    } else if (warp >= mma_warp && warp < mma_warp + C::kMmaWarps) {
        // ------------------------------------------------------------ products
        constexpr int kStreams = C::kMmaWarps == 2 ? 1 : 2;   // streams this warp issues for
        const int my_g = warp - mma_warp;
        const uint32_t idesc_pv = make_idesc(kQRows, D, 1);
        const uint32_t k_lo0 = desc_lo(kv_smem, 16), v_lo0 = desc_lo(kv_smem + C::kKVBytes, C::kKVHalfBytes), q_lo0 = desc_lo(q_smem, 16);
        constexpr uint32_t kStageLo = C::kStageBytes >> 4, kQLo = C::kQBytes >> 4;
        auto await = [&](uint32_t bar, uint32_t parity) -> bool {
            return warp_wait_lean(bar, parity, status, kStatusMmaTimeout, abort_flag);
        };
        // of each stream: the tile whose P V is due; tiles and units begun
        uint32_t pv_stage[kStreams] = {}, pv_nch[kStreams] = {}, pv_first[kStreams] = {}, t[kStreams] = {}, un[kStreams] = {};
        uint32_t stage = 0, phase = 0;   // of the next tile
        bool shared = false;             // the unit's tiles are for both streams
        auto issue_pv = [&](const int i, const uint32_t last) -> bool {
            const int g = kStreams == 2 ? i : my_g;
            const uint32_t tile = t[i] - 1u, buf = buf_of(tile);
            if (!await(p_full0 + 16 * g + 8 * buf, par_of(tile))) return false;
            // (a unit's first P V overwrites O: the softmax warps arrive for that tile only after they have read O of the unit before)
            tc_fence_after();
            const uint32_t empty = kv_empty0 + 8 * pv_stage[i];
            // (one issuer and shared tiles: the second stream's product, behind the first's, frees the stage)
            umma_pv(tmem + C::kOCol + g * D, tmem + C::kSCol + (g * C::kSBufs + buf) * kKT, v_lo0 + pv_stage[i] * kStageLo, kDescHi, idesc_pv,
                    pv_first[i] ^ 1u, pv_nch[i], kStreams == 2 && i == 0 ? (shared ? 0u : 1u) : 1u, empty, last, o_full0 + 8 * g);
            if (C::kMmaWarps == 2) umma_commit_elected(pv_done0 + 8 * g);
            return true;
        };
        auto step = [&]() {
            if (++stage == C::kStages) {
                stage = 0;
                phase ^= 1u;
            }
        };
        // Two issuing warps: a tile of the other's stream is waited for and given back all the same.  A wait tells one phase of a stage from the
        // one before it only, so that a warp which left tiles out could take the landing of an older tile for that of its own, or,
        // while the other frees and fills the stage without it, fall two phases behind.
        auto pass = [&]() -> bool {
            if (!await(kv_full0 + 8 * stage, phase)) return false;
            if (lane == 0) mbar_arrive(kv_empty0 + 8 * stage);
            __syncwarp();
            step();
            return true;
        };
        EncoderBounds ahead = bounds_at(0);
        for (int32_t n = 0; n < n_units; ++n) {
            const Unit u = unit_at(n);
            const int32_t blocks = blocks_of(ahead);
            ahead = bounds_at(n + 1);
            const int n_tiles = (blocks + kTileBlocks - 1) / kTileBlocks;
            const bool apart = u.two && !u.shared;
            shared = u.shared;
            if (kStreams == 1 && my_g == 1 && !u.two) {
                for (int j = 0; j < n_tiles; ++j)
                    if (!pass()) goto stopped;
                continue;
            }
            for (int j = 0; j < n_tiles; ++j) {
                const uint32_t nch = (uint32_t)min(kTileBlocks, blocks - j * kTileBlocks), idesc_s = make_idesc(kQRows, nch * 16, 0);
                // Two S buffers and shared tiles: S first, to run while the softmax of the tile before finishes.  One buffer: P V first,
                // as this S overwrites its P; tiles of the streams' own, too: the stage it frees is what the next tile waits for.
                const bool s_first = C::kSBufs == 2 && !apart;
#pragma unroll
                for (int i = 0; i < kStreams; ++i) {
                    const int g = kStreams == 2 ? i : my_g;
                    if (kStreams == 2 && i == 1 && !u.two) continue;
                    if (kStreams == 1 && apart && g == 1 && !pass()) goto stopped;   // (stream A's tile)
                    const uint32_t qb = qbuf_of(un[i] - (j == 0 ? 0u : 1u));
                    if (j == 0) {
                        if (!await(q_full0 + 16 * g + 8 * qb, qpar_of(un[i]))) goto stopped;
                        ++un[i];
                    }
                    if (!s_first && j > 0 && !issue_pv(i, 0u)) goto stopped;
                    if (!(u.shared && i == 1)) {   // (one issuer: the second stream of a shared tile finds it landed)
                        if (!await(kv_full0 + 8 * stage, phase)) goto stopped;
                        if (kHeld || j == n_tiles - 1) fence_async_smem();   // (a tile that warps wrote, or may have written a part of)
                    }
                    tc_fence_after();
                    const uint32_t buf = buf_of(t[i]);
                    umma_s<D, C::kQHalfBytes, C::kKVHalfBytes>(tmem + C::kSCol + (g * C::kSBufs + buf) * kKT, q_lo0 + (g * C::kQBufs + qb) * kQLo,
                                                              k_lo0 + stage * kStageLo, kDescHi, idesc_s, s_full0 + 16 * g + 8 * buf);
                    if (s_first && j > 0 && !issue_pv(i, 0u)) goto stopped;
                    pv_stage[i] = stage;
                    pv_nch[i] = nch;
                    pv_first[i] = j == 0;
                    ++t[i];
                    if (kStreams == 2 && apart && i == 0) step();
                }
                step();
                if (kStreams == 1 && apart && my_g == 0 && !pass()) goto stopped;    // (stream B's tile)
            }
            // The last P V of the unit does not wait for the next unit's first S: its output is due.
#pragma unroll
            for (int i = 0; i < kStreams; ++i)
                if (n_tiles > 0 && !(kStreams == 2 && i == 1 && !u.two) && !issue_pv(i, 1u)) goto stopped;
        }
    stopped:;
    } else {
        // ------------------------------------------------------------ softmax and output (warps 0-7)
        const int g = warp >> 2, wq = warp & 3, r = wq * 32 + lane;
        const uint32_t lane_base = ((uint32_t)(wq * 32)) << 16;
        const uint32_t s_tmem0 = tmem + C::kSCol + g * C::kSBufs * kKT + lane_base, o_tmem = tmem + C::kOCol + g * D + lane_base;
        const bool q_loader = wq == 0 && lane == 0;
        // the output rows start on 32-byte boundaries (the interface only promises 16)
        const bool o_sectors = ((reinterpret_cast<uintptr_t>(O) | (uintptr_t)(2 * o_row) | (uintptr_t)(2 * o_head) | (uintptr_t)(2 * o_tok)) & 31u) == 0;
        uint32_t q_asked = 0;     // query tiles requested
        int32_t q_next = 0;       // first unit not yet searched for one
        // (one lane) the queries of the first unit from q_next on that has any; `at_next` is what is known of unit q_next's row
        auto load_next_q = [&](EncoderBounds at_next) {
            while (q_next < n_units) {
                const Unit u = unit_at(q_next);
                const bool none = (g == 1 && !u.two) || blocks_of(at_next) == 0;
                ++q_next;
                if (none) {
                    at_next = bounds_at(q_next);
                    continue;
                }
                if (C::kBulkOut && !q_place_free(g, q_asked)) {
                    report(status, kStatusSyncTimeout, abort_flag);
                    return;
                }
                load_q(u, g, q_asked);
                ++q_asked;
                return;
            }
        };
        if (q_loader) {
            prefetch_tensormap(&q_map);
            if (C::kBulkOut) prefetch_tensormap(&o_map);
            if (!C::kLoaderQ) load_next_q(bounds_at(0));
        }
        __syncwarp();
        uint32_t t = 0, un = 0;   // tiles and units of this stream
        bool ok = true, to_release = false;
        EncoderBounds ahead = bounds_at(0);
        auto release_q = [&]() {   // the output of the last unit leaves the place of its queries to the next ones
            if (to_release) {
                if (lane == 0) {
                    bulk_wait_read<0>();
                    mbar_arrive(q_free0 + 16 * g + 8 * qbuf_of(C::kQBufs == 2 ? un + 1u : 0u));
                }
                if (!C::kLoaderQ && q_loader) load_next_q(ahead);   // (of unit n + 1 = q_next)
                __syncwarp();
                to_release = false;
            }
        };
        for (int32_t n = 0; ok && n < n_units; ++n) {
            const Unit u = unit_at(n);
            const int32_t len = ahead.len(enc), blocks = blocks_of(ahead);
            ahead = bounds_at(n + 1);
            if (g == 1 && !u.two) continue;
            const int n_tiles = (blocks + kTileBlocks - 1) / kTileBlocks;
            const int32_t valid_rows = min(kQRows, T - u.qt(g) * kQRows);
            const bool warp_live = wq * 32 < valid_rows;
            float m_ref = 0.f, l = 0.f, nb = 0.f;
            for (int j = 0; j < n_tiles; ++j, ++t) {
                const uint32_t buf = buf_of(t), s_tmem = s_tmem0 + buf * kKT;
                if (!__all_sync(0xffffffffu, mbar_wait(s_full0 + 16 * g + 8 * buf, par_of(t), abort_flag))) {
                    report(status, kStatusSyncTimeout, abort_flag);
                    ok = false;
                    break;
                }
                tc_fence_after();
                if (!C::kBulkOut && j == n_tiles - 1 && q_loader) load_next_q(ahead);   // the last S has landed: its queries are no longer read
                if (warp_live) {
                    const int groups = min(kTileBlocks, blocks - j * kTileBlocks);
                    uint64_t keep = ~0ull;   // a bit per column that holds a key
                    if (kHeld) {
                        if (j < kHeldTab) {
                            keep = mask_tab[j];
                        } else {
                            keep = held_tile(held, j, nullptr);
                        }
                    } else if (len - j * kKT < kKT) {
                        keep = (1ull << (len - j * kKT)) - 1ull;
                    }
                    uint32_t sr[kKT];
                    tmem_ld64(s_tmem, sr);
                    if (keep != ~0ull) {
                        const uint32_t lo = (uint32_t)keep, hi = (uint32_t)(keep >> 32);
#pragma unroll
                        for (int i = 0; i < kKT; ++i)
                            if ((((i < 32 ? lo : hi) >> (i & 31)) & 1u) == 0u) sr[i] = 0xff800000u;  // -inf
                    }
                    auto tile_max = [&]() -> float {
                        float mx[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) mx[c] = max3(__uint_as_float(sr[c]), __uint_as_float(sr[4 + c]), __uint_as_float(sr[8 + c]));
#pragma unroll
                        for (int i = 12; i < kKT - 4; i += 8)
#pragma unroll
                            for (int c = 0; c < 4; ++c) mx[c] = max3(mx[c], __uint_as_float(sr[i + c]), __uint_as_float(sr[i + 4 + c]));
#pragma unroll
                        for (int c = 0; c < 4; ++c) mx[c] = fmaxf(mx[c], __uint_as_float(sr[kKT - 4 + c]));
                        return fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
                    };
                    if (j == 0) {
                        m_ref = tile_max();
                        nb = fmaf(-m_ref, scale_log2, -kLowered);
                    }
                    // P over S, bf16 (the type of V) for the product; the sums take the probabilities as they are.  Blocks behind the last one
                    // are not read by the product and keep stale bits.
                    auto exp_tile = [&]() -> float {
                        float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
                        for (int grp = 0; grp < kTileBlocks; ++grp) {
                            if (grp < groups) {
                                uint32_t pk[8];
#pragma unroll
                                for (int ii = 0; ii < 8; ++ii) {
                                    const int i = grp * 8 + ii, c = 2 * i;
                                    float x0, x1, p0, p1;
                                    fma2(x0, x1, __uint_as_float(sr[c]), __uint_as_float(sr[c + 1]), scale_log2, scale_log2, nb, nb);
                                    if (C::kPolyEvery > 0 && i % (C::kPolyEvery > 0 ? C::kPolyEvery : 1) == 0) {
                                        exp2_poly2_nan(p0, p1, x0, x1);
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
                        return sum0 + sum1;
                    };
                    float tile_sum = exp_tile();
                    // (the polynomial ends at 2^126, so that it cannot hide a row that has outgrown its reference)
                    const bool over = !(tile_sum <= kSumLimit);
                    if (__any_sync(0xffffffffu, over)) {
                        // Rare.  The P V before must be done: with one S buffer it was issued before this S, whose arrival covers it; with two it
                        // has an arrival of its own (the next one needs the P that this tile has not announced yet).
                        if (C::kSBufs == 2 && j > 0) {
                            if (!__all_sync(0xffffffffu, mbar_wait(pv_done0 + 8 * g, (t - 1u) & 1u, abort_flag))) {
                                report(status, kStatusSyncTimeout, abort_flag);
                                ok = false;
                                break;
                            }
                            tc_fence_after();
                        }
                        tmem_wait_st();
                        const float mt = tile_max();
                        float alpha = 1.f;
                        if (over || fmaf(mt, scale_log2, nb) > kRescaleLog2 - kLowered) {
                            if (m_ref != mt) alpha = fast_exp2((m_ref - mt) * scale_log2);
                            m_ref = mt;
                            nb = mt == -INFINITY ? -kLowered : fmaf(-mt, scale_log2, -kLowered);
                            l *= alpha;
                        }
                        if (j > 0) {
#pragma unroll 1
                            for (int cb = 0; cb < D / 8; ++cb) {
                                uint32_t o[8];
                                tmem_ld8(o_tmem + cb * 8, o);
#pragma unroll
                                for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                tmem_st8(o_tmem + cb * 8, o);
                            }
                        }
                        tile_sum = exp_tile();
                        // Scores of minus infinity alone so far: probabilities and a sum of 0.  An infinite term makes the next tile's sum infinite or no
                        // number, whatever its scores are, and brings the row here again.
                        if (m_ref == -INFINITY) nb = INFINITY;
                    }
                    l += tile_sum;
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full0 + 16 * g + 8 * buf);
                if (C::kBulkOut && C::kQBufs == 2 && j == 0) release_q();   // (of the unit before)
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
            if (!C::kBulkOut && warp_live && n_tiles > 0) {
                const float inv = l > 0.f ? 1.f / l : 0.f;   // (no key but those of minus infinity: zeros)
                __nv_bfloat16* dst = O + u.row * o_row + u.head(g) * o_head + (int64_t)(u.qt(g) * kQRows + r) * o_tok;
#pragma unroll
                for (int cb = 0; cb < D / 32; ++cb) {
                    uint32_t o[32];
                    tmem_ld32(o_tmem + cb * 32, o);
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
            } else if (warp_live && n_tiles > 0) {
                // Through the place of the unit's queries, which nobody reads any more, and out as one bulk copy per 64 channels: stores straight
                // from the registers, a row per thread, take a memory transaction for every 32 bytes.  Rows past T are outside the tensor.
                const float inv = l > 0.f ? 1.f / l : 0.f;   // (no key but those of minus infinity: zeros)
                const uint32_t place = q_smem + (g * C::kQBufs + qbuf_of(un - 1u)) * C::kQBytes + wq * 32 * 128;
                uint8_t* mine = smem_raw + (place - raw) + lane * 128;
                constexpr int kCols = kHeld ? 32 : 64;   // (as many at a time as there are registers for)
#pragma unroll
                for (int cb = 0; cb < D; cb += kCols) {
                    uint32_t o[kCols];
                    if constexpr (kCols == 64) tmem_ld64(o_tmem + cb, o);
                    else tmem_ld32(o_tmem + cb, o);
#pragma unroll
                    for (int c = 0; c < kCols / 8; ++c) {
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(o[8 * c + 2 * i]) * inv, __uint_as_float(o[8 * c + 2 * i + 1]) * inv);
                            w[i] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                        *reinterpret_cast<uint4*>(mine + (cb >> 6) * C::kQHalfBytes + ((((cb & 63) / 8 + c) ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    const int3 c = coords(opos, u.qt(g) * kQRows + wq * 32, u.head(g), u.row);
#pragma unroll
                    for (int h = 0; h < C::kHalves; ++h) tma_store_4d(&o_map, place + h * C::kQHalfBytes, h * 64, c.x, c.y, c.z);
                    bulk_commit();
                }
            } else if (warp_live && r < valid_rows) {   // a row without keys: zeros
                uint4* dst = reinterpret_cast<uint4*>(O + u.row * o_row + u.head(g) * o_head + (int64_t)(u.qt(g) * kQRows + r) * o_tok);
#pragma unroll
                for (int c = 0; c < D / 8; ++c) dst[c] = make_uint4(0, 0, 0, 0);
            }
            if (C::kBulkOut && n_tiles > 0) {
                to_release = true;
                if (C::kQBufs == 1) release_q();
            }
            tc_fence_before();   // the reads of O come before the arrival on p_full for the next unit's first tile
        }
        if (lane == 0) bulk_wait_all();   // the output is written before the CTA ends
        if (!C::kLoaderQ && q_loader && q_asked > 0) await_q(g, q_asked - 1u);
    }

    // ---------------------------------------------------------------- teardown
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {   // (the same for all threads) a launch that gave up: its products end before tensor memory is given back
        if (warp >= mma_warp && warp < mma_warp + C::kMmaWarps) {
            const uint32_t drained = smem_u32(&bars->drained[warp - mma_warp]);
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
    using C = TilesCfg<D, kHeld>;
    TilePlan plan;
    const int32_t nqt = (T + kQRows - 1) / kQRows;
    plan.heads = kv_heads * group;
    plan.sms = (uint32_t)sm_count;
    const int64_t streams = (int64_t)nqt * plan.heads, per_row = (streams + 1) / 2;
    if (T < 1 || (int64_t)rows * per_row > 0x3fffffffll) return cudaErrorInvalidValue;   // (indices one round of CTAs beyond are formed)
    plan.nqt.set(nqt);
    plan.group.set(group);
    plan.units_per_row.set((int32_t)per_row);
    plan.units = (int32_t)(rows * per_row);
    CUtensorMap qm;
    int pos[3];
    if (!tc_encode_q_map(Q, T, rows, plan.heads, D, kQRows, &qm, pos)) return cudaErrorNotSupported;
    CUtensorMap om, km, vm, vm16;
    int opos[3] = {1, 2, 3}, kpos[3] = {1, 2, 3}, vpos[3] = {1, 2, 3};
    memset(&om, 0, sizeof(om));
    if (C::kBulkOut && !tc_encode_q_map(O, T, rows, plan.heads, D, kOutRows, &om, opos)) return cudaErrorNotSupported;
    memset(&km, 0, sizeof(km));
    memset(&vm, 0, sizeof(vm));
    memset(&vm16, 0, sizeof(vm16));
    if (!kHeld) {
        const int32_t kv_rows = enc.row_maps ? rows : 1;
        if (!tc_encode_q_map(Strided{enc.K, enc.row, enc.head, enc.tok}, enc.keys, kv_rows, kv_heads, D, kKT, &km, kpos) ||
            !tc_encode_q_map(Strided{enc.V, enc.row, enc.head, enc.tok}, enc.keys, kv_rows, kv_heads, D, kKT, &vm, vpos) ||
            !tc_encode_q_map(Strided{enc.V, enc.row, enc.head, enc.tok}, enc.keys, kv_rows, kv_heads, D, kBlock, &vm16, vpos))
            return cudaErrorNotSupported;
    }
    static SharedMemoryOptIn opt_in;
    const cudaError_t oe = opt_in.ensure(attend_tiles_kernel<D, kHeld>, (int)C::kSmemBytes);
    if (oe != cudaSuccess) return oe;
    const int64_t slots = (int64_t)sm_count * C::kCtasPerSm, grid = std::min<int64_t>(plan.units, slots), rest = plan.units % slots;
    // Where SMs hold two CTAs and an eighth to two thirds of them have a unit in the last round, these must not share SMs: launched onto an
    // idle chip they do not, onto SMs that come free one by one they do.
    const bool uneven = C::kCtasPerSm == 2 && plan.units > slots && 8 * rest > slots && 3 * rest <= 2 * slots;
    return launch_kernel(!uneven, attend_tiles_kernel<D, kHeld>, dim3((unsigned)grid), dim3(C::kThreads), KernelMemory(C::kSmemBytes), stream, qm,
                         make_int3(pos[0], pos[1], pos[2]), om, make_int3(opos[0], opos[1], opos[2]), km, vm, vm16, make_int3(kpos[0], kpos[1], kpos[2]),
                         (__nv_bfloat16*)O.ptr, O.row, O.head, O.token, enc, held, T, plan,
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
