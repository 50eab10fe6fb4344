// Forward pass of the attention to states (rib_cross.cuh) for B200 (sm_100a): TMA loads, tcgen05 products with accumulators in tensor memory,
// softmax in registers.
//
// Work item = two tiles of up to 128 rows of one (context, kv head) group x one run of its key blocks of 128.  A persistent CTA walks items:
//     S = Q K^T           (M128, N = 128, or what the last block has rounded up to 16; K = 32 or 64 channels)
//     P = exp2((S - m) log2e / sqrt(d)), written over S as bf16
//     O (+)= P V          (A from tensor memory, V an MN-major tile)
// Two threads own a row, one for each half of a block's keys: four softmax warps on every sub-partition of the SM, which hide one another's waits.  The exponentials are what bounds it -
// 2 x 128 x 128 of them take 2048 cycles of the SM's special-function units -, and what keeps the warps from them is every other step of theirs, so there are two forms of the softmax.
//   Fast form (first pass over the items): the reference m of a row is the maximum of the item's first 32 keys (fewer where the block is cut), read by both threads, and stays; no maximum is kept and nothing is rescaled.
//   fp32 and bf16 carry 8 exponent bits, so weights up to 2^100 relative to the reference are as exact as those below 1.  A row whose sum says that its scores left that range (more than 69 above
//   the reference, in nats; infinities, NaN) or whose values overflowed makes its item be noted, and
//   Exact form (second pass of the same launch): a running maximum over both halves, which they tell each other through shared memory, and which moves, and with it O and the row's sum, when a
//   block exceeds it by more than 2^8 in the exponentials.  Its weights are held down by 2^8 times the number of states, so that no sum of them times values passes the largest value.
// An eighth of the exponentials is taken on the FMA pipe, which has the time: 256 x 256 tokens to 1024 states 127 us, with none 132, with a quarter 127; heads of 64, 128 x 128 tokens 41 and 44.
// (256 x 256 tokens to 1024 states, us: a thread to a row, blocks of 64 keys, one warp for all loads and products 170; the exact form for every item 179; the fast one, then without the FMA pipe, 135.)
// Three buffers of scores rotate among the (block, tile) units, so that the scores of one tile are taken under the other's exponentials, and an item's output
// is normalised and stored behind the exponentials of the next item's first block, when its last product is long complete.
//
// Roles (640 threads): warp 0 loads, warp 1 issues S, warps 2 and 3 P V of tile 0 and 1 (2: owns the tensor memory), warps 4-11 softmax and output of tile 0 (4-7 first half of
// the keys), 12-19 of tile 1.  Every wait is bounded (tests/test_cross_barriers.py is a model of them).
#include "rib_cross.cuh"

namespace rib {
namespace {

using namespace sm100;

constexpr int kThreads = 640, kRows = 128, kKeys = 128, kMaxRedo = 64;      // kMaxRedo: items that a CTA can note for the exact pass (more: all of its items are redone)
constexpr uint32_t kMaxStages = 4, kBuffers = 3, kTmemCols = 512, kColO = kBuffers * kKeys;

// kSFull, kPReady, kPVDone: 2 * tile + parity of the block (on_block): a parity wait cannot tell its own phase from one two phases on, so a barrier's next phase needs what the waiter does after
// this one.  kDrain: one per issuing warp.
enum Bar { kQFull = 0, kQEmpty = 2, kSFull = 4, kPReady = 8, kPVDone = 12, kDrain = 16, kKFull = 19, kKEmpty = kKFull + kMaxStages, kVFull = kKEmpty + kMaxStages, kVEmpty = kVFull + kMaxStages,
           kPair = kVEmpty + kMaxStages, kBars = kPair + 8 };       // kPair: 4 * tile + quarter of the rows
template <int DP> struct Cfg {
    static constexpr uint32_t kStages = DP == 32 ? kMaxStages : 3;
    static constexpr uint32_t kRow = DP * 2, kTileBytes = kRows * kRow;                          // 128 rows, or 128 keys
    static constexpr uint32_t kOutBytes = 32 * DP;                                                // a softmax warp's 32 rows of DP / 2 channels
    static constexpr uint32_t kOffQ = 0, kOffK = 4 * kTileBytes, kOffV = kOffK + kStages * kTileBytes, kOffOut = kOffV + kStages * kTileBytes, kOffSums = kOffOut + 16 * kOutBytes;
    static constexpr uint32_t kOffMaxima = kOffSums + 2 * 4 * kRows * 4;                          // sums: [2 item parities][2 tiles][2 halves][128]; maxima: the same of block parities
    static constexpr uint32_t kOffBar = kOffMaxima + 2 * 4 * kRows * 4, kOffMisc = kOffBar + kBars * 8, kOffRedo = kOffMisc + 16, kSmem = kOffRedo + kMaxRedo * 4 + 1024;
    static_assert(kSmem <= 232448, "shared memory of a CTA");
    static_assert(kColO + 2 * DP <= kTmemCols, "tensor memory has 512 columns");
};

struct Params {
    const int* lengths;
    __nv_bfloat16* out;
    float* lse;
    float *part_out, *part_lse;          // splits > 1: [splits][groups][rows][DP], [splits][groups][rows]
    int* status;
    int d, L, heads, kv_heads, G, rows_per_tile, tokens_per_tile, blocks_per_split, splits, items, vector, tma_out, exact_only;      // items: pairs of tiles x splits x groups
    int tokens, shared;                  // tokens of a context; shared: one context, several maps
    long long rows, groups;
    float scale_log2, inv_sqrt_d, bits;  // bits: the exact form's weights, up to 2^8 each, are held down by 2^bits
    FastDiv by_pairs, by_splits, by_kv, by_pixels, by_group;
    int pixels;
};

struct Item { int pair, split, group, context, kv, first, blocks, length; };      // first: key block

// blocks of a context's first `length` keys that belong to the split
__device__ __forceinline__ Item decode(const Params& p, int item)
{
    Item c;
    p.by_pairs.divmod(item, item, c.pair);
    p.by_splits.divmod(item, c.group, c.split);
    p.by_kv.divmod(c.group, c.context, c.kv);
    c.length = p.lengths ? min(max(p.lengths[c.context], 0), p.L) : p.L;
    c.first = c.split * p.blocks_per_split;
    c.blocks = max(0, min(c.first + p.blocks_per_split, (c.length + kKeys - 1) / kKeys) - c.first);
    return c;
}

// Where the rows of one of an item's tiles go: their first token and its context, their first head, split x groups + group.
struct Place { int token0, context, head0, group; };

// Of the item's j-th block: its keys, that number rounded up to 16 (the columns of its scores), and the columns of the first half of them.
struct Block { int keys, columns, half; };
__device__ __forceinline__ Block block_of(const Item& c, int j)
{
    Block b;
    b.keys = min(kKeys, c.length - (c.first + j) * kKeys);
    b.columns = (b.keys + 15) & ~15;
    b.half = ((b.columns >> 4) + 1) >> 1 << 4;
    return b;
}

// 2^x of a pair on the FMA pipe: 2^round(x) times a polynomial of degree 5 in what is left, which is 1 at 0 and off by 1e-7 on [-1/2, 1/2] (a fit of least largest error).  From 128 on and for NaN the result
// is NaN, so that the row is redone; below -127, infinities among them, it is 0.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ float2 exp2_pair(float2 x)
{
    const auto both = [](float v) { return make_float2(v, v); };
    x = make_float2(min_nan(max_nan(x.x, -127.f), 128.5f), min_nan(max_nan(x.y, -127.f), 128.5f));
    const float2 r = __fadd2_rn(x, both(12582912.f)), n = __fadd2_rn(r, both(-12582912.f)), f = __ffma2_rn(n, both(-1.f), x);      // (1.5 x 2^23: its last bits are the whole number)
    float2 y = __ffma2_rn(f, both(0.00132647238f), both(0.00967151299f));
    y = __ffma2_rn(f, y, both(0.0555073358f));
    y = __ffma2_rn(f, y, both(0.240222424f));
    y = __ffma2_rn(f, y, both(0.693147004f));
    y = __ffma2_rn(f, y, both(1.f));
    y = make_float2(__uint_as_float(__float_as_uint(y.x) + (__float_as_uint(r.x) << 23)), __uint_as_float(__float_as_uint(y.y) + (__float_as_uint(r.y) << 23)));
    return __ffma2_rn(x, both(0.f), y);                   // (the sum of a NaN's bits and its shifted ones is a number)
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
rib_cross_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_out,
                     const __grid_constant__ Params p)
{
    using C = Cfg<DP>;
    using T = CrossTile<DP>;
    constexpr uint32_t kStages = C::kStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
    auto bar = [&](int i) { return base + C::kOffBar + 8u * i; };
    // (blocks -1 and -2 have the parity that a barrier without a completed phase answers yes to)
    auto on_block = [&](int which, int tile, uint32_t block) { return bar(which + 2 * tile + (block & 1)); };
    auto parity = [](uint32_t block) { return (block >> 1) & 1; };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + C::kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + C::kOffMisc + 4);      // [1] stays 0: used by the drain waits
    int* redo_count = reinterpret_cast<int*>(base_ptr + C::kOffMisc + 12);                       // notes taken (duplicates included)
    volatile int* redo_list = reinterpret_cast<volatile int*>(base_ptr + C::kOffRedo);           // ordinals of items among this CTA's
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        abort_flag[0] = 0; abort_flag[1] = 0;
        *redo_count = 0;
        for (int i = 0; i < kBars; ++i) mbar_init(bar(i), i >= kPReady && i < kPVDone ? 8 : i >= kVEmpty ? 2 : 1);
        fence_barrier_init();
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
    }
    if (warp == 2) {
        tmem_alloc(base + C::kOffMisc, kTmemCols);
        tmem_relinquish();
    }
    // rows that the boxes of Q do not reach (G does not divide 128)
    for (int i = 0; i < 4; ++i) cross_zero_rows(base_ptr + C::kOffQ + i * C::kTileBytes, C::kRow, p.rows_per_tile, kRows, threadIdx.x, kThreads);
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    cudaGridDependencySynchronize();                      // it may have overtaken the kernel before
    uint32_t blk = 0, live = 0;                           // blocks and items (with blocks) so far
    uint32_t sb = warp == 3 || warp >= 12 ? 1u : 0u;      // score buffer of the next unit: (2 blk + tile) mod kBuffers
    uint32_t met = 0;                                     // times that the two warps of a row have met
    const int my_items = (int)blockIdx.x < p.items ? (p.items - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0;

    for (int pass = 0; pass < 2; ++pass) {
    const bool fast = pass == 0 && !p.exact_only;
    // pass 0: every item of this CTA; pass 1: the items noted by the fast form (all of them when the notes overflowed)
    const int noted = pass == 0 ? 0 : *redo_count;
    const bool all_items = pass == 0 || noted > kMaxRedo;
    const int count = all_items ? my_items : noted;
    auto item_at = [&](int i) { return (int)blockIdx.x + (all_items ? i : redo_list[i]) * (int)gridDim.x; };
    if (warp == 0) {
        // ============================================ loads
        const uint32_t first_blk = blk, first_live = live;      // (those of the pass before have all landed)
        uint32_t k_asked = blk, v_asked = blk, q_asked = live;
        for (int i = 0; i < count && ok; ++i) {
            const Item c = decode(p, item_at(i));
            if (!c.blocks) continue;
            const uint32_t buf = live & 1;
            if (live >= 2 && !mbar_wait_warp(bar(kQEmpty + buf), ((live >> 1) - 1) & 1, abort_flag, p.status)) { ok = false; break; }
            if (elect_one()) {
                mbar_arrive_expect_tx(bar(kQFull + buf), 2u * (uint32_t)p.rows_per_tile * C::kRow);
                for (int t = 0; t < 2; ++t)
                    tma_load_4d(base + C::kOffQ + (2 * buf + t) * C::kTileBytes, &tm_q, bar(kQFull + buf), 0, c.kv * p.G, (2 * c.pair + t) * p.tokens_per_tile, c.context);
            }
            __syncwarp();
            ++q_asked;
            for (int j = 0; j < c.blocks; ++j, ++blk) {
                const uint32_t st = blk % kStages, use = blk / kStages;
                const int key = (c.first + j) * kKeys;
                if (use > 0 && !mbar_wait_warp(bar(kKEmpty + st), (use - 1) & 1, abort_flag, p.status)) { ok = false; break; }
                if (elect_one()) {
                    mbar_arrive_expect_tx(bar(kKFull + st), C::kTileBytes);
                    tma_load_4d(base + C::kOffK + st * C::kTileBytes, &tm_k, bar(kKFull + st), 0, c.kv, key, c.context);
                }
                __syncwarp();
                ++k_asked;
                if (use > 0 && !mbar_wait_warp(bar(kVEmpty + st), (use - 1) & 1, abort_flag, p.status)) { ok = false; break; }
                if (elect_one()) {
                    mbar_arrive_expect_tx(bar(kVFull + st), C::kTileBytes);
                    tma_load_4d(base + C::kOffV + st * C::kTileBytes, &tm_v, bar(kVFull + st), 0, c.kv, key, c.context);
                }
                __syncwarp();
                ++v_asked;
            }
            ++live;
        }
        if (!ok) {      // gave up: copies in flight land before the CTA may exit
            for (uint32_t i = max(first_live, q_asked > 2 ? q_asked - 2 : 0u); i < q_asked; ++i) mbar_wait_warp(bar(kQFull + (i & 1)), (i >> 1) & 1, abort_flag + 1, p.status);
            for (uint32_t i = max(first_blk, k_asked > kStages ? k_asked - kStages : 0u); i < k_asked; ++i) mbar_wait_warp(bar(kKFull + i % kStages), (i / kStages) & 1, abort_flag + 1, p.status);
            for (uint32_t i = max(first_blk, v_asked > kStages ? v_asked - kStages : 0u); i < v_asked; ++i) mbar_wait_warp(bar(kVFull + i % kStages), (i / kStages) & 1, abort_flag + 1, p.status);
        }
    } else if (warp == 1) {
        // ============================================ S of both tiles
        for (int i = 0; i < count && ok; ++i) {
            const Item c = decode(p, item_at(i));
            if (!c.blocks) continue;
            const uint32_t buf = live & 1;
            if (!mbar_wait_warp(bar(kQFull + buf), (live >> 1) & 1, abort_flag, p.status)) { ok = false; break; }
            for (int j = 0; j < c.blocks && ok; ++j, ++blk) {
                const uint32_t st = blk % kStages;
                if (!mbar_wait_warp(bar(kKFull + st), (blk / kStages) & 1, abort_flag, p.status)) { ok = false; break; }
                const uint32_t idesc = idesc_bf16_f32(kRows, block_of(c, j).columns, false);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    // the scores overwrite the columns that P V of three units before, one of the other tile, reads P from: it has completed
                    const uint32_t before = blk - 2 + t;
                    if (!mbar_wait_warp(on_block(kPVDone, t ^ 1, before), parity(before), abort_flag, p.status)) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t q = smem_desc_at(T::kDesc, base + C::kOffQ + (2 * buf + t) * C::kTileBytes), k = smem_desc_at(T::kDesc, base + C::kOffK + st * C::kTileBytes);
#pragma unroll
                        for (int kk = 0; kk < DP / 16; ++kk) mma_ss(tmem + sb * kKeys, q + T::kStepK * kk, k + T::kStepK * kk, idesc, kk ? 1u : 0u);
                        mma_commit(on_block(kSFull, t, blk));
                        if (t == 1) {
                            mma_commit(bar(kKEmpty + st));
                            if (j == c.blocks - 1) mma_commit(bar(kQEmpty + buf));
                        }
                    }
                    __syncwarp();
                    sb = sb == kBuffers - 1 ? 0u : sb + 1;
                }
            }
            ++live;
        }
    } else if (warp < 4) {
        // ============================================ P V: warp 2 for tile 0, warp 3 for tile 1
        const int t = warp - 2;
        for (int i = 0; i < count && ok; ++i) {
            const Item c = decode(p, item_at(i));
            for (int j = 0; j < c.blocks; ++j, ++blk) {
                const uint32_t st = blk % kStages;
                const Block b = block_of(c, j);
                if (!mbar_wait_warp(bar(kVFull + st), (blk / kStages) & 1, abort_flag, p.status)) { ok = false; break; }
                if (b.keys < b.columns) {      // values behind the last key: weights of 0 times what lies there must not become NaN.  (Either warp, before its own product.)
                    cross_zero_rows(base_ptr + C::kOffV + st * C::kTileBytes, C::kRow, b.keys, b.columns, lane, 32);
                    fence_proxy_async();
                    __syncwarp();
                }
                // (the first product of an item overwrites O: the softmax warps have read it before they hand over P)
                if (!mbar_wait_warp(on_block(kPReady, t, blk), parity(blk), abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t v = smem_desc_at(T::kDesc, base + C::kOffV + st * C::kTileBytes);
                    constexpr uint32_t kIdesc = idesc_bf16_f32(kRows, DP, true);
                    const int k_steps = b.columns >> 4, first = b.half >> 4;
                    for (int kk = 0; kk < k_steps; ++kk)      // P of a half of the keys lies in the second half of its scores' columns
                        mma_ts(tmem + kColO + t * DP, tmem + sb * kKeys + 8 * kk + (kk >= first ? b.columns >> 1 : b.half >> 1), v + T::kStepRows * kk, kIdesc, (j || kk) ? 1u : 0u);
                    mma_commit(on_block(kPVDone, t, blk));
                    mma_commit(bar(kVEmpty + st));
                }
                __syncwarp();
                sb = sb == 0 ? 2u : sb - 1;
            }
        }
    } else {
        // ============================================ softmax and output: two threads to a row
        const int t = (warp - 4) >> 3, half = ((warp - 4) >> 2) & 1, quarter = warp & 3, pair_bar = (int)bar(kPair + 4 * t + quarter);
        const int row = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16, t_o = tmem + lanes + kColO + t * DP + half * (DP / 2);
        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
        const float threshold = 8.f / p.scale_log2;
        volatile float* const maxima = reinterpret_cast<volatile float*>(base_ptr + C::kOffMaxima) + t * 2 * kRows + row;        // [block parity][2 tiles][half][128]
        volatile float* const sums = reinterpret_cast<volatile float*>(base_ptr + C::kOffSums) + t * 2 * kRows + row;            // [item parity][2 tiles][half][128]
        int row_token, row_head;
        p.by_group.divmod(row, row_token, row_head);
        // Both halves of a row have come here: what either wrote before is there for the other.
        auto meet = [&]() -> bool {
            __syncwarp();
            if (lane == 0) mbar_arrive((uint32_t)pair_bar);
            return mbar_wait_warp((uint32_t)pair_bar, met++ & 1, abort_flag, p.status);
        };
        // Normalises and stores this thread's half of the channels of a row; O and both halves' sums are complete.
        // (Fast form: it notes items that have to be redone; what is stored of them now is overwritten then.)
        const int c0 = half * (DP / 2);
        auto output = [&](const Place& c, float m, uint32_t item_parity, int ordinal) {
            const float l = sums[item_parity * 4 * kRows] + sums[item_parity * 4 * kRows + kRows];
            const int token = c.token0 + row_token;
            const bool mine = row < p.rows_per_tile && token < p.tokens;
            const float inverse = p.splits > 1 && l == 0.f ? 0.f : __fdividef(1.f, l);      // (a run of keys that all weigh nothing adds nothing)
            float2 nothing = make_float2(0.f, 0.f);       // not 0: some output is no number or infinite
            if (p.tma_out) {
                if (lane == 0) bulk_wait_group_read<0>();      // the rows of before have left
                __syncwarp();
            }
            uint8_t* const stage = base_ptr + C::kOffOut + (warp - 4) * C::kOutBytes + lane * DP;
            const int swizzle = DP == 32 ? (lane >> 2) & 1 : (lane >> 1) & 3;
#pragma unroll
            for (int g = 0; g < DP / 32; ++g) {           // 16 channels at a time
                uint32_t o[16];
                float x[16];
                tmem_ld16(t_o + 16 * g, o);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = inverse == 0.f ? 0.f : __uint_as_float(o[e]) * inverse;
                if (fast) {
#pragma unroll
                    for (int e = 0; e < 16; e += 2) nothing = __ffma2_rn(make_float2(__uint_as_float(o[e]), __uint_as_float(o[e + 1])), make_float2(0.f, 0.f), nothing);
                }
                if (p.tma_out) {
                    // (stores of threads that have a row each touch 32 lines apiece and held up the load-store unit for 1500 to 2900 cycles an item)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        *reinterpret_cast<uint4*>(stage + (((2 * g + k) ^ swizzle) << 4)) = make_uint4(pack_bf16x2(x[8 * k], x[8 * k + 1]), pack_bf16x2(x[8 * k + 2], x[8 * k + 3]),
                                                                                                   pack_bf16x2(x[8 * k + 4], x[8 * k + 5]), pack_bf16x2(x[8 * k + 6], x[8 * k + 7]));
                } else if (mine && p.splits > 1) {
                    float* const part = p.part_out + ((long long)c.group * p.rows + token * p.G + row_head) * DP + c0 + 16 * g;
#pragma unroll
                    for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4*>(part + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                } else if (mine) {
                    cross_store_row(p.out + ((long long)(c.context * p.tokens + token) * p.heads + c.head0 + row_head) * p.d, c0 + 16 * g, p.d, x, p.vector != 0);
                }
                __syncwarp();
            }
            if (p.tma_out) {
                fence_proxy_async();
                __syncwarp();
                if (lane == 0 && mine && c0 < p.d) {           // (mine: of the warp's first row; if that is no token, none is)
                    tma_store_4d(&tm_out, base + C::kOffOut + (warp - 4) * C::kOutBytes, c0, c.head0, token, c.context);
                    bulk_commit_group();
                }
            }
            if (fast) {
                // a score left the range that the fixed reference covers, or weights times values overflowed, for which a weight above those of the item's first keys is enough: looked for in every row
                const bool bad = mine && (!(l > 0.f && l < 0x1p100f) || nothing.x + nothing.y != 0.f);
                if (__any_sync(0xffffffffu, bad) && lane == 0) {
                    const int slot = atomicAdd(redo_count, 1);
                    if (slot < kMaxRedo) redo_list[slot] = ordinal;
                }
            }
            if (mine && half == 0) {
                const float lse = m * p.inv_sqrt_d + (__logf(l) + (fast ? 0.f : p.bits * 0.6931471805599453f));
                if (p.splits > 1) {
                    p.part_lse[(long long)c.group * p.rows + token * p.G + row_head] = l == 0.f ? -INFINITY : lse;
                } else if (p.lse) {
                    int image = c.context, pixel = token;
                    if (p.shared) p.by_pixels.divmod(token, image, pixel);
                    p.lse[(long long)(image * p.heads + c.head0 + row_head) * p.pixels + pixel] = lse;
                }
            }
            __syncwarp();
        };
        // Rows of an item without keys.
        auto nothing_to_attend_to = [&](const Place& c) {
            const int token = c.token0 + row_token;
            if (row >= p.rows_per_tile || token >= p.tokens) return;
            if (p.splits > 1) {
                const long long at = (long long)c.group * p.rows + token * p.G + row_head;
                if (half == 0) p.part_lse[at] = -INFINITY;
#pragma unroll 1
                for (int e = c0; e < c0 + DP / 2; ++e) p.part_out[at * DP + e] = 0.f;
                return;
            }
            const int head = c.head0 + row_head;
            __nv_bfloat16* dst = p.out + ((long long)(c.context * p.tokens + token) * p.heads + head) * p.d;
#pragma unroll 1
            for (int e = c0; e < min(p.d, c0 + DP / 2); ++e) dst[e] = __float2bfloat16_rn(0.f);
            if (p.lse && half == 0) {
                int image = c.context, pixel = token;
                if (p.shared) p.by_pixels.divmod(token, image, pixel);
                p.lse[(long long)(image * p.heads + head) * p.pixels + pixel] = -INFINITY;
            }
        };
        auto largest = [](const uint32_t (&s)[32]) {
            float mx[4] = {kCrossLowest, kCrossLowest, kCrossLowest, kCrossLowest};
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
#pragma unroll
                for (int i = 0; i < 4; ++i) mx[i] = max3(mx[i], __uint_as_float(s[e + 2 * i]), __uint_as_float(s[e + 2 * i + 1]));
            }
            return fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
        };
        int pending = -1;                                 // the item whose output is still to be stored (its number among those of the pass), where its rows go, and its reference
        Place before{};
        float m_before = 0.f;
        const int warp_token = __shfl_sync(0xffffffffu, row_token, 0);
        // (The code of the output stands once: behind the first block of an item, and behind the last item once more without one.  Twice the code, three sites, missed the instruction
        // cache on every fourth fetch.)
#pragma unroll 1
        for (int i = 0; i <= count && ok; ++i) {
            const bool last = i == count;
            const Item c = decode(p, item_at(last ? 0 : i));
            const Place here{(2 * c.pair + t) * p.tokens_per_tile, c.context, c.kv * p.G, c.split * (int)p.groups + c.group};
            if (!last && !c.blocks) { nothing_to_attend_to(here); continue; }
            if (last && pending < 0) break;
            // (rows of a warp that are no tokens take part in the waits alone; what they leave behind is nobody's)
            const bool idle = here.token0 + warp_token >= p.tokens || quarter * 32 >= p.rows_per_tile;
            float m = 0.f, l = 0.f;
#pragma unroll 1
            for (int j = 0; j < (last ? 1 : c.blocks); ++j, ++blk) {
                if (!last) {
                const Block b = block_of(c, j);
                if (!mbar_wait_warp(on_block(kSFull, t, blk), parity(blk), abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
                const uint32_t t_block = tmem + lanes + sb * kKeys, t_s = t_block + (half ? b.half : 0);
                sb = sb == 0 ? 2u : sb - 1;
                const int columns = half ? b.columns - b.half : b.half, keys = half ? b.keys - b.half : min(b.keys, b.half);      // of this half: up to 64; may be none
                if (fast) {
                    if (j == 0 && !idle) {      // the item's reference, the same for both halves: of keys whose scores the first half does not write P over
                        uint32_t a[32];
                        tmem_ld32(t_block, a);
                        tmem_wait_ld();
                        const int count = min(b.keys, b.half >> 1);
                        if (count < 32) {
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (e >= count) a[e] = 0xff800000u;
                        }
                        m = largest(a);
                    }
                } else {
                    // (the scores are read twice, for their maximum and for the exponentials: 64 of them and P do not fit a thread's registers)
                    float most = kCrossLowest;
                    if (!idle && columns == 64 && keys == 64) {
                        uint32_t a[2][32];
                        tmem_ld32(t_s, a[0]);
                        tmem_ld32(t_s + 32, a[1]);
                        tmem_wait_ld();
                        most = fmaxf(largest(a[0]), largest(a[1]));
                    } else if (!idle) {
    #pragma unroll 1
                        for (int g = 0; g < columns; g += 32) {
                            uint32_t a[32];
                            tmem_ld32(t_s + g, a);
                            tmem_wait_ld();
    #pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (g + e >= keys) a[e] = 0xff800000u;
                            most = fmaxf(most, largest(a));
                        }
                    }
                    maxima[(blk & 1) * 4 * kRows + half * kRows] = most;
                    if (!meet()) { ok = false; break; }
                    most = fmaxf(most, maxima[(blk & 1) * 4 * kRows + (half ^ 1) * kRows]);
                    if (j == 0) {
                        m = most;
                    } else {
                        // The reference moves, and O and l with it, only when the maximum grew by more than the threshold: the result is exact after the division since l carries the
                        // same reference.
                        const bool need = most > m + threshold;
                        if (__any_sync(0xffffffffu, need)) {
                            if (!mbar_wait_warp(on_block(kPVDone, t, blk - 1), parity(blk - 1), abort_flag, p.status)) { ok = false; break; }
                            tc_fence_after();
                            const float factor = need ? ex2_approx((m - most) * p.scale_log2) : 1.f;
                            if (need) { l *= factor; m = most; }
    #pragma unroll 1
                            for (int g = 0; g < DP / 16; ++g) {
                                uint32_t o[8];
                                tmem_ld8(t_o + 8 * g, o);
                                tmem_wait_ld();
    #pragma unroll
                                for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                                tmem_st8(t_o + 8 * g, o);
                            }
                        }
                    }
                }
                // (exact form: the difference first, which is exact at the largest score however large that is; otherwise scores beyond 1e9 lose their row to the rounding of -m scale, and come here)
                const float minus = fast ? 0.f : -m, below = fast ? -m * p.scale_log2 : -p.bits;
                const float2 minus2 = make_float2(minus, minus), neg2 = make_float2(below, below);
                float2 sum_a = make_float2(0.f, 0.f), sum_b = make_float2(0.f, 0.f);
                auto weights = [&](const uint32_t (&s)[16], uint32_t (&packed)[8], bool any) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 score = make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1]));
                        const float2 x = __ffma2_rn(any ? __fadd2_rn(score, minus2) : score, scale2, neg2);
                        const float2 e = i == 7 ? exp2_pair(x) : make_float2(ex2_approx(x.x), ex2_approx(x.y));
                        if (i & 1) sum_b = __fadd2_rn(sum_b, e); else sum_a = __fadd2_rn(sum_a, e);
                        packed[i] = pack_bf16x2(e.x, e.y);
                    }
                };
                // 64 keys, 16 at a time, the load of the next ones under the exponentials of these.  P goes into the second half of the columns, whose keys are therefore taken first, so that
                // it lies where scores have been read, and not where the other half reads the reference from.
                if (!idle && fast && columns == 64 && keys == 64) {
                    uint32_t a[16], b[16], packed[8];
                    tmem_ld16(t_s + 48, a);
                    tmem_ld16(t_s + 32, b);
                    tmem_wait_ld();
                    weights(a, packed, false);
                    tmem_st8(t_s + 56, packed);
                    tmem_ld16(t_s + 16, a);
                    weights(b, packed, false);
                    tmem_wait_ld();
                    tmem_st8(t_s + 48, packed);
                    tmem_ld16(t_s, b);
                    weights(a, packed, false);
                    tmem_wait_ld();
                    tmem_st8(t_s + 40, packed);
                    weights(b, packed, false);
                    tmem_st8(t_s + 32, packed);
                } else if (!idle) {
#pragma unroll 1
                    for (int g = columns - 16; g >= 0; g -= 16) {
                        uint32_t s[16], packed[8];
                        tmem_ld16(t_s + g, s);
                        tmem_wait_ld();
                        if (g + 16 > keys) {
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if (g + e >= keys) s[e] = 0xff800000u;
                        }
                        weights(s, packed, true);
                        tmem_st8(t_s + (columns + g) / 2, packed);
                    }
                }
                l += (sum_a.x + sum_a.y) + (sum_b.x + sum_b.y);
                tmem_wait_st();
                }
                if (j == 0 && pending >= 0) {
                    // that P V was the last one of the item before; the halves meet once more behind their sums of it (exact form: they have)
                    if (((fast || last) && !meet()) || !mbar_wait_warp(on_block(kPVDone, t, blk - 1), parity(blk - 1), abort_flag, p.status)) { ok = false; break; }
                    tc_fence_after();
                    output(before, m_before, (live - 1) & 1, pending);
                }
                if (last) break;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(on_block(kPReady, t, blk));
            }
            if (!ok || last) break;
            sums[(live & 1) * 4 * kRows + half * kRows] = l;
            pending = i;
            before = here;
            m_before = m;
            ++live;
        }
        if (p.tma_out && lane == 0) bulk_wait_group<0>();      // (the CTA's shared memory is read until then; and what the exact pass stores comes behind what this one did)
    }
    if (pass == 1 || !fast) break;                   // CTA-uniform: `fast` depends on the kernel arguments only
    // ---- between the passes: every role has finished its items; has the fast form noted any?
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const int notes = *redo_count;
    if (notes == 0 || abort_flag[0]) break;          // CTA-uniform: shared memory read after the barrier
    if (threadIdx.x == 0 && notes <= kMaxRedo) {
        // several warps may have noted the same item: keep each ordinal once
        int kept = 0;
        for (int a = 0; a < notes; ++a) {
            const int v = redo_list[a];
            bool seen = false;
            for (int b = 0; b < kept; ++b) seen = seen || redo_list[b] == v;
            if (!seen) redo_list[kept++] = v;
        }
        *redo_count = kept;
    }
    __syncthreads();
    }
    if (warp >= 1 && warp < 4) {
        // everything issued by this warp has finished before the tensor memory is released
        if (elect_one()) mma_commit(bar(kDrain + warp - 1));
        __syncwarp();
        mbar_wait_warp(bar(kDrain + warp - 1), 0, abort_flag + 1, p.status);
    }
    // ================================================================================ common tail
    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

// Joins the splits of a row: out = sum_s w_s out_s / sum_s w_s, w_s = exp(lse_s - max lse).  kLanes threads have eight channels of a row; with eight of them, from nine
// splits on, each takes every eighth split, and they meet in a fixed order.  (The forward pass with one / eight, us of the call alone: 16 x 16 tokens, heads of 32, 4 splits 17 / 28, 8 splits 17 / 21, 12 splits 18 / 20,
// 16 splits 18.6 / 19.2, 24 splits 19.4 / 18.8, 37 splits 23 / 18; one token, 6 heads, 64 splits of 8192 states 21 / 13.)
struct JoinParams {
    const float *part_out, *part_lse;
    const int* lengths;
    __nv_bfloat16* out;
    float* lse;
    int splits, stride, d, heads, kv_heads, G, chunks, vector, pixels;
    float down, up;                      // of the splits' weights: 2^-cross_bits(splits), and back
    long long groups, rows, tokens;
    FastDiv by_pixels;
};
template <int kLanes>
__global__ void __launch_bounds__(128) rib_cross_join_kernel(const JoinParams p)
{
    const long long thread = ((long long)blockIdx.x * 128 + threadIdx.x) / kLanes, all = p.groups * p.rows;
    const int part = threadIdx.x % kLanes;
    const bool mine = thread < all * p.chunks;           // (the others go along: lanes meet in shuffles)
    const long long at = mine ? thread / p.chunks : 0;
    const int chunk = mine ? (int)(thread - at * p.chunks) : 0;
    cudaGridDependencySynchronize();                     // it may have overtaken the kernel that computes the splits
    // eight splits' loads under way at once
    constexpr int kAtOnce = 8;
    float most = -INFINITY, total = 0.f, x[8];
    for (int s0 = part; s0 < p.splits; s0 += kAtOnce * kLanes) {
        float lse[kAtOnce];
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) lse[s] = s0 + s * kLanes < p.splits ? p.part_lse[(s0 + s * kLanes) * all + at] : -INFINITY;
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) most = fmaxf(most, lse[s]);
    }
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    for (int s0 = part; s0 < p.splits; s0 += kAtOnce * kLanes) {
        float lse[kAtOnce];
        float4 lo[kAtOnce], hi[kAtOnce];
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) {
            const int split = min(s0 + s * kLanes, p.splits - 1);
            lse[s] = s0 + s * kLanes < p.splits ? p.part_lse[split * all + at] : -INFINITY;
            const float4* src = reinterpret_cast<const float4*>(p.part_out + (split * all + at) * p.stride + 8 * chunk);
            lo[s] = src[0]; hi[s] = src[1];
        }
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) {
            if (lse[s] == -INFINITY) continue;           // (no keys, or none that weighs anything)
            const float w = expf(lse[s] - most) * p.down;
            total += w;
            x[0] += w * lo[s].x; x[1] += w * lo[s].y; x[2] += w * lo[s].z; x[3] += w * lo[s].w;
            x[4] += w * hi[s].x; x[5] += w * hi[s].y; x[6] += w * hi[s].z; x[7] += w * hi[s].w;
        }
    }
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += __shfl_xor_sync(0xffffffffu, x[e], o);
    }
    if (!mine || part) return;
    const long long group = at / p.rows, r = at - group * p.rows, token = r / p.G;
    const int context = (int)(group / p.kv_heads), head = (int)(group - (long long)context * p.kv_heads) * p.G + (int)(r - token * p.G);
    const bool none = p.lengths && p.lengths[context] <= 0;
    const float inverse = none ? 0.f : 1.f / total;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = none ? 0.f : x[e] * inverse;
    const long long pixel_of_all = (long long)context * p.tokens + token;
    sm100::cross_store_row(p.out + (pixel_of_all * p.heads + head) * p.d, 8 * chunk, p.d, x, p.vector != 0);
    if (p.lse && chunk == 0) {
        int image, pixel;
        p.by_pixels.divmod((int)pixel_of_all, image, pixel);
        p.lse[((long long)image * p.heads + head) * p.pixels + pixel] = none ? -INFINITY : most + logf(total * p.up);
    }
}

__global__ void __launch_bounds__(256) rib_cross_pad_kernel(const CrossPad args)
{
    cudaGridDependencySynchronize();                      // it may have overtaken the kernel before
    const __nv_bfloat16* src = args.src[blockIdx.y];
    __nv_bfloat16* dst = args.dst[blockIdx.y];
    const long long words = args.rows[blockIdx.y] * (args.width / 8);
    const int per = args.width / 8;
    for (long long w = (long long)blockIdx.x * 256 + threadIdx.x; w < words; w += (long long)gridDim.x * 256) {
        const long long row = w / per;
        const int c0 = 8 * (int)(w - row * per);
        uint32_t v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c0 + e < args.d) v[e >> 1] |= (uint32_t)__bfloat16_as_ushort(src[row * args.d + c0 + e]) << (16 * (e & 1));
        *reinterpret_cast<uint4*>(dst + row * args.width + c0) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

template <int DP>
cudaError_t launch_fwd(const CrossProblem& p, const CrossPlan& plan, float* part_out, float* part_lse, cudaStream_t stream)
{
    if (!encode_fn()) return cudaErrorNotSupported;
    CUtensorMap tm_q, tm_k, tm_v;
    if (!cross_rows_map(&tm_q, p.q, p.contexts, p.tokens, p.heads, p.width, DP, plan.G, plan.tokens_per_tile) ||
        !cross_rows_map(&tm_k, p.k, p.contexts, p.L, p.kv_heads, p.width, DP, 1, kKeys) || !cross_rows_map(&tm_v, p.v, p.contexts, p.L, p.kv_heads, p.width, DP, 1, kKeys))
        return cudaErrorInvalidValue;
    // rows of 16-byte words whose tokens fill whole warps, and no partial results: the output leaves by TMA, a warp's rows at a time
    const bool tma_out = p.d % 8 == 0 && 32 % plan.G == 0 && plan.splits == 1;
    CUtensorMap tm_out = tm_q;
    if (tma_out && !cross_rows_map(&tm_out, p.out_w, p.contexts, p.tokens, p.heads, p.d, DP / 2, plan.G, 32 / plan.G)) return cudaErrorInvalidValue;
    static KernelSetup setup;
    int sms = 0;
    if (cudaError_t e = setup.prepare(rib_cross_fwd_kernel<DP>, Cfg<DP>::kSmem, &sms)) return e;
    Params a{};
    a.lengths = p.lengths; a.out = p.out_w; a.lse = p.lse_w; a.part_out = part_out; a.part_lse = part_lse; a.status = p.status;
    a.d = p.d; a.L = p.L; a.heads = p.heads; a.kv_heads = p.kv_heads; a.G = plan.G; a.rows_per_tile = plan.rows_per_tile; a.tokens_per_tile = plan.tokens_per_tile;
    a.blocks_per_split = plan.blocks_per_split; a.splits = plan.splits; a.items = plan.groups * plan.splits * plan.pairs;
    a.vector = p.d % 8 == 0; a.tma_out = tma_out; a.exact_only = p.exact_softmax;
    a.tokens = (int)p.tokens; a.shared = p.tokens != p.pixels; a.rows = plan.rows; a.groups = plan.groups;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)p.d); a.inv_sqrt_d = 1.f / sqrtf((float)p.d); a.bits = 8.f + (float)cross_bits(p.L);
    a.by_pairs = make_fast_div(plan.pairs); a.by_splits = make_fast_div(plan.splits); a.by_kv = make_fast_div(p.kv_heads);
    a.by_pixels = make_fast_div((int)p.pixels); a.by_group = make_fast_div(plan.G); a.pixels = (int)p.pixels;
    const int grid = a.items < kCrossSms ? a.items : kCrossSms;
    ProfileScope scope(RIB_KERNEL_CROSS_FWD, stream);
    return launch_overtaking(rib_cross_fwd_kernel<DP>, grid, kThreads, Cfg<DP>::kSmem, stream, tm_q, tm_k, tm_v, tm_out, a);
}

cudaError_t join(const CrossProblem& p, const CrossPlan& plan, const float* part_out, const float* part_lse, int stride, cudaStream_t stream)
{
    JoinParams j{};
    j.part_out = part_out; j.part_lse = part_lse; j.lengths = p.lengths; j.out = p.out_w; j.lse = p.lse_w;
    j.splits = plan.splits; j.stride = stride; j.d = p.d; j.heads = p.heads; j.kv_heads = p.kv_heads; j.G = plan.G; j.chunks = (p.d + 7) / 8;
    j.vector = p.d % 8 == 0; j.pixels = (int)p.pixels; j.groups = plan.groups; j.rows = plan.rows; j.tokens = p.tokens; j.by_pixels = make_fast_div((int)p.pixels);
    j.up = (float)(1 << cross_bits(plan.splits)); j.down = 1.f / j.up;
    const bool eight = plan.splits > 8;
    const long long threads = j.groups * j.rows * j.chunks * (eight ? 8 : 1);
    ProfileScope scope(RIB_KERNEL_CROSS_JOIN, stream);
    return launch_overtaking(eight ? rib_cross_join_kernel<8> : rib_cross_join_kernel<1>, (unsigned)((threads + 127) / 128), 128, 0, stream, j);
}

int tile_width(int d) { return d <= 32 ? 32 : 64; }

struct FwdLayout { size_t q, k, v, part_out, part_lse, bytes; };
FwdLayout fwd_layout(const CrossProblem& p, const CrossPlan& plan)
{
    FwdLayout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += cross_align(bytes); return here; };
    if (cross_padded(p)) {
        const size_t width = (p.d + 7) / 8 * 8;
        l.q = take(2 * width * p.tokens * p.contexts * p.heads);
        l.k = take(2 * width * p.L * p.contexts * p.kv_heads);
        l.v = take(2 * width * p.L * p.contexts * p.kv_heads);
    }
    if (plan.splits > 1) {
        l.part_out = take(sizeof(float) * tile_width(p.d) * plan.splits * plan.groups * plan.rows);
        l.part_lse = take(sizeof(float) * plan.splits * plan.groups * plan.rows);
    }
    l.bytes = at;
    return l;
}

}  // namespace

bool cross_padded(const CrossProblem& p) { return p.d % 8 != 0; }

CrossPlan cross_plan(const CrossProblem& p)
{
    CrossPlan c{};
    auto tiled = [&](int rows, int* tokens_per_tile, int* rows_per_tile, int* tiles) {
        *tokens_per_tile = rows / c.G;
        if (*tokens_per_tile > p.tokens) *tokens_per_tile = (int)p.tokens;      // (a box is no larger than the tensor has to be)
        *rows_per_tile = *tokens_per_tile * c.G;
        *tiles = (int)((p.tokens + *tokens_per_tile - 1) / *tokens_per_tile);
    };
    c.G = p.heads / p.kv_heads;
    tiled(kRows, &c.tokens_per_tile, &c.rows_per_tile, &c.tiles);
    tiled(kCrossBlock, &c.kv_tokens_per_tile, &c.kv_rows_per_tile, &c.row_tiles);
    c.groups = p.contexts * p.kv_heads;
    c.rows = p.tokens * c.G;
    // Fewer items than SMs: the key blocks are dealt out to several CTAs, whose results are joined.
    auto split = [&](long long items, int blocks, int* splits, int* per) {
        long long n = items >= kCrossSms ? 1 : kCrossSms / items;
        if (n > blocks) n = blocks;
        *per = (int)((blocks + n - 1) / n);
        *splits = (blocks + *per - 1) / *per;
    };
    c.pairs = (c.tiles + 1) / 2;
    split((long long)c.groups * c.pairs, (p.L + kKeys - 1) / kKeys, &c.splits, &c.blocks_per_split);
    c.few_rows = c.rows <= kCrossFewRows;
    // Eight blocks to an SM, of 128 keys or more.  Four of them are resident, and the second four even out what lengths of their own leave idle.  Us with four / eight / sixteen: 64 contexts of 64 to 4096 states,
    // 6 heads of 32, 37 / 31 / 33; all of 4096 45 / 49 / 49; two rows there 47 / 35 / 35; 16 contexts of 256 to 4096, 2 heads of 64, 10 / 12 / 12; 16 of 63 to 1000, 6 heads of 32, 8 / 10 / 10; 256 contexts 35 / 35 / 37.
    if (c.few_rows) {
        const long long most = 8 * kCrossSms / c.groups, runs = (p.L + 127) / 128;
        c.splits = (int)(most < 1 ? 1 : most < runs ? most : runs);
    }
    c.dq_tiles = (c.row_tiles + 1) / 2;
    split((long long)c.groups * c.dq_tiles, (p.L + kCrossBlock - 1) / kCrossBlock, &c.dq_splits, &c.dq_blocks_per_split);
    // dK and dV: a CTA to an SM; runs of row tiles such that the last round of CTAs is not a mostly empty one.  In us: 0.5 a tile, 3 for what a CTA begins and ends with, and the way of
    // the partial sums to memory and back.  Where one kernel takes all three gradients, runs of pairs of tiles: 1.4 a pair and block of keys, 4.  (Nothing is known here of lengths.)
    c.key_tiles = (p.L + 127) / 128;
    c.short_bwd = p.L <= (p.d <= 32 ? 256 : 128);
    const long long units = c.short_bwd ? c.groups : (long long)c.groups * c.key_tiles;
    const int steps = c.short_bwd ? c.dq_tiles : c.row_tiles;
    const double step = c.short_bwd ? 1.4 * c.key_tiles : 0.5, ends = c.short_bwd ? 4 : 3;
    double best = 0;
    for (int s = 1; s <= steps && s <= 64; ++s) {
        const int per = (steps + s - 1) / s, used = (steps + per - 1) / per;
        if (used != s) continue;
        const double cost = (double)((units * s + kCrossSms - 1) / kCrossSms) * (step * per + ends) + (s > 1 ? 3 + s * (double)c.groups * p.L * (p.d <= 32 ? 32 : 64) * 16 / 4e6 : 0);
        if (s == 1 || cost < best) { best = cost; c.row_splits = s; c.row_tiles_per_split = c.short_bwd ? 2 * per : per; }
    }
    if (c.short_bwd) c.dq_splits = 1;
    return c;
}

cudaError_t cross_pad(const CrossPad& args, cudaStream_t stream)
{
    long long most = 0;
    for (int i = 0; i < args.tensors; ++i) most = args.rows[i] > most ? args.rows[i] : most;
    const long long blocks = (most * (args.width / 8) + 255) / 256;
    return launch_overtaking(rib_cross_pad_kernel, dim3((unsigned)(blocks < 4 * kCrossSms ? blocks : 4 * kCrossSms), (unsigned)args.tensors), 256, 0, stream, args);
}

size_t cross_fwd_workspace(const CrossProblem& p) { return fwd_layout(p, cross_plan(p)).bytes; }

cudaError_t cross_fwd(CrossProblem p, cudaStream_t stream, int* launches)
{
    const CrossPlan plan = cross_plan(p);
    const FwdLayout l = fwd_layout(p, plan);
    uint8_t* ws = static_cast<uint8_t*>(p.workspace);
    *launches = 1;
    p.width = p.d;
    if (cross_padded(p)) {
        CrossPad pad{};
        pad.tensors = 3; pad.d = p.d; pad.width = (p.d + 7) / 8 * 8;
        const __nv_bfloat16** src[3] = {&p.q, &p.k, &p.v};
        const size_t off[3] = {l.q, l.k, l.v};
        for (int i = 0; i < 3; ++i) {
            pad.src[i] = *src[i];
            pad.dst[i] = reinterpret_cast<__nv_bfloat16*>(ws + off[i]);
            pad.rows[i] = p.contexts * (i ? (long long)p.L * p.kv_heads : p.tokens * p.heads);
            *src[i] = pad.dst[i];
        }
        p.width = pad.width;
        if (cudaError_t e = cross_pad(pad, stream)) return e;
        ++*launches;
    }
    float *part_out = reinterpret_cast<float*>(ws + l.part_out), *part_lse = reinterpret_cast<float*>(ws + l.part_lse);
    const int stride = tile_width(p.d);
    cudaError_t e;
    if (plan.few_rows) e = cross_fwd_rows(p, plan, part_out, part_lse, stride, stream);
    else if (p.L <= kCrossShort) e = cross_fwd_short(p, plan, stream);
    else e = stride == 32 ? launch_fwd<32>(p, plan, part_out, part_lse, stream) : launch_fwd<64>(p, plan, part_out, part_lse, stream);
    if (e) return e;
    if (plan.splits > 1) {
        ++*launches;
        return join(p, plan, part_out, part_lse, stride, stream);
    }
    return cudaSuccess;
}

}  // namespace rib
