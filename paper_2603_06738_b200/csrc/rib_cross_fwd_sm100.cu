// Forward pass of the attention to states (rib_cross.cuh) for B200 (sm_100a): TMA loads, tcgen05 products with accumulators in tensor memory,
// softmax in registers.
//
// Work item = up to 128 rows of one (context, kv head) group x one run of its key blocks of 64.  A CTA of five warps walks items:
//     S = Q K^T           (M128, N = 64, or what the last block has rounded up to 16; K = 32 or 64 channels)
//     P = exp2((S - m) log2e / sqrt(d)), a row to a thread, written over S as bf16
//     O (+)= P V          (A from tensor memory, V an MN-major tile)
// with a running maximum m per row that moves, and rescales O and the row's sum, only when a block exceeds it by more than 2^8 in the exponentials.
// The key blocks of all items of a CTA are one stream of steps: three buffers of scores, so that the scores of the next two steps, which may belong to the next item, are there or under
// way while the softmax warps work, and an item's output is normalised and stored behind the exponentials of the next item's first block, when its last product is long complete.
// The exponentials bound it: 128 x 64 of them take 512 cycles of the SM's special-function units, the products about 130 (d = 32) to 260 cycles; two CTAs to an SM
// (256 columns of tensor memory each) fill one another's gaps.
//
// Roles: warps 0-3 softmax and output of rows 32 w .. 32 w + 31; warp 4 loads (query tiles, a ring of key blocks) and issues the products.  Every wait is bounded.
#include "rib_cross.cuh"

namespace rib {
namespace {

using namespace sm100;

constexpr int kThreads = 160, kRows = 128, kBlocksPerSm = 2;
constexpr uint32_t kBuffers = 3, kTmemCols = 256, kColO = kBuffers * kCrossBlock;

template <int DP> struct Cfg {
    static constexpr int kStages = DP == 32 ? 8 : 4, kTiles = DP == 32 ? 4 : 3;
    static constexpr uint32_t kRow = DP * 2, kQBytes = kRows * kRow, kKBytes = kCrossBlock * kRow;
    static constexpr uint32_t kOffQ = 0, kOffK = kTiles * kQBytes, kOffV = kOffK + kStages * kKBytes, kOffBar = kOffV + kStages * kKBytes;
    // barriers: query tiles, key blocks; of each buffer of scores: scores there, P there, P V done; all products done.  (A parity wait cannot tell its own phase
    // from one two phases on: a buffer's next phases need what the waiter does after this one.)
    static constexpr int kQFull = 0, kKFull = kTiles, kSFull = kKFull + kStages, kPReady = kSFull + kBuffers, kPVDone = kPReady + kBuffers, kDrain = kPVDone + kBuffers, kBars = kDrain + 1;
    static constexpr uint32_t kOffMisc = kOffBar + kBars * 8, kSmem = kOffMisc + 16;
    static_assert(kTiles >= (int)kBuffers && kStages > (int)kBuffers, "the scores of kBuffers steps, each of an item of its own, are taken before the first product");
    static_assert(kQBytes % 1024 == 0 && kKBytes % 1024 == 0, "swizzle atoms need aligned tiles");
    static_assert(kBlocksPerSm * (kSmem + 1024) <= 233472, "shared memory of an SM");
    static_assert(kColO + DP <= kTmemCols, "tensor memory of a CTA");
};

struct Params {
    const int* lengths;
    __nv_bfloat16* out;
    float* lse;
    float *part_out, *part_lse;          // splits > 1: [splits][groups][rows][DP], [splits][groups][rows]
    int* status;
    int d, L, heads, kv_heads, G, rows_per_tile, tokens_per_tile, blocks_per_split, splits, items, vector;
    long long tokens, rows, groups;
    float scale_log2, inv_sqrt_d;
    FastDiv by_tiles, by_splits, by_kv, by_pixels, by_group;
    int pixels;
};

struct Item { int tile, split, group, context, kv, first, blocks, length; };

// blocks of a context's first `length` keys that belong to the split
__device__ __forceinline__ Item decode(const Params& p, int item)
{
    Item c;
    p.by_tiles.divmod(item, item, c.tile);
    p.by_splits.divmod(item, c.group, c.split);
    p.by_kv.divmod(c.group, c.context, c.kv);
    c.length = p.lengths ? min(max(__ldg(p.lengths + c.context), 0), p.L) : p.L;
    c.first = c.split * p.blocks_per_split;
    c.blocks = max(0, min(c.first + p.blocks_per_split, (c.length + kCrossBlock - 1) / kCrossBlock) - c.first);
    return c;
}

// A place in the CTA's stream of steps (key blocks of its items, one item after the other; items without keys have none).
struct Cursor {
    Item c;
    int item, block;
    uint32_t step, live;                 // steps and items with steps before it
    __device__ __forceinline__ void settle(const Params& p)          // to the next item that has a block
    {
        while (item < p.items) {
            c = decode(p, item);
            if (c.blocks) return;
            item += gridDim.x;
        }
    }
    __device__ __forceinline__ void begin(const Params& p) { item = blockIdx.x; block = 0; step = live = 0; settle(p); }
    __device__ __forceinline__ bool there(const Params& p) const { return item < p.items; }
    __device__ __forceinline__ void advance(const Params& p)
    {
        ++step;
        if (++block < c.blocks) return;
        block = 0;
        ++live;
        item += gridDim.x;
        settle(p);
    }
    __device__ __forceinline__ int keys() const { return min(kCrossBlock, c.length - (c.first + block) * kCrossBlock); }
};

template <int DP>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
rib_cross_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ Params p)
{
    using C = Cfg<DP>;
    using T = CrossTile<DP>;
    constexpr int kStages = C::kStages, kTiles = C::kTiles;
    extern __shared__ __align__(1024) uint8_t base_ptr[];
    const uint32_t base = smem_u32(base_ptr);
    auto bar = [&](int i) { return base + C::kOffBar + 8u * i; };
    auto on_step = [&](int which, uint32_t step) { return bar(which + step % kBuffers); };
    auto parity = [](uint32_t step) { return (step / kBuffers) & 1; };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + C::kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + C::kOffMisc + 4);      // [1] stays 0: used by the drain waits
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (base & 1023u) {                                   // (never seen: the declaration above asks for it; swizzled tiles would be misread)
        if (threadIdx.x == 0) atomicExch(p.status, 1);
        return;
    }

    if (threadIdx.x == 0) {
        abort_flag[0] = 0; abort_flag[1] = 0;
        for (int i = 0; i < C::kBars; ++i) mbar_init(bar(i), i >= C::kPReady && i < C::kPVDone ? 4 : 1);
        fence_barrier_init();
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
    }
    if (warp == 4) {
        tmem_alloc(base + C::kOffMisc, kTmemCols);
        tmem_relinquish();
    }
    // rows that the boxes of Q do not reach (G does not divide 128)
    for (int i = 0; i < kTiles; ++i) cross_zero_rows(base_ptr + C::kOffQ + i * C::kQBytes, C::kRow, p.rows_per_tile, kRows, threadIdx.x, kThreads);
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;

    if (warp == 4) {
        // ============================================ loads and products: the whole warp walks, one elected lane issues
        Cursor load, score, value;                        // the next step to load, to take the scores of, to multiply with its values
        load.begin(p); score.begin(p); value.begin(p);
        uint32_t q_loaded = 0;
        // Loads as far ahead as there is room: a stage is free once its step's P V is complete (all before value.step are), a query tile once its item's
        // scores are (`scored` items).
        auto load_ahead = [&](uint32_t scored) {
            for (; load.there(p); load.advance(p)) {
                if (load.step == value.step + kStages) return;
                if (load.block == 0 && load.live == scored + kTiles) return;
                if (elect_one()) {
                    if (load.block == 0) {
                        const uint32_t buf = load.live % kTiles;
                        mbar_arrive_expect_tx(bar(C::kQFull + buf), (uint32_t)p.rows_per_tile * C::kRow);
                        tma_load_4d(base + C::kOffQ + buf * C::kQBytes, &tm_q, bar(C::kQFull + buf), 0, load.c.kv * p.G, load.c.tile * p.tokens_per_tile, load.c.context);
                    }
                    const uint32_t st = load.step % kStages;
                    const int key = (load.c.first + load.block) * kCrossBlock;
                    mbar_arrive_expect_tx(bar(C::kKFull + st), 2 * C::kKBytes);
                    tma_load_4d(base + C::kOffK + st * C::kKBytes, &tm_k, bar(C::kKFull + st), 0, load.c.kv, key, load.c.context);
                    tma_load_4d(base + C::kOffV + st * C::kKBytes, &tm_v, bar(C::kKFull + st), 0, load.c.kv, key, load.c.context);
                }
                __syncwarp();
                if (load.block == 0) ++q_loaded;
            }
        };
        // The scores of the next step, into the buffer whose P the product before the last one has read.
        auto issue_scores = [&]() -> bool {
            const uint32_t st = score.step % kStages, buf = score.live % kTiles;
            const int keys = score.keys(), columns = (keys + 15) & ~15;
            if ((score.block == 0 && !mbar_wait_warp(bar(C::kQFull + buf), (score.live / kTiles) & 1, abort_flag, p.status)) ||
                !mbar_wait_warp(bar(C::kKFull + st), (score.step / kStages) & 1, abort_flag, p.status)) return false;
            if (keys < columns) {      // values behind the last key: weights of 0 times what lies there must not become NaN
                cross_zero_rows(base_ptr + C::kOffV + st * C::kKBytes, C::kRow, keys, columns, lane, 32);
                fence_proxy_async();
                __syncwarp();
            }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t q = smem_desc_at(T::kDesc, base + C::kOffQ + buf * C::kQBytes), k = smem_desc_at(T::kDesc, base + C::kOffK + st * C::kKBytes);
                const uint32_t idesc = idesc_bf16_f32(kRows, columns, false), at = tmem + score.step % kBuffers * kCrossBlock;
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk) mma_ss(at, q + T::kStepK * kk, k + T::kStepK * kk, idesc, kk ? 1u : 0u);
                mma_commit(on_step(C::kSFull, score.step));
            }
            __syncwarp();
            score.advance(p);
            return true;
        };
        load_ahead(0);
        for (uint32_t i = 0; i < kBuffers && ok && score.there(p); ++i) ok = issue_scores();
        while (ok && value.there(p)) {
            // (the first product of an item overwrites O: the softmax warps have read it before they hand over P)
            if (!mbar_wait_warp(on_step(C::kPReady, value.step), parity(value.step), abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t v = smem_desc_at(T::kDesc, base + C::kOffV + (value.step % kStages) * C::kKBytes);
                constexpr uint32_t kIdesc = idesc_bf16_f32(kRows, DP, true);
                const int k_steps = (value.keys() + 15) / 16;
                const uint32_t at = tmem + value.step % kBuffers * kCrossBlock;
                for (int kk = 0; kk < k_steps; ++kk) mma_ts(tmem + kColO, at + 8 * kk, v + T::kStepRows * kk, kIdesc, (value.block || kk) ? 1u : 0u);
                mma_commit(on_step(C::kPVDone, value.step));
            }
            __syncwarp();
            // The product before this one is complete by now, or soon: its buffer takes the scores of the step after the next, and its stage another block.
            if (value.step > 0 && !mbar_wait_warp(on_step(C::kPVDone, value.step - 1), parity(value.step - 1), abort_flag, p.status)) { ok = false; break; }
            load_ahead(value.live + (value.block + 1 == value.c.blocks ? 1u : 0u));
            if (value.step > 0 && score.there(p)) ok = issue_scores();
            value.advance(p);
        }
        if (!ok) {      // gave up: copies in flight land before the CTA may exit (waiting for those that have been waited for is harmless)
            for (uint32_t i = value.step; i < load.step; ++i) mbar_wait_warp(bar(C::kKFull + i % kStages), (i / kStages) & 1, abort_flag + 1, p.status);
            for (uint32_t i = value.live; i < q_loaded; ++i) mbar_wait_warp(bar(C::kQFull + i % kTiles), (i / kTiles) & 1, abort_flag + 1, p.status);
        }
        // what has been issued is complete before the tensor memory is released
        if (elect_one()) mma_commit(bar(C::kDrain));
        __syncwarp();
        mbar_wait_warp(bar(C::kDrain), 0, abort_flag + 1, p.status);
    } else {
        // ============================================ softmax and output: a row to a thread
        const int row = threadIdx.x;
        const uint32_t lanes = (uint32_t)(warp * 32) << 16, t_o = tmem + lanes + kColO;
        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
        const float threshold = 8.f / p.scale_log2;
        int row_token, row_head;
        p.by_group.divmod(row, row_token, row_head);
        uint32_t step = 0;
        // Normalises and stores a row of the item; O is complete.
        auto output = [&](const Item& c, float m, float l) {
            const bool none = c.blocks == 0;
            const long long token = (long long)c.tile * p.tokens_per_tile + row_token;
            const bool mine = row < p.rows_per_tile && token < p.tokens;
            const float inverse = none || (p.splits > 1 && l == 0.f) ? 0.f : 1.f / l;      // (a run of keys that all weigh nothing adds nothing)
            const float lse = none ? -INFINITY : m * p.inv_sqrt_d + logf(l);
            const int head = c.kv * p.G + row_head;
            const long long at = ((long long)c.split * p.groups + c.group) * p.rows + token * p.G + row_head;
            __nv_bfloat16* dst = p.out + (((long long)c.context * p.tokens + token) * p.heads + head) * p.d;
#pragma unroll
            for (int g = 0; g < DP / 32; ++g) {
                uint32_t o[32];
                float x[32];
                if (!none) { tmem_ld32(t_o + 32 * g, o); tmem_wait_ld(); }
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = none || inverse == 0.f ? 0.f : __uint_as_float(o[e]) * inverse;
                if (mine && p.splits > 1) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(p.part_out + at * DP + 32 * g + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                } else if (mine) {
                    cross_store_row(dst, 32 * g, p.d, x, p.vector != 0);
                }
                __syncwarp();
            }
            if (mine && p.splits > 1) {
                p.part_lse[at] = l == 0.f ? -INFINITY : lse;
            } else if (mine && p.lse) {
                int image, pixel;
                p.by_pixels.divmod((int)(c.context * p.tokens + token), image, pixel);
                p.lse[((long long)image * p.heads + head) * p.pixels + pixel] = lse;
            }
        };
        int pending = -1;                                 // the item whose output is still to be stored, with its reference and sum
        float m_before = 0.f, l_before = 0.f;
        for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            const Item c = decode(p, item);
            if (!c.blocks) { output(c, 0.f, 0.f); continue; }
            float m = 0.f, l = 0.f;
            for (int j = 0; j < c.blocks; ++j, ++step) {
                if (!mbar_wait_warp(on_step(C::kSFull, step), parity(step), abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
                const uint32_t t_s = tmem + lanes + step % kBuffers * kCrossBlock;
                uint32_t a[64];
                tmem_ld32(t_s, *reinterpret_cast<uint32_t(*)[32]>(a));
                tmem_ld32(t_s + 32, *reinterpret_cast<uint32_t(*)[32]>(a + 32));
                tmem_wait_ld();
                const int keys = c.length - (c.first + j) * kCrossBlock;
                if (keys < kCrossBlock) {
#pragma unroll
                    for (int e = 0; e < 64; ++e)
                        if (e >= keys) a[e] = 0xff800000u;
                }
                float mx[4] = {kCrossLowest, kCrossLowest, kCrossLowest, kCrossLowest};
#pragma unroll
                for (int e = 0; e < 64; e += 8) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx[i] = max3(mx[i], __uint_as_float(a[e + 2 * i]), __uint_as_float(a[e + 2 * i + 1]));
                }
                const float most = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
                if (j == 0) {
                    m = most;
                } else {
                    // The reference moves, and O and l with it, only when the maximum grew by more than the threshold: the result is exact after
                    // the division since l carries the same reference.
                    const bool need = most > m + threshold;
                    if (__any_sync(0xffffffffu, need)) {
                        if (!mbar_wait_warp(on_step(C::kPVDone, step - 1), parity(step - 1), abort_flag, p.status)) { ok = false; break; }
                        tc_fence_after();
                        const float factor = need ? ex2_approx((m - most) * p.scale_log2) : 1.f;
                        if (need) { l *= factor; m = most; }
#pragma unroll
                        for (int g = 0; g < DP / 8; ++g) {
                            uint32_t o[8];
                            tmem_ld8(t_o + 8 * g, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                            tmem_st8(t_o + 8 * g, o);
                        }
                    }
                }
                const float2 neg2 = make_float2(-m * p.scale_log2, -m * p.scale_log2);
                float2 sum_a = make_float2(0.f, 0.f), sum_b = make_float2(0.f, 0.f);
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    if (16 * g >= keys) break;            // (the product takes the keys there are, rounded up to 16)
                    uint32_t packed[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 x = __ffma2_rn(make_float2(__uint_as_float(a[16 * g + 2 * i]), __uint_as_float(a[16 * g + 2 * i + 1])), scale2, neg2);
                        const float2 e = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                        if (i & 1) sum_b = __fadd2_rn(sum_b, e); else sum_a = __fadd2_rn(sum_a, e);
                        packed[i] = pack_bf16x2(e.x, e.y);
                    }
                    tmem_st8(t_s + 8 * g, packed);
                }
                l += (sum_a.x + sum_a.y) + (sum_b.x + sum_b.y);
                tmem_wait_st();
                if (j == 0 && pending >= 0) {
                    if (!mbar_wait_warp(on_step(C::kPVDone, step - 1), parity(step - 1), abort_flag, p.status)) { ok = false; break; }
                    tc_fence_after();
                    output(decode(p, pending), m_before, l_before);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(on_step(C::kPReady, step));
            }
            pending = item;
            m_before = m; l_before = l;
        }
        if (ok && pending >= 0 && mbar_wait_warp(on_step(C::kPVDone, step - 1), parity(step - 1), abort_flag, p.status)) {
            tc_fence_after();
            output(decode(p, pending), m_before, l_before);
        }
    }
    // ================================================================================ common tail
    tc_fence_before();
    __syncthreads();
    if (warp == 4) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

// Joins the splits of a row: out = sum_s w_s out_s / sum_s w_s, w_s = exp(lse_s - max lse).  A thread has eight channels of a row.
struct JoinParams {
    const float *part_out, *part_lse;
    const int* lengths;
    __nv_bfloat16* out;
    float* lse;
    int splits, stride, d, heads, kv_heads, G, chunks, vector, pixels;
    long long groups, rows, tokens;
    FastDiv by_pixels;
};
__global__ void __launch_bounds__(256) rib_cross_join_kernel(const JoinParams p)
{
    const long long thread = (long long)blockIdx.x * 256 + threadIdx.x, all = p.groups * p.rows;
    const long long at = thread / p.chunks;
    const int chunk = (int)(thread - at * p.chunks);
    if (at >= all) return;
    float most = -INFINITY, total = 0.f, x[8];
    for (int s = 0; s < p.splits; ++s) most = fmaxf(most, p.part_lse[s * all + at]);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    for (int s = 0; s < p.splits; ++s) {
        const float lse = p.part_lse[s * all + at];
        if (lse == -INFINITY) continue;
        const float w = expf(lse - most);
        const float4* src = reinterpret_cast<const float4*>(p.part_out + (s * all + at) * p.stride + 8 * chunk);
        const float4 lo = src[0], hi = src[1];
        total += w;
        x[0] += w * lo.x; x[1] += w * lo.y; x[2] += w * lo.z; x[3] += w * lo.w;
        x[4] += w * hi.x; x[5] += w * hi.y; x[6] += w * hi.z; x[7] += w * hi.w;
    }
    const long long group = at / p.rows, r = at - group * p.rows, token = r / p.G;
    const int context = (int)(group / p.kv_heads), head = (int)(group - (long long)context * p.kv_heads) * p.G + (int)(r - token * p.G);
    const bool none = p.lengths && __ldg(p.lengths + context) <= 0;
    const float inverse = none ? 0.f : 1.f / total;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = none ? 0.f : x[e] * inverse;
    const long long pixel_of_all = (long long)context * p.tokens + token;
    sm100::cross_store_row(p.out + (pixel_of_all * p.heads + head) * p.d, 8 * chunk, p.d, x, p.vector != 0);
    if (p.lse && chunk == 0) {
        int image, pixel;
        p.by_pixels.divmod((int)pixel_of_all, image, pixel);
        p.lse[((long long)image * p.heads + head) * p.pixels + pixel] = none ? -INFINITY : most + logf(total);
    }
}

__global__ void __launch_bounds__(256) rib_cross_pad_kernel(const CrossPad args)
{
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
        !cross_rows_map(&tm_k, p.k, p.contexts, p.L, p.kv_heads, p.width, DP, 1, kCrossBlock) || !cross_rows_map(&tm_v, p.v, p.contexts, p.L, p.kv_heads, p.width, DP, 1, kCrossBlock))
        return cudaErrorInvalidValue;
    static KernelSetup setup;
    int sms = 0;
    if (cudaError_t e = setup.prepare(rib_cross_fwd_kernel<DP>, Cfg<DP>::kSmem, &sms)) return e;
    Params a{};
    a.lengths = p.lengths; a.out = p.out_w; a.lse = p.lse_w; a.part_out = part_out; a.part_lse = part_lse; a.status = p.status;
    a.d = p.d; a.L = p.L; a.heads = p.heads; a.kv_heads = p.kv_heads; a.G = plan.G; a.rows_per_tile = plan.rows_per_tile; a.tokens_per_tile = plan.tokens_per_tile;
    a.blocks_per_split = plan.blocks_per_split; a.splits = plan.splits; a.items = plan.groups * plan.splits * plan.tiles;
    a.vector = p.d % 8 == 0;
    a.tokens = p.tokens; a.rows = plan.rows; a.groups = plan.groups;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)p.d); a.inv_sqrt_d = 1.f / sqrtf((float)p.d);
    a.by_tiles = make_fast_div(plan.tiles); a.by_splits = make_fast_div(plan.splits); a.by_kv = make_fast_div(p.kv_heads);
    a.by_pixels = make_fast_div((int)p.pixels); a.by_group = make_fast_div(plan.G); a.pixels = (int)p.pixels;
    const int slots = kCrossSms * kBlocksPerSm, grid = a.items < slots ? a.items : slots;
    ProfileScope scope(RIB_KERNEL_CROSS_FWD, stream);
    rib_cross_fwd_kernel<DP><<<grid, kThreads, Cfg<DP>::kSmem, stream>>>(tm_q, tm_k, tm_v, a);
    return cudaGetLastError();
}

cudaError_t join(const CrossProblem& p, const CrossPlan& plan, const float* part_out, const float* part_lse, int stride, cudaStream_t stream)
{
    JoinParams j{};
    j.part_out = part_out; j.part_lse = part_lse; j.lengths = p.lengths; j.out = p.out_w; j.lse = p.lse_w;
    j.splits = plan.splits; j.stride = stride; j.d = p.d; j.heads = p.heads; j.kv_heads = p.kv_heads; j.G = plan.G; j.chunks = (p.d + 7) / 8;
    j.vector = p.d % 8 == 0; j.pixels = (int)p.pixels; j.groups = plan.groups; j.rows = plan.rows; j.tokens = p.tokens; j.by_pixels = make_fast_div((int)p.pixels);
    const long long threads = j.groups * j.rows * j.chunks;
    ProfileScope scope(RIB_KERNEL_CROSS_JOIN, stream);
    rib_cross_join_kernel<<<(unsigned)((threads + 255) / 256), 256, 0, stream>>>(j);
    return cudaGetLastError();
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
    c.blocks = (p.L + kCrossBlock - 1) / kCrossBlock;
    c.rows = p.tokens * c.G;
    // Fewer items than CTAs that the card holds: the key blocks are dealt out to several, whose results are joined.
    auto split = [&](long long items, long long slots, int* splits, int* per) {
        long long n = items >= slots ? 1 : slots / items;
        if (n > c.blocks) n = c.blocks;
        *per = (int)((c.blocks + n - 1) / n);
        *splits = (c.blocks + *per - 1) / *per;
    };
    split((long long)c.groups * c.tiles, (long long)kCrossSms * kBlocksPerSm, &c.splits, &c.blocks_per_split);
    c.dq_tiles = (c.row_tiles + 1) / 2;
    split((long long)c.groups * c.dq_tiles, kCrossSms, &c.dq_splits, &c.dq_blocks_per_split);
    // dK and dV: a CTA to an SM; runs of row tiles such that the last round of CTAs is not a mostly empty one.  In us: 0.3 a tile, 3 for what a CTA begins and
    // ends with, and the way of the partial sums to memory and back.
    c.key_tiles = (p.L + 127) / 128;
    const long long units = (long long)c.groups * c.key_tiles;
    double best = 0;
    for (int s = 1; s <= c.row_tiles && s <= 64; ++s) {
        const int per = (c.row_tiles + s - 1) / s, used = (c.row_tiles + per - 1) / per;
        if (used != s) continue;
        const double cost = (double)((units * s + kCrossSms - 1) / kCrossSms) * (0.3 * per + 3) + (s > 1 ? 3 + s * (double)c.groups * p.L * (p.d <= 32 ? 32 : 64) * 16 / 4e6 : 0);
        if (s == 1 || cost < best) { best = cost; c.row_splits = s; c.row_tiles_per_split = per; }
    }
    return c;
}

cudaError_t cross_pad(const CrossPad& args, cudaStream_t stream)
{
    long long most = 0;
    for (int i = 0; i < args.tensors; ++i) most = args.rows[i] > most ? args.rows[i] : most;
    const long long blocks = (most * (args.width / 8) + 255) / 256;
    rib_cross_pad_kernel<<<dim3((unsigned)(blocks < 4 * kCrossSms ? blocks : 4 * kCrossSms), (unsigned)args.tensors), 256, 0, stream>>>(args);
    return cudaGetLastError();
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
    if (cudaError_t e = tile_width(p.d) == 32 ? launch_fwd<32>(p, plan, part_out, part_lse, stream) : launch_fwd<64>(p, plan, part_out, part_lse, stream)) return e;
    if (plan.splits > 1) {
        ++*launches;
        return join(p, plan, part_out, part_lse, tile_width(p.d), stream);
    }
    return cudaSuccess;
}

}  // namespace rib
