// Backward pass of the attention to states (rib_cross.cuh) for B200 (sm_100a), for sequences that one CTA cannot hold (rib_cross_short_bwd_sm100.cu has the others): two kernels over tcgen05 products:
//     P = exp(S - lse),   dS = P o (dO V^T - D),   D = rowsum(dO o O)
//     dQ = dS K / sqrt(d)                      rows on the lanes, a CTA per tile of rows, walking the keys
//     dV = P^T dO,  dK = dS^T Q / sqrt(d)      keys on the lanes, a CTA per tile of 128 keys, walking the rows
// Each computes P for itself: an exponential more per score than one kernel for all three would take, and no sum of dQ over key tiles in memory, so that
// every sum has one order and the results are the same from run to run.  Where there are too few tiles to fill the card, keys (dQ) or rows (dK, dV) are dealt
// out to several CTAs, whose fp32 sums a last kernel adds.  dQ runs beside dK and dV, on the SMs that those leave free.  A first kernel takes D and brings lse and D into the order in which tiles of rows read them.
// P and dS enter the products as bf16 (a rounding of at most 2^-8 of each, as everywhere in this library; dQ's share of it is as large as that of its own last rounding); sums are fp32.  dS in two parts would take
// that away for a third product and half as many instructions again, where instructions and their latencies are what bounds both kernels:
// a step of 128 x 64 scores takes 950 cycles for dQ and 890 for dK and dV, 512 of them exponentials (an eighth of which on the FMA pipe: 327 -> 340 us).  256 x 256 tokens, 6 heads of 32, to 1024 states, us: statistics 13, dQ 160, dK and dV 146 (exponentials alone: 90 each).
#include "rib_cross.cuh"

namespace rib {
namespace {

using namespace sm100;

constexpr int kRows = 128, kRowTile = 64;            // lanes of a product; rows of a tile of the statistics
constexpr float kLog2e = 1.4426950408889634f;

// -lse log2 e and -D of the rows of a group, in tiles of 64 entries of which tokens_per_tile x G are used, two by two: (-lse, -lse', -D, -D').  Entries that are
// no row have (-infinity, 0), a weight of 0.  `tiles` is even: dQ takes two of them at a time.
struct RowStats { float* at; int tokens_per_tile, tiles, G; FastDiv by_tokens; };
__device__ __forceinline__ float* stats_entry(float* at, long long entry) { return at + 4 * (entry >> 1) + (entry & 1); }      // -lse; -D two behind
__device__ __forceinline__ long long stats_index(const RowStats& s, long long group, long long token, int head)
{
    int tile, t;
    s.by_tokens.divmod((int)token, tile, t);
    return (group * s.tiles + tile) * kRowTile + t * s.G + head;
}

// 32 columns of scores s and dP of a lane -> dS as bf16, in the first 16 of dP's.  x = s scale + neg, P = 2^x held to 1 whatever the roundings of large scores and lse make of it, dS = P (dP + d).
// 16 columns at a time: dS goes where columns lie that have been read.  `stats(i)` gives (neg, neg', d, d') of columns 2 i, 2 i + 1; columns from `columns` on weigh nothing, whatever they hold, and
// chunks that have none of them are left out.
template <typename Stats>
__device__ __forceinline__ void weights_in_place(uint32_t t_s, uint32_t t_dp, int columns, float2 scale2, Stats stats)
{
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        if (16 * g >= columns) break;
        uint32_t a[16], b[16], pd[8];
        tmem_ld16(t_s + 16 * g, a);
        tmem_ld16(t_dp + 16 * g, b);
        tmem_wait_ld();
        if (columns < 16 * g + 16) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (16 * g + e >= columns) { a[e] = 0xff800000u; b[e] = 0u; }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 st = stats(8 * g + i);
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1])), scale2, make_float2(st.x, st.y));
            const float2 w = make_float2(ex2_approx(min_nan(x.x, 0.f)), ex2_approx(min_nan(x.y, 0.f)));
            const float2 z = __fmul2_rn(w, __fadd2_rn(make_float2(__uint_as_float(b[2 * i]), __uint_as_float(b[2 * i + 1])), make_float2(st.z, st.w)));
            pd[i] = pack_bf16x2(z.x, z.y);
        }
        tmem_st8(t_dp + 8 * g, pd);
    }
    tmem_wait_st();
}
// The same for keys on the lanes, 32 keys and 32 rows of a warp in four pieces of 16 x 16 (piece c: lanes 16 (c % 2) .., columns 16 (c / 2) ..), read as 16-lane fragments: a thread has 2 keys and 4 rows of a piece,
// and takes 16 words of statistics where a key to a thread takes 64 (`stats`: at (-lse, -lse', -D, -D') of its first two rows; 163 -> 152 us on 256 x 256 tokens to 1024 states).
__device__ __forceinline__ void weights_by_keys(uint32_t t_s, uint32_t t_dp, float2 scale2, const float4* stats)
{
    auto load = [&](int c, uint32_t (&a)[8], uint32_t (&b)[8]) {
        const uint32_t at = ((uint32_t)(16 * (c & 1)) << 16) + 16 * (c >> 1);
        tmem_ld_16x256b_x2(t_s + at, a);
        tmem_ld_16x256b_x2(t_dp + at, b);
    };
    auto work = [&](int c, const uint32_t (&a)[8], const uint32_t (&b)[8], const float4 (&st)[2]) {
        uint32_t pp[4], pd[4];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int r = 0; r < 2; ++r) {                 // keys lane / 4 and lane / 4 + 8 of the fragment
                const int i = 4 * q + 2 * r;
                const float2 x = __ffma2_rn(make_float2(__uint_as_float(a[i]), __uint_as_float(a[i + 1])), scale2, make_float2(st[q].x, st[q].y));
                const float2 w = make_float2(ex2_approx(min_nan(x.x, 0.f)), ex2_approx(min_nan(x.y, 0.f)));
                const float2 z = __fmul2_rn(w, __fadd2_rn(make_float2(__uint_as_float(b[i]), __uint_as_float(b[i + 1])), make_float2(st[q].z, st[q].w)));
                pp[2 * q + r] = pack_bf16x2(w.x, w.y);
                pd[2 * q + r] = pack_bf16x2(z.x, z.y);
            }
        const uint32_t at = ((uint32_t)(16 * (c & 1)) << 16) + 8 * (c >> 1);
        tmem_st_16x128b_x2(t_s + at, pp);
        tmem_st_16x128b_x2(t_dp + at, pd);
    };
    uint32_t a0[8], b0[8], a1[8], b1[8];
    float4 sa[2], sb[2];
    load(0, a0, b0);
    load(1, a1, b1);
    sa[0] = stats[0]; sa[1] = stats[4];
    tmem_wait_ld();
    work(0, a0, b0, sa);
    load(2, a0, b0);
    sb[0] = stats[8]; sb[1] = stats[12];
    work(1, a1, b1, sa);
    tmem_wait_ld();
    load(3, a1, b1);
    work(2, a0, b0, sb);
    tmem_wait_ld();
    work(3, a1, b1, sb);
    tmem_wait_st();
}
// where the K16 step kk of P or dS lies among its 64 columns
__device__ __forceinline__ uint32_t weights_at(int kk) { return 32 * (kk >> 1) + 8 * (kk & 1); }

// ------------------------------------------------------------------------------------------------ D, lse
struct PrepareParams {
    const __nv_bfloat16 *out, *dout;
    const float* lse;
    RowStats stats;
    int rows, entries, tokens, pixels;               // rows: tokens of all contexts x heads; entries: of the statistics
    int d, heads, kv_heads, G, lane_bits, row_blocks, vector;
    FastDiv by_heads, by_group, by_pixels, by_tokens_of_context, by_tiles;
};
constexpr int kPrepareRows = 4;                      // of a thread, their loads under way at once
__global__ void __launch_bounds__(256) rib_cross_bwd_prepare_kernel(const __grid_constant__ PrepareParams p)
{
    cudaGridDependencySynchronize();                      // it may have overtaken the kernel before
    if ((int)blockIdx.x >= p.row_blocks) {            // entries that are no row
        const int e = (blockIdx.x - p.row_blocks) * 256 + threadIdx.x;
        if (e >= p.entries) return;
        const int within = e % kRowTile;
        int group, tile, t, g;
        p.by_tiles.divmod(e / kRowTile, group, tile);
        p.by_group.divmod(within, t, g);
        if (t >= p.stats.tokens_per_tile || (long long)tile * p.stats.tokens_per_tile + t >= p.tokens) {
            float* at = stats_entry(p.stats.at, e);
            at[0] = -INFINITY; at[2] = 0.f;
        }
        return;
    }
    // rows in the order of memory, 2^lane_bits lanes to a row
    const int part = threadIdx.x & ((1 << p.lane_bits) - 1), rows_at_once = 256 >> p.lane_bits;
    const long long first = (long long)blockIdx.x * (kPrepareRows * rows_at_once) + (threadIdx.x >> p.lane_bits);
    float sum[kPrepareRows];
    if (p.vector) {
        uint4 a[kPrepareRows], b[kPrepareRows];
#pragma unroll
        for (int k = 0; k < kPrepareRows; ++k) {
            const long long row = first + k * rows_at_once;
            const bool there = row < p.rows && 8 * part < p.d;
            a[k] = there ? *(reinterpret_cast<const uint4*>(p.out + row * p.d) + part) : make_uint4(0u, 0u, 0u, 0u);
            b[k] = there ? *(reinterpret_cast<const uint4*>(p.dout + row * p.d) + part) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int k = 0; k < kPrepareRows; ++k) {
            const uint32_t x[4] = {a[k].x, a[k].y, a[k].z, a[k].w}, y[4] = {b[k].x, b[k].y, b[k].z, b[k].w};
            sum[k] = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[k] = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), sum[k]);
                sum[k] = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), sum[k]);
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < kPrepareRows; ++k) {
            const long long row = first + k * rows_at_once;
            sum[k] = 0.f;
            if (row < p.rows)
                for (int c = part; c < p.d; c += 1 << p.lane_bits) sum[k] = fmaf(__bfloat162float(p.out[row * p.d + c]), __bfloat162float(p.dout[row * p.d + c]), sum[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < kPrepareRows; ++k)
        for (int o = (1 << p.lane_bits) >> 1; o; o >>= 1) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], o);
#pragma unroll
    for (int k = 0; k < kPrepareRows; ++k) {
        const long long row = first + k * rows_at_once;
        if (row >= p.rows || part != 0) continue;
        int token_of_all, head, image, pixel, context, token, kv, g;
        p.by_heads.divmod((int)row, token_of_all, head);
        p.by_pixels.divmod(token_of_all, image, pixel);
        p.by_tokens_of_context.divmod(token_of_all, context, token);
        p.by_group.divmod(head, kv, g);
        const float lse = p.lse[((long long)image * p.heads + head) * p.pixels + pixel];
        float* at = stats_entry(p.stats.at, stats_index(p.stats, (long long)context * p.kv_heads + kv, token, g));
        at[0] = -lse * kLog2e; at[2] = -sum[k];
    }
}

// -------------------------------------------------------------------------------------------------- dQ
// Work item = two tiles of rows of a group (128 lanes) x a run of its key blocks of 64; a persistent CTA walks items, whose key blocks are one stream of steps:
//     S = Q K^T,  dP = dO V^T   (M128 N64)     P, dS over them     dQ += dS K   (A from tensor memory)
// Three sets of 64 + 64 columns rotate among the steps, each with eight warps of its own, two threads to a row (one: 172 against 167 us), so that one set's exponentials run under the others' products; dQ has
// two accumulators, and four warps that store one while the next item is under way.
// (The first form had four CTAs to an SM with one set of 64 columns each, S and dP one after the other: 256 x 256 tokens to 1024 states 283 us.)
constexpr int kDqThreads = 1024, kSets = 3;
constexpr uint32_t kTmemCols = 512, kColAcc = kSets * 128;

template <int DP> struct DqCfg {
    static constexpr int kStages = DP == 32 ? 8 : 6, kTiles = DP == 32 ? 4 : 3;
    static constexpr uint32_t kRow = DP * 2, kQBytes = kRows * kRow, kKBytes = kCrossBlock * kRow, kStatBytes = kRows * 8;
    static constexpr uint32_t kOffQ = 0, kOffDO = kTiles * kQBytes, kOffK = 2 * kTiles * kQBytes, kOffV = kOffK + kStages * kKBytes, kOffStats = kOffV + kStages * kKBytes,
                              kOffInfo = kOffStats + kTiles * kStatBytes, kOffBar = (kOffInfo + kStages * 4 + 7) & ~7u;
    // barriers: rows, key blocks, there and free again; of a set: scores and dP there, P and dS there, dS K done; of an accumulator: complete, stored; all products done
    static constexpr int kQFull = 0, kQEmpty = kQFull + kTiles, kKFull = kQEmpty + kTiles, kKEmpty = kKFull + kStages, kSFull = kKEmpty + kStages, kReady = kSFull + kSets,
                         kFree = kReady + kSets, kAccFull = kFree + kSets, kAccFree = kAccFull + 2, kDrain = kAccFree + 2, kBars = kDrain + 2;
    static constexpr uint32_t kOffMisc = kOffBar + kBars * 8, kSmem = kOffMisc + 16 + 1024;
    static_assert(kSmem <= 232448, "shared memory of a CTA");
    static_assert(kColAcc + 2 * DP <= kTmemCols, "tensor memory has 512 columns");
};

struct DqParams {
    const int* lengths;
    __nv_bfloat16* dq;
    float* part;                         // splits > 1: [splits][groups][rows][DP]
    int* status;
    const float* stats;
    int d, L, heads, kv_heads, G, rows_per_tile, tokens_per_tile, row_tiles, blocks_per_split, splits, items, vector;
    long long tokens, rows, groups;
    float scale_log2, inv_sqrt_d;
    FastDiv by_tiles, by_splits, by_kv, by_group;
};

struct DqItem { int tile, split, group, context, kv, first, blocks, length; };      // tile: of 128 rows
__device__ __forceinline__ DqItem decode(const DqParams& p, int item)
{
    DqItem c;
    p.by_tiles.divmod(item, item, c.tile);
    p.by_splits.divmod(item, c.group, c.split);
    p.by_kv.divmod(c.group, c.context, c.kv);
    c.length = p.lengths ? min(max(__ldcg(p.lengths + c.context), 0), p.L) : p.L;      // (past L1: the kernel waits for nobody)
    c.first = c.split * p.blocks_per_split;
    c.blocks = max(0, min(c.first + p.blocks_per_split, (c.length + kCrossBlock - 1) / kCrossBlock) - c.first);
    return c;
}

template <int DP>
__global__ void __launch_bounds__(kDqThreads, 1)
rib_cross_bwd_dq_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                        const __grid_constant__ DqParams p)
{
    using C = DqCfg<DP>;
    using T = CrossTile<DP>;
    constexpr uint32_t kStages = C::kStages, kTiles = C::kTiles;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
    auto bar = [&](int i) { return base + C::kOffBar + 8u * i; };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + C::kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + C::kOffMisc + 4);      // [1] stays 0: used by the drain waits
    volatile int* info = reinterpret_cast<volatile int*>(base_ptr + C::kOffInfo);               // of a key block's stage: keys + 128 x (slot of its rows + 8 x parity of their barrier's phase)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        abort_flag[0] = 0; abort_flag[1] = 0;
        for (int i = 0; i < C::kBars; ++i) mbar_init(bar(i), i >= C::kReady && i < C::kFree ? 8 : i >= C::kAccFree && i < C::kDrain ? 4 : 1);
        fence_barrier_init();
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_do); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
    }
    if (warp == 24) {
        tmem_alloc(base + C::kOffMisc, kTmemCols);
        tmem_relinquish();
    }
    // rows that the boxes do not reach (G does not divide 64)
    for (uint32_t i = 0; i < 4 * kTiles; ++i) cross_zero_rows(base_ptr + i * (C::kQBytes / 2), C::kRow, p.rows_per_tile, kRowTile, threadIdx.x, kDqThreads);
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    // It runs beside the kernel for dK and dV, the one before it in the stream, and waits for that only at its end.  What it reads - statistics, padded copies, lengths, the caller's tensors - is of kernels before
    // that one, which have ended and whose writes have reached L2: every CTA of dK and dV says so by starting this kernel behind its own wait for them, not before.  All reads here go to L2 (TMA, bulk copies, loads
    // past L1).  So the trigger stays behind that wait, and no kernel comes between the two launches.

    if (warp == 24) {
        // ============================================ loads
        uint32_t step = 0, live = 0, asked = 0;            // asked: items whose rows have been asked for
        for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            const DqItem c = decode(p, item);
            if (!c.blocks) continue;
            const uint32_t slot = live % kTiles;
            if (live >= kTiles && !mbar_wait_warp(bar(C::kQEmpty + slot), (live / kTiles - 1) & 1, abort_flag, p.status)) { ok = false; break; }
            if (elect_one()) {
                const uint32_t at = slot * C::kQBytes, half = C::kQBytes / 2, full = bar(C::kQFull + slot);
                const int token = 2 * c.tile * p.tokens_per_tile;
                mbar_arrive_expect_tx(full, 4u * (uint32_t)p.rows_per_tile * C::kRow + C::kStatBytes);
                for (int i = 0; i < 2; ++i) {
                    tma_load_4d(base + C::kOffQ + at + i * half, &tm_q, full, 0, c.kv * p.G, token + i * p.tokens_per_tile, c.context);
                    tma_load_4d(base + C::kOffDO + at + i * half, &tm_do, full, 0, c.kv * p.G, token + i * p.tokens_per_tile, c.context);
                }
                bulk_load_1d(base + C::kOffStats + slot * C::kStatBytes, p.stats + ((long long)c.group * p.row_tiles + 2 * c.tile) * (2 * kRowTile), C::kStatBytes, full);
            }
            __syncwarp();
            ++asked;
            for (int j = 0; j < c.blocks; ++j, ++step) {
                const uint32_t st = step % kStages;
                if (step >= kStages && !mbar_wait_warp(bar(C::kKEmpty + st), (step / kStages - 1) & 1, abort_flag, p.status)) { ok = false; break; }
                if (elect_one()) {
                    const int key = (c.first + j) * kCrossBlock;
                    info[st] = min(kCrossBlock, c.length - key) + 128 * (int)(slot + 8 * (live / kTiles & 1));
                    mbar_arrive_expect_tx(bar(C::kKFull + st), 2 * C::kKBytes);
                    tma_load_4d(base + C::kOffK + st * C::kKBytes, &tm_k, bar(C::kKFull + st), 0, c.kv, key, c.context);
                    tma_load_4d(base + C::kOffV + st * C::kKBytes, &tm_v, bar(C::kKFull + st), 0, c.kv, key, c.context);
                }
                __syncwarp();
            }
            ++live;
        }
        if (!ok) {      // gave up: copies in flight land before the CTA may exit
            for (uint32_t i = step > kStages ? step - kStages : 0; i < step; ++i) mbar_wait_warp(bar(C::kKFull + i % kStages), (i / kStages) & 1, abort_flag + 1, p.status);
            for (uint32_t i = asked > kTiles ? asked - kTiles : 0; i < asked; ++i) mbar_wait_warp(bar(C::kQFull + i % kTiles), (i / kTiles) & 1, abort_flag + 1, p.status);
        }
    } else if (warp == 25) {
        // ============================================ S and dP
        uint32_t step = 0, live = 0;
        for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            const DqItem c = decode(p, item);
            if (!c.blocks) continue;
            const uint32_t slot = live % kTiles;
            if (!mbar_wait_warp(bar(C::kQFull + slot), (live / kTiles) & 1, abort_flag, p.status)) { ok = false; break; }
            ++live;
            for (int j = 0; j < c.blocks; ++j, ++step) {
                const uint32_t st = step % kStages, set = step % kSets, round = step / kSets;
                const int keys = min(kCrossBlock, c.length - (c.first + j) * kCrossBlock), columns = (keys + 15) & ~15;
                if (!mbar_wait_warp(bar(C::kKFull + st), (step / kStages) & 1, abort_flag, p.status) ||
                    (round > 0 && !mbar_wait_warp(bar(C::kFree + set), (round - 1) & 1, abort_flag, p.status))) { ok = false; break; }
                if (keys < columns) {      // keys behind the last one: dS of 0 times what lies there must not become NaN
                    cross_zero_rows(base_ptr + C::kOffK + st * C::kKBytes, C::kRow, keys, columns, lane, 32);
                    fence_proxy_async();
                    __syncwarp();
                }
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t q = smem_desc_at(T::kDesc, base + C::kOffQ + slot * C::kQBytes), g = smem_desc_at(T::kDesc, base + C::kOffDO + slot * C::kQBytes);
                    const uint64_t k = smem_desc_at(T::kDesc, base + C::kOffK + st * C::kKBytes), v = smem_desc_at(T::kDesc, base + C::kOffV + st * C::kKBytes);
                    const uint32_t idesc = idesc_bf16_f32(kRows, columns, false);
#pragma unroll
                    for (int kk = 0; kk < DP / 16; ++kk) mma_ss(tmem + set * 128, q + T::kStepK * kk, k + T::kStepK * kk, idesc, kk ? 1u : 0u);
#pragma unroll
                    for (int kk = 0; kk < DP / 16; ++kk) mma_ss(tmem + set * 128 + 64, g + T::kStepK * kk, v + T::kStepK * kk, idesc, kk ? 1u : 0u);
                    mma_commit(bar(C::kSFull + set));
                }
                __syncwarp();
            }
        }
    } else if (warp == 26) {
        // ============================================ dQ
        uint32_t step = 0, live = 0;
        for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            const DqItem c = decode(p, item);
            if (!c.blocks) continue;
            const uint32_t slot = live % kTiles, acc = live & 1;
            for (int j = 0; j < c.blocks; ++j, ++step) {
                const uint32_t st = step % kStages, set = step % kSets, round = step / kSets;
                if (!mbar_wait_warp(bar(C::kReady + set), round & 1, abort_flag, p.status) ||
                    (j == 0 && live >= 2 && !mbar_wait_warp(bar(C::kAccFree + acc), (live / 2 - 1) & 1, abort_flag, p.status))) { ok = false; break; }
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t k = smem_desc_at(T::kDesc, base + C::kOffK + st * C::kKBytes);
                    constexpr uint32_t kIdesc = idesc_bf16_f32(kRows, DP, true);
                    const int k_steps = (min(kCrossBlock, c.length - (c.first + j) * kCrossBlock) + 15) / 16;
                    for (int kk = 0; kk < k_steps; ++kk) mma_ts(tmem + kColAcc + acc * DP, tmem + set * 128 + 64 + weights_at(kk), k + T::kStepRows * kk, kIdesc, (j || kk) ? 1u : 0u);
                    mma_commit(bar(C::kFree + set));
                    mma_commit(bar(C::kKEmpty + st));
                    if (j == c.blocks - 1) {
                        mma_commit(bar(C::kAccFull + acc));
                        mma_commit(bar(C::kQEmpty + slot));
                    }
                }
                __syncwarp();
            }
            ++live;
        }
    } else if (warp < 24) {
        // ============================================ P and dS, two threads to a row
        const int set = warp >> 3, half = (warp >> 2) & 1, row = (warp & 3) * 32 + lane;
        const uint32_t t_s = tmem + ((uint32_t)((warp & 3) * 32) << 16) + set * 128 + 32 * half;
        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
        uint32_t steps = 0;
        for (long long item = blockIdx.x + (long long)lane * gridDim.x; item < p.items; item += 32ll * gridDim.x) steps += (uint32_t)decode(p, (int)item).blocks;
        steps = __reduce_add_sync(0xffffffffu, steps);
        for (uint32_t step = set; step < steps; step += kSets) {
            const uint32_t st = step % kStages;
            // (all of these have arrived when the scores are there: the waits show this thread what the producer wrote beside the key block, and the statistics)
            if (!mbar_wait_warp(bar(C::kSFull + set), (step / kSets) & 1, abort_flag, p.status) || !mbar_wait_warp(bar(C::kKFull + st), (step / kStages) & 1, abort_flag, p.status)) { ok = false; break; }
            const int here = info[st], keys = here & 127, slot = here >> 7 & 7;
            if (!mbar_wait_warp(bar(C::kQFull + slot), here >> 10, abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            const float* stats = stats_entry(reinterpret_cast<float*>(base_ptr + C::kOffStats + slot * C::kStatBytes), row);
            const float neg = stats[0], d = stats[2];
            const auto of_row = [&](int) { return make_float4(neg, neg, d, d); };
            if (keys == kCrossBlock) weights_in_place(t_s, t_s + 64, 32, scale2, of_row);
            else weights_in_place(t_s, t_s + 64, keys - 32 * half, scale2, of_row);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::kReady + set));
        }
    } else if (warp >= 28) {
        // ============================================ stores of dQ
        const int row = (warp & 3) * 32 + lane, within = row & (kRowTile - 1);
        int row_token, row_head;
        p.by_group.divmod(within, row_token, row_head);
        uint32_t live = 0;
        for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            const DqItem c = decode(p, item);
            const bool none = c.blocks == 0;
            const uint32_t acc = live & 1;
            if (!none) {
                if (!mbar_wait_warp(bar(C::kAccFull + acc), (live / 2) & 1, abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
            }
            const long long token = (long long)(2 * c.tile + (row >= kRowTile ? 1 : 0)) * p.tokens_per_tile + row_token;
            const bool mine = within < p.rows_per_tile && token < p.tokens;
            const long long at = ((long long)c.split * p.groups + c.group) * p.rows + token * p.G + row_head;
            __nv_bfloat16* dst = p.dq + (((long long)c.context * p.tokens + token) * p.heads + c.kv * p.G + row_head) * p.d;
            const uint32_t t_acc = tmem + ((uint32_t)((warp & 3) * 32) << 16) + kColAcc + acc * DP;
#pragma unroll
            for (int g = 0; g < DP / 32; ++g) {
                uint32_t o[32];
                float x[32];
                if (!none) { tmem_ld32(t_acc + 32 * g, o); tmem_wait_ld(); }
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = none ? 0.f : __uint_as_float(o[e]) * p.inv_sqrt_d;
                if (g == DP / 32 - 1 && !none) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::kAccFree + acc));
                }
                if (mine && p.splits > 1) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(p.part + at * DP + 32 * g + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                } else if (mine) {
                    cross_store_row(dst, 32 * g, p.d, x, p.vector != 0);
                }
                __syncwarp();
            }
            if (!none) ++live;
        }
    }
    if (warp == 25 || warp == 26) {
        // everything issued by this warp has finished before the tensor memory is released
        if (elect_one()) mma_commit(bar(C::kDrain + warp - 25));
        __syncwarp();
        mbar_wait_warp(bar(C::kDrain + warp - 25), 0, abort_flag + 1, p.status);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 24) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
    if (blockIdx.x == gridDim.x - 1) cudaGridDependencySynchronize();      // what comes behind this kernel comes behind the one beside it too: its last CTA ends after that
}

// ----------------------------------------------------------------------------------------------- dK, dV
// A CTA has one tile of 128 keys of a group, K and V of it in shared memory, dV and dK in tensor memory, and walks a run of the group's tiles of 64 rows:
//     S^T = K Q^T,  dP^T = V dO^T   (M128 N64)      P^T, dS^T over them      dV += P^T dO,  dK += dS^T Q   (A from tensor memory)
// Three sets of 64 + 64 columns rotate among the tiles, each with eight warps of its own, two threads to a key (one: 178 against 163 us), so that one set's exponentials run under the others' products.
constexpr int kKvThreads = 896;
constexpr uint32_t kColDV = kColAcc;

template <int DP> struct KvCfg {
    static constexpr int kStages = 6;
    static constexpr uint32_t kRow = DP * 2, kKeyBytes = kRows * kRow, kRowBytes = kRowTile * kRow, kStatBytes = kRowTile * 8;
    static constexpr uint32_t kOffK = 0, kOffV = kKeyBytes, kOffQ = 2 * kKeyBytes, kOffDO = kOffQ + kStages * kRowBytes, kOffStats = kOffDO + kStages * kRowBytes,
                              kOffBar = kOffStats + kStages * kStatBytes;
    static constexpr int kKVFull = 0, kFull = 1, kEmpty = kFull + kStages, kSFull = kEmpty + kStages, kReady = kSFull + kSets, kFree = kReady + kSets, kAccFull = kFree + kSets,
                         kDrain = kAccFull + 1, kBars = kDrain + 2;
    static constexpr uint32_t kOffMisc = kOffBar + kBars * 8, kSmem = kOffMisc + 16 + 1024;
    static_assert(kRowBytes % 1024 == 0 && kSmem <= 232448, "swizzle atoms need aligned tiles; shared memory of a CTA");
    static_assert(kColDV + 2 * DP <= kTmemCols, "tensor memory has 512 columns");
};

struct KvParams {
    const int* lengths;
    const float* stats;
    __nv_bfloat16 *dk, *dv;
    float *part_dk, *part_dv;            // splits > 1: [splits][groups][L][DP]
    int* status;
    int d, L, kv_heads, G, key_tiles, splits, row_tiles, stat_tiles, tiles_per_split, rows_per_tile, tokens_per_tile, vector;
    long long groups;
    float scale_log2, inv_sqrt_d;
};

template <int DP>
__global__ void __launch_bounds__(kKvThreads, 1)
rib_cross_bwd_dkv_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                         const __grid_constant__ KvParams p)
{
    using C = KvCfg<DP>;
    using T = CrossTile<DP>;
    constexpr int kStages = C::kStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
    auto bar = [&](int i) { return base + C::kOffBar + 8u * i; };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + C::kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + C::kOffMisc + 4);      // [1] stays 0: used by the drain waits
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        abort_flag[0] = 0; abort_flag[1] = 0;
        for (int i = 0; i < C::kBars; ++i) mbar_init(bar(i), i >= C::kReady && i < C::kReady + kSets ? 8 : 1);
        fence_barrier_init();
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_do); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
    }
    if (warp == 24) {
        tmem_alloc(base + C::kOffMisc, kTmemCols);
        tmem_relinquish();
    }
    for (int i = 0; i < 2 * kStages; ++i) cross_zero_rows(base_ptr + C::kOffQ + i * C::kRowBytes, C::kRow, p.rows_per_tile, kRowTile, threadIdx.x, kKvThreads);
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    cudaGridDependencySynchronize();                      // it may have overtaken the kernel before: statistics, copies
    cudaTriggerProgrammaticLaunchCompletion();            // dQ needs no more than those, and has SMs that this kernel leaves free (it does not wait for them itself: never before the line above)
    int rest = blockIdx.x;
    const int split = rest % p.splits; rest /= p.splits;
    const int key_tile = rest % p.key_tiles, group = rest / p.key_tiles, context = group / p.kv_heads, kv = group - context * p.kv_heads;
    const int length = p.lengths ? min(max(p.lengths[context], 0), p.L) : p.L;
    const int first = split * p.tiles_per_split, key0 = key_tile * kRows;
    const int tiles = key0 < length ? min(p.row_tiles - first, p.tiles_per_split) : 0;       // CTA-uniform

    if (warp == 24) {
        // ============================================ loads
        int t = 0;
        if (tiles > 0 && elect_one()) {
            mbar_arrive_expect_tx(bar(C::kKVFull), 2 * C::kKeyBytes);
            tma_load_4d(base + C::kOffK, &tm_k, bar(C::kKVFull), 0, kv, key0, context);
            tma_load_4d(base + C::kOffV, &tm_v, bar(C::kKVFull), 0, kv, key0, context);
        }
        __syncwarp();
        for (; t < tiles; ++t) {
            const uint32_t st = t % kStages, use = t / kStages;
            if (use > 0 && !mbar_wait_warp(bar(C::kEmpty + st), (use - 1) & 1, abort_flag, p.status)) { ok = false; break; }
            if (elect_one()) {
                const int tile = first + t;
                mbar_arrive_expect_tx(bar(C::kFull + st), 2u * (uint32_t)p.rows_per_tile * C::kRow + C::kStatBytes);
                tma_load_4d(base + C::kOffQ + st * C::kRowBytes, &tm_q, bar(C::kFull + st), 0, kv * p.G, tile * p.tokens_per_tile, context);
                tma_load_4d(base + C::kOffDO + st * C::kRowBytes, &tm_do, bar(C::kFull + st), 0, kv * p.G, tile * p.tokens_per_tile, context);
                bulk_load_1d(base + C::kOffStats + st * C::kStatBytes, p.stats + ((long long)group * p.stat_tiles + tile) * (2 * kRowTile), C::kStatBytes, bar(C::kFull + st));
            }
            __syncwarp();
        }
        if (!ok) {      // gave up: copies in flight land before the CTA may exit
            for (int i = t > kStages ? t - kStages : 0; i < t; ++i) mbar_wait_warp(bar(C::kFull + i % kStages), (i / kStages) & 1, abort_flag + 1, p.status);
            if (tiles > 0) mbar_wait_warp(bar(C::kKVFull), 0, abort_flag + 1, p.status);
        }
    } else if (warp == 25) {
        // ============================================ S^T and dP^T
        if (tiles > 0) ok = mbar_wait_warp(bar(C::kKVFull), 0, abort_flag, p.status);
        for (int t = 0; t < tiles && ok; ++t) {
            const uint32_t st = t % kStages, set = t % kSets, round = t / kSets;
            if (!mbar_wait_warp(bar(C::kFull + st), (t / kStages) & 1, abort_flag, p.status) ||
                (round > 0 && !mbar_wait_warp(bar(C::kFree + set), (round - 1) & 1, abort_flag, p.status))) { ok = false; break; }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t k = smem_desc_at(T::kDesc, base + C::kOffK), v = smem_desc_at(T::kDesc, base + C::kOffV);
                const uint64_t q = smem_desc_at(T::kDesc, base + C::kOffQ + st * C::kRowBytes), g = smem_desc_at(T::kDesc, base + C::kOffDO + st * C::kRowBytes);
                constexpr uint32_t kIdesc = idesc_bf16_f32(kRows, kRowTile, false);
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk) mma_ss(tmem + set * 128, k + T::kStepK * kk, q + T::kStepK * kk, kIdesc, kk ? 1u : 0u);
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk) mma_ss(tmem + set * 128 + 64, v + T::kStepK * kk, g + T::kStepK * kk, kIdesc, kk ? 1u : 0u);
                mma_commit(bar(C::kSFull + set));
            }
            __syncwarp();
        }
    } else if (warp == 26) {
        // ============================================ dV and dK
        for (int t = 0; t < tiles; ++t) {
            const uint32_t st = t % kStages, set = t % kSets, round = t / kSets;
            if (!mbar_wait_warp(bar(C::kReady + set), round & 1, abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t q = smem_desc_at(T::kDesc, base + C::kOffQ + st * C::kRowBytes), g = smem_desc_at(T::kDesc, base + C::kOffDO + st * C::kRowBytes);
                constexpr uint32_t kIdesc = idesc_bf16_f32(kRows, DP, true);
#pragma unroll
                for (int kk = 0; kk < kRowTile / 16; ++kk) mma_ts(tmem + kColDV, tmem + set * 128 + weights_at(kk), g + T::kStepRows * kk, kIdesc, (t || kk) ? 1u : 0u);
#pragma unroll
                for (int kk = 0; kk < kRowTile / 16; ++kk) mma_ts(tmem + kColDV + DP, tmem + set * 128 + 64 + weights_at(kk), q + T::kStepRows * kk, kIdesc, (t || kk) ? 1u : 0u);
                mma_commit(bar(C::kFree + set));
                mma_commit(bar(C::kEmpty + st));
                if (t == tiles - 1) mma_commit(bar(C::kAccFull));
            }
            __syncwarp();
        }
    } else if (warp < 24) {
        // ============================================ P^T and dS^T, two threads to a key; then dV and dK
        const int set = warp >> 3, half = (warp >> 2) & 1;
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, t_s = tmem + lanes + set * 128 + 32 * half, t_dp = t_s + 64;
        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
        for (int t = set; t < tiles; t += kSets) {
            const uint32_t st = t % kStages, round = t / kSets;
            // (the statistics arrive with the rows: what the scores were computed from has landed, and this wait shows it to this thread)
            if (!mbar_wait_warp(bar(C::kSFull + set), round & 1, abort_flag, p.status) || !mbar_wait_warp(bar(C::kFull + st), (t / kStages) & 1, abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            const float4* stats = reinterpret_cast<const float4*>(base_ptr + C::kOffStats + st * C::kStatBytes);
            weights_by_keys(t_s, t_dp, scale2, stats + 16 * half + (lane & 3));
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::kReady + set));
        }
        if (ok && tiles > 0 && set == 0) {
            ok = mbar_wait_warp(bar(C::kAccFull), 0, abort_flag, p.status);
            tc_fence_after();
        }
        // four warps store dV, four dK
        if (ok && set == 0) {
            const int key = key0 + row;
            const bool mine = key < p.L, zero = tiles <= 0 || key >= length;
            const float scale = half == 0 ? 1.f : p.inv_sqrt_d;
            __nv_bfloat16* dst = (half == 0 ? p.dv : p.dk) + (((long long)context * p.L + key) * p.kv_heads + kv) * p.d;
            float* part = (half == 0 ? p.part_dv : p.part_dk) + (((long long)split * p.groups + group) * p.L + key) * DP;
#pragma unroll
            for (int g = 0; g < DP / 32; ++g) {
                uint32_t o[32];
                float x[32];
                if (tiles > 0) { tmem_ld32(tmem + lanes + kColDV + half * DP + 32 * g, o); tmem_wait_ld(); }
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = zero ? 0.f : __uint_as_float(o[e]) * scale;
                if (mine && p.splits > 1) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(part + 32 * g + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                } else if (mine) {
                    cross_store_row(dst, 32 * g, p.d, x, p.vector != 0);
                }
                __syncwarp();
            }
        }
    }
    if (warp == 25 || warp == 26) {
        // everything issued by this warp has finished before the tensor memory is released
        if (elect_one()) mma_commit(bar(C::kDrain + warp - 25));
        __syncwarp();
        mbar_wait_warp(bar(C::kDrain + warp - 25), 0, abort_flag + 1, p.status);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 24) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

// ------------------------------------------------------------------------------------ sums of the splits
struct SumTensor { const float* part; __nv_bfloat16* dst; long long rows; int splits, G, heads; long long rows_of_group, tokens; };      // rows of all groups; dst [contexts][tokens][heads][d], heads = groups of a context x G
struct SumParams { SumTensor t[3]; int d, stride, chunks, vector, blocks; };      // blocks: of a tensor
// kLanes threads have eight channels of a row; with eight of them each takes every eighth split, and they meet in a fixed order.  (Backward with one / eight, us of the call alone: 4 x 64 x 64 tokens, 6 heads of 32, to
// 200 states, 6 splits, 33 / 37; 10 x 64 x 64 to one dictionary of 128, 24 splits, 40 / 38; 180 x 320 to 77, also 24, 46 / 44.)
template <int kLanes>
__global__ void __launch_bounds__(256) rib_cross_bwd_sum_kernel(const __grid_constant__ SumParams p)
{
    const SumTensor t = p.t[blockIdx.x / p.blocks];
    const long long thread = ((long long)(blockIdx.x % p.blocks) * 256 + threadIdx.x) / kLanes;
    const int part = threadIdx.x % kLanes;
    const bool mine = thread < t.rows * p.chunks;        // (the others go along: lanes meet in shuffles)
    const long long at = mine ? thread / p.chunks : 0;
    const int chunk = mine ? (int)(thread - at * p.chunks) : 0;
    cudaGridDependencySynchronize();                      // it may have overtaken the kernel before
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
#pragma unroll 8
    for (int s = part; s < t.splits; s += kLanes) {
        const float4* src = reinterpret_cast<const float4*>(t.part + (s * t.rows + at) * p.stride + 8 * chunk);
        const float4 lo = src[0], hi = src[1];
        x[0] += lo.x; x[1] += lo.y; x[2] += lo.z; x[3] += lo.w;
        x[4] += hi.x; x[5] += hi.y; x[6] += hi.z; x[7] += hi.w;
    }
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += __shfl_xor_sync(0xffffffffu, x[e], o);
    }
    if (!mine || part) return;
    const long long group = at / t.rows_of_group, r = at - group * t.rows_of_group, token = r / t.G;
    const int per_context = t.heads / t.G;
    const long long context = group / per_context;
    const int head = (int)(group - context * per_context) * t.G + (int)(r - token * t.G);
    cross_store_row(t.dst + ((context * t.tokens + token) * t.heads + head) * p.d, 8 * chunk, p.d, x, p.vector != 0);
}

// ------------------------------------------------------------------------------------------------ host
int tile_width(int d) { return d <= 32 ? 32 : 64; }

int stat_tiles(const CrossPlan& plan) { return (plan.row_tiles + 1) / 2 * 2; }

struct BwdLayout { size_t q, dout, k, v, out, stats, part_dq, part_dk, part_dv, bytes; };
BwdLayout bwd_layout(const CrossProblem& p, const CrossPlan& plan)
{
    BwdLayout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += cross_align(bytes); return here; };
    if (cross_padded(p)) {
        const size_t width = (p.d + 7) / 8 * 8, queries = 2 * width * p.tokens * p.contexts * p.heads, keys = 2 * width * p.L * p.contexts * p.kv_heads;
        l.q = take(queries); l.dout = take(queries); l.k = take(keys); l.v = take(keys);
        if (plan.short_bwd) l.out = take(queries);
    }
    if (!plan.short_bwd) l.stats = take(sizeof(float) * 2 * kRowTile * stat_tiles(plan) * plan.groups);
    const size_t row = sizeof(float) * tile_width(p.d);
    if (plan.dq_splits > 1) l.part_dq = take(row * plan.dq_splits * plan.groups * plan.rows);
    if (plan.row_splits > 1) {
        l.part_dk = take(row * plan.row_splits * plan.groups * p.L);
        l.part_dv = take(row * plan.row_splits * plan.groups * p.L);
    }
    l.bytes = at;
    return l;
}

template <int DP>
cudaError_t launch_bwd(const CrossProblem& p, const CrossPlan& plan, const RowStats& stats, float* part_dq, float* part_dk, float* part_dv, cudaStream_t stream)
{
    if (!encode_fn()) return cudaErrorNotSupported;
    CUtensorMap tm_q, tm_do, tm_k, tm_v, kv_k, kv_v;
    const auto rows = [&](CUtensorMap* m, const void* x) { return cross_rows_map(m, x, p.contexts, p.tokens, p.heads, p.width, DP, plan.G, plan.kv_tokens_per_tile); };
    const auto keys = [&](CUtensorMap* m, const void* x, int n) { return cross_rows_map(m, x, p.contexts, p.L, p.kv_heads, p.width, DP, 1, n); };
    if (!rows(&tm_q, p.q) || !rows(&tm_do, p.dout) || !keys(&tm_k, p.k, kCrossBlock) || !keys(&tm_v, p.v, kCrossBlock) || !keys(&kv_k, p.k, kRows) || !keys(&kv_v, p.v, kRows))
        return cudaErrorInvalidValue;
    static KernelSetup dq_setup, kv_setup;
    int sms = 0;
    if (cudaError_t e = dq_setup.prepare(rib_cross_bwd_dq_kernel<DP>, DqCfg<DP>::kSmem, &sms)) return e;
    if (cudaError_t e = kv_setup.prepare(rib_cross_bwd_dkv_kernel<DP>, KvCfg<DP>::kSmem, &sms)) return e;
    const float scale_log2 = kLog2e / sqrtf((float)p.d), inv_sqrt_d = 1.f / sqrtf((float)p.d);
    DqParams a{};
    a.lengths = p.lengths; a.dq = p.dq; a.part = part_dq; a.status = p.status; a.stats = stats.at;
    a.d = p.d; a.L = p.L; a.heads = p.heads; a.kv_heads = p.kv_heads; a.G = plan.G; a.rows_per_tile = plan.kv_rows_per_tile; a.tokens_per_tile = plan.kv_tokens_per_tile;
    a.row_tiles = stats.tiles; a.blocks_per_split = plan.dq_blocks_per_split; a.splits = plan.dq_splits; a.items = plan.groups * plan.dq_splits * plan.dq_tiles; a.vector = p.d % 8 == 0;
    a.tokens = p.tokens; a.rows = plan.rows; a.groups = plan.groups; a.scale_log2 = scale_log2; a.inv_sqrt_d = inv_sqrt_d;
    a.by_tiles = make_fast_div(plan.dq_tiles); a.by_splits = make_fast_div(plan.dq_splits); a.by_kv = make_fast_div(p.kv_heads); a.by_group = make_fast_div(plan.G);
    KvParams b{};
    b.lengths = p.lengths; b.stats = stats.at; b.dk = p.dk; b.dv = p.dv; b.part_dk = part_dk; b.part_dv = part_dv; b.status = p.status;
    b.d = p.d; b.L = p.L; b.kv_heads = p.kv_heads; b.G = plan.G; b.key_tiles = plan.key_tiles; b.splits = plan.row_splits; b.row_tiles = plan.row_tiles; b.stat_tiles = stats.tiles;
    b.tiles_per_split = plan.row_tiles_per_split; b.rows_per_tile = plan.kv_rows_per_tile; b.tokens_per_tile = plan.kv_tokens_per_tile; b.vector = p.d % 8 == 0;
    b.groups = plan.groups; b.scale_log2 = scale_log2; b.inv_sqrt_d = inv_sqrt_d;
    {
        ProfileScope scope(RIB_KERNEL_CROSS_BWD_DKV, stream);
        if (cudaError_t e = launch_overtaking(rib_cross_bwd_dkv_kernel<DP>, plan.groups * plan.key_tiles * plan.row_splits, kKvThreads, KvCfg<DP>::kSmem, stream, tm_q, tm_do, kv_k, kv_v, b)) return e;
    }
    // It begins on SMs that the kernel before it leaves free.  Contexts of their own lengths leave it CTAs without keys, and those SMs for longer: runs of half the length then, so that they take more of them
    // (us of both with the statistics, one run an SM / two: 4 x 48 x 48 tokens, 8 heads of 64 on 2, to 512 to 2048 states 129 / 114, 16 x 64 x 64, 4 heads of 32, to up to 512 109 / 102; full contexts of 2048 161 / 164).
    const int most = (p.lengths ? 2 : 1) * kCrossSms, grid = a.items < most ? a.items : most;
    ProfileScope scope(RIB_KERNEL_CROSS_BWD_DQ, stream);
    return launch_overtaking(rib_cross_bwd_dq_kernel<DP>, grid, kDqThreads, DqCfg<DP>::kSmem, stream, tm_q, tm_do, tm_k, tm_v, a);
}

}  // namespace

size_t cross_bwd_workspace(const CrossProblem& p) { return bwd_layout(p, cross_plan(p)).bytes; }

cudaError_t cross_bwd(CrossProblem p, cudaStream_t stream, int* launches)
{
    const CrossPlan plan = cross_plan(p);
    const BwdLayout l = bwd_layout(p, plan);
    uint8_t* ws = static_cast<uint8_t*>(p.workspace);
    *launches = 3;
    RowStats stats{};
    stats.at = reinterpret_cast<float*>(ws + l.stats);
    stats.tokens_per_tile = plan.kv_tokens_per_tile; stats.tiles = stat_tiles(plan); stats.G = plan.G; stats.by_tokens = make_fast_div(plan.kv_tokens_per_tile);
    if (plan.short_bwd) *launches = 1;
    else {
        PrepareParams a{};
        a.out = p.out; a.dout = p.dout; a.lse = p.lse_in; a.stats = stats;
        a.rows = (int)(p.tokens * p.contexts * p.heads); a.entries = plan.groups * stats.tiles * kRowTile; a.tokens = (int)p.tokens; a.pixels = (int)p.pixels;
        a.d = p.d; a.heads = p.heads; a.kv_heads = p.kv_heads; a.G = plan.G; a.vector = p.d % 8 == 0;
        a.lane_bits = p.d <= 8 ? 0 : p.d <= 16 ? 1 : p.d <= 32 ? 2 : 3;
        const int per_block = kPrepareRows * (256 >> a.lane_bits);
        a.row_blocks = a.rows / per_block + (a.rows % per_block != 0);
        a.by_heads = make_fast_div(p.heads); a.by_group = make_fast_div(plan.G); a.by_pixels = make_fast_div((int)p.pixels); a.by_tokens_of_context = make_fast_div((int)p.tokens);
        a.by_tiles = make_fast_div(stats.tiles);
        {
            ProfileScope scope(RIB_KERNEL_CROSS_BWD_PREPARE, stream);
            if (cudaError_t e = launch_overtaking(rib_cross_bwd_prepare_kernel, a.row_blocks + (a.entries + 255) / 256, 256, 0, stream, a)) return e;
        }
    }
    p.width = p.d;
    if (cross_padded(p)) {
        CrossPad pad{};
        pad.tensors = plan.short_bwd ? 5 : 4; pad.d = p.d; pad.width = (p.d + 7) / 8 * 8;
        const __nv_bfloat16** src[5] = {&p.q, &p.dout, &p.k, &p.v, &p.out};
        const size_t off[5] = {l.q, l.dout, l.k, l.v, l.out};
        for (int i = 0; i < pad.tensors; ++i) {
            pad.src[i] = *src[i];
            pad.dst[i] = reinterpret_cast<__nv_bfloat16*>(ws + off[i]);
            pad.rows[i] = p.contexts * (i == 2 || i == 3 ? (long long)p.L * p.kv_heads : p.tokens * p.heads);
            *src[i] = pad.dst[i];
        }
        p.width = pad.width;
        if (cudaError_t e = cross_pad(pad, stream)) return e;
        ++*launches;
    }
    float *part_dq = reinterpret_cast<float*>(ws + l.part_dq), *part_dk = reinterpret_cast<float*>(ws + l.part_dk), *part_dv = reinterpret_cast<float*>(ws + l.part_dv);
    if (cudaError_t e = plan.short_bwd ? cross_bwd_short(p, plan, part_dk, part_dv, stream) : tile_width(p.d) == 32 ? launch_bwd<32>(p, plan, stats, part_dq, part_dk, part_dv, stream) : launch_bwd<64>(p, plan, stats, part_dq, part_dk, part_dv, stream)) return e;
    SumParams s{};
    int tensors = 0;
    if (plan.dq_splits > 1) s.t[tensors++] = SumTensor{part_dq, p.dq, plan.groups * plan.rows, plan.dq_splits, plan.G, p.heads, plan.rows, p.tokens};
    if (plan.row_splits > 1) {
        s.t[tensors++] = SumTensor{part_dk, p.dk, (long long)plan.groups * p.L, plan.row_splits, 1, p.kv_heads, p.L, p.L};
        s.t[tensors++] = SumTensor{part_dv, p.dv, (long long)plan.groups * p.L, plan.row_splits, 1, p.kv_heads, p.L, p.L};
    }
    if (!tensors) return cudaSuccess;
    s.d = p.d; s.stride = tile_width(p.d); s.chunks = (p.d + 7) / 8; s.vector = p.d % 8 == 0;
    long long most = 0;
    for (int i = 0; i < tensors; ++i) most = s.t[i].rows > most ? s.t[i].rows : most;
    ++*launches;
    ProfileScope scope(RIB_KERNEL_CROSS_BWD_SUM, stream);
    int splits = 0;
    for (int i = 0; i < tensors; ++i) splits = s.t[i].splits > splits ? s.t[i].splits : splits;
    const bool eight = splits > 8;
    s.blocks = (int)((most * s.chunks * (eight ? 8 : 1) + 255) / 256);
    return launch_overtaking(eight ? rib_cross_bwd_sum_kernel<8> : rib_cross_bwd_sum_kernel<1>, s.blocks * tensors, 256, 0, stream, s);
}

}  // namespace rib
