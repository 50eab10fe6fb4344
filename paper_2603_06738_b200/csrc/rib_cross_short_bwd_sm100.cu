// Backward pass of the attention to short sequences of states (rib_cross.cuh) in one kernel: up to 256 states in heads of up to 32 channels, up to 128 in wider ones, so that a CTA has all keys of a group and
// dQ is complete where it is taken.
//     S^T = K Q^T,  dP^T = V dO^T            (M128 N64: 128 keys on the lanes, 64 rows)
//     P^T = exp2(S^T scale - lse),  dS^T = P^T o (dP^T - D),   D = rowsum(dO o O)
//     dV += P^T dO                           (A from tensor memory)
//     dK += dS^T Q                           (A = dS in shared memory, K-major)
//     dQ  = dS K                             (A = the same tile, MN-major: two tiles of 64 rows are its 128 lanes; over one or two blocks of keys)
// P and dS enter the products as bf16 (a rounding of at most 2^-8 of each, as everywhere in this library); statistics and sums are fp32.
//
// A CTA has a group of rows and keys and a run of the group's row tiles, two by two.  Unit of the pipeline is (row tile, block of 128 keys); three buffers of S^T and two of dP^T rotate among the units, and
// two sets of arithmetic warps take the even and the odd row tiles, so that one set's exponentials run under the other's products.  D is taken here as well, by four warps of their own.
// The sums over rows that several CTAs share are joined in a fixed order by the kernel that joins those of the long form: results are the same from run to run.
// What sets the pace is the loop  scores -> arithmetic -> dV -> next scores of the buffer  (1800 cycles of issue, products and barriers, 2150 of arithmetic) over the three units in flight: 1375 cycles a
// unit of 128 keys and 64 rows, of which exponentials take 512 and the products 300.  With statistics by two warps and S^T and dP^T issued by a warp each it was 1650, with dP^T beside dQ 1700; O in registers
// instead of beside dO 1450; a third buffer of dP^T, where there is one block of keys, takes 2 %.
// With the sums that follow, us: 16 x 96 x 96 tokens, 6 heads of 32, to 16 to 256 states 119 (the statistics, dQ, dK and dV, and sums of the long form, each a kernel: 204), 10 x 64 x 64 to one dictionary of 128
// 31 (54), 180 x 320 to 77 37 (70), to 256 66 (103).
//
// Roles (896 threads): warps 0-15 arithmetic (0-7 even, 8-15 odd row tiles; then dV and dK), 16 loads, 17 S^T and dP^T, 18 dV and dK (and owns the tensor memory), 19 dQ, 20-23 store dQ, 24-27 lse and D.
// Every wait is bounded (tests/test_cross_short_barriers.py is a model of them).
#include "rib_cross.cuh"

namespace rib {
namespace {

using namespace sm100;

constexpr int kThreads = 896, kKeys = 128, kRowTile = 64;
constexpr uint32_t kTmemCols = 512, kColDP = 3 * kRowTile, kColAcc = kColDP + 2 * kRowTile, kColDQ = kColAcc + 128;      // S^T; dP^T; dV, dK of each block of keys; dQ
constexpr float kLog2e = 1.4426950408889634f;

template <int DP> struct Cfg {
    static constexpr int kBlocks = 64 / DP, kStages = DP == 32 ? 6 : 4, kDQs = 64 / DP;                    // blocks of keys; row tiles under way; accumulators of dQ
    static constexpr uint32_t kRow = DP * 2, kKeyBytes = kKeys * kRow, kRowBytes = kRowTile * kRow, kStatBytes = kRowTile * 8, kDSHalf = kKeys * 128;
    static constexpr uint32_t kOffK = 0, kOffV = kOffK + kBlocks * kKeyBytes, kOffQ = kOffV + kBlocks * kKeyBytes, kOffDO = kOffQ + kStages * kRowBytes, kOffO = kOffDO + kStages * kRowBytes, kOffDS = kOffO + kStages * kRowBytes,
                              kOffOut = kOffDS + 4 * kDSHalf, kOffStats = kOffOut + 2 * kRowBytes, kOffBar = kOffStats + kStages * kStatBytes;
    // barriers: keys; row tiles there, their statistics there, free again; scores there, P and dS there (of a unit mod 6: a set sees every phase of its own); P read, dP read; dS read; dQ there, read; dV and dK
    // complete; all products of a warp done
    static constexpr int kKVFull = 0, kFull = 1, kStats = kFull + kStages, kEmpty = kStats + kStages, kSFull = kEmpty + kStages, kReady = kSFull + 6, kPFree = kReady + 6, kDPFree = kPFree + 3,
                         kDSFree = kDPFree + 2, kDQFull = kDSFree + 2, kDQFree = kDQFull + 2, kAccFull = kDQFree + 2, kDrain = kAccFull + 1, kBars = kDrain + 3;
    static constexpr uint32_t kOffMisc = kOffBar + kBars * 8, kSmem = kOffMisc + 16 + 1024;
    static constexpr int arrivals(int i)
    {
        return i >= kStats && i < kEmpty ? 2 : i >= kReady && i < kPFree ? 8 : i >= kDPFree && i < kDSFree ? 8 : i >= kDSFree && i < kDQFull ? 2 : i >= kDQFree && i < kAccFull ? 4 : 1;
    }
    static_assert(kSmem <= 232448, "shared memory of a CTA");
    static_assert(kColDQ + kDQs * DP <= kTmemCols, "tensor memory has 512 columns");
};

// A place in a ring of n and the parity of its round, without divisions.
struct Place {
    uint32_t at, round;
    __device__ __forceinline__ void step(uint32_t by, uint32_t n)
    {
        at += by;
        if (at >= n) { at -= n; round ^= 1u; }
    }
};

struct Params {
    const int* lengths;
    const float* lse;
    __nv_bfloat16 *dq, *dk, *dv;
    float *part_dk, *part_dv;            // splits > 1: [splits][groups][L][DP]
    int* status;
    int d, L, heads, kv_heads, G, splits, pairs, pairs_per_split, rows_per_tile, tokens_per_tile, vector, tma_out, tokens, pixels, shared, contexts;
    long long groups;
    float scale_log2, inv_sqrt_d;
    FastDiv by_group, by_pixels;
};

// The context of a rank when those of more blocks of keys come first (by a whole warp).
__device__ __forceinline__ int context_of_rank(const Params& p, int rank, int lane)
{
    for (int want = 2; want >= 0; --want)
        for (int c0 = 0; c0 < p.contexts; c0 += 32) {
            const int c = c0 + lane, length = c < p.contexts ? min(max(p.lengths[c], 0), p.L) : -kKeys;
            const uint32_t those = __ballot_sync(0xffffffffu, (length + kKeys - 1) / kKeys == want && c < p.contexts);
            if (rank < __popc(those)) return c0 + __ffs(__ballot_sync(0xffffffffu, (those >> lane & 1u) && __popc(those & ((1u << lane) - 1u)) == rank)) - 1;
            rank -= __popc(those);
        }
    return 0;
}

template <int DP, bool kLongFirst>
__global__ void __launch_bounds__(kThreads, 1)
rib_cross_short_bwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_out, const __grid_constant__ CUtensorMap tm_k,
                           const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_dq, const __grid_constant__ Params p)
{
    using C = Cfg<DP>;
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
        for (int i = 0; i < C::kBars; ++i) mbar_init(bar(i), C::arrivals(i));
        fence_barrier_init();
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_do); prefetch_tensormap(&tm_out); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
    }
    if (warp == 18) {
        tmem_alloc(base + C::kOffMisc, kTmemCols);
        tmem_relinquish();
    }
    // rows that the boxes do not reach (G does not divide 64); dS of keys that are never there
    for (int i = 0; i < 3 * kStages; ++i) cross_zero_rows(base_ptr + C::kOffQ + i * C::kRowBytes, C::kRow, p.rows_per_tile, kRowTile, threadIdx.x, kThreads);
    cross_zero_rows(base_ptr + C::kOffDS, 128, 0, 4 * kKeys, threadIdx.x, kThreads);
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    cudaGridDependencySynchronize();                      // it may have overtaken the kernel before

    const int split = blockIdx.x % p.splits;
    int group = blockIdx.x / p.splits, context = group / p.kv_heads;
    const int kv = group - context * p.kv_heads;
    if constexpr (kLongFirst) {
        volatile int* shared_context = reinterpret_cast<volatile int*>(base_ptr + C::kOffMisc + 12);
        if (warp == 0) {
            const int c = context_of_rank(p, context, lane);
            if (lane == 0) *shared_context = c;
        }
        __syncthreads();
        context = *shared_context;
        group = context * p.kv_heads + kv;
    }
    const int length = p.lengths ? min(max(p.lengths[context], 0), p.L) : p.L;
    const int first_pair = split * p.pairs_per_split, pairs = min(p.pairs - first_pair, p.pairs_per_split);
    const int blocks = (length + kKeys - 1) / kKeys, first = 2 * first_pair;
    // one block of keys of 32 channels leaves the columns of the other's dV and dK to a third buffer of dP^T, which is then free with its buffer of S^T
    const bool third = DP == 32 && blocks == 1;
    auto column_dp = [&](uint32_t buf, int h) { return tmem + (!third ? kColDP + h * kRowTile : buf == 2 ? kColAcc + 2 * DP : kColDP + buf * kRowTile); };
    const int tiles = blocks ? 2 * pairs : 0, units = tiles * blocks;      // unit u: block (u / 2) mod blocks of keys, row tile 2 (u / 2 / blocks) + (u mod 2)

    if (warp == 16) {
        // ============================================ loads
        int t = 0;
        if (tiles > 0 && elect_one()) {
            mbar_arrive_expect_tx(bar(C::kKVFull), (uint32_t)blocks * 2 * C::kKeyBytes);
            for (int b = 0; b < blocks; ++b) {
                tma_load_4d(base + C::kOffK + b * C::kKeyBytes, &tm_k, bar(C::kKVFull), 0, kv, b * kKeys, context);
                tma_load_4d(base + C::kOffV + b * C::kKeyBytes, &tm_v, bar(C::kKVFull), 0, kv, b * kKeys, context);
            }
        }
        __syncwarp();
        for (; t < tiles; ++t) {
            const uint32_t st = t % kStages, use = t / kStages;
            if (use > 0 && !mbar_wait_warp(bar(C::kEmpty + st), (use - 1) & 1, abort_flag, p.status)) { ok = false; break; }
            if (elect_one()) {
                const int token = (first + t) * p.tokens_per_tile;
                mbar_arrive_expect_tx(bar(C::kFull + st), 3u * (uint32_t)p.rows_per_tile * C::kRow);
                tma_load_4d(base + C::kOffQ + st * C::kRowBytes, &tm_q, bar(C::kFull + st), 0, kv * p.G, token, context);
                tma_load_4d(base + C::kOffDO + st * C::kRowBytes, &tm_do, bar(C::kFull + st), 0, kv * p.G, token, context);
                tma_load_4d(base + C::kOffO + st * C::kRowBytes, &tm_out, bar(C::kFull + st), 0, kv * p.G, token, context);
            }
            __syncwarp();
        }
        if (!ok) {      // gave up: copies in flight land before the CTA may exit
            for (int i = t > kStages ? t - kStages : 0; i < t; ++i) mbar_wait_warp(bar(C::kFull + i % kStages), (i / kStages) & 1, abort_flag + 1, p.status);
            if (tiles > 0) mbar_wait_warp(bar(C::kKVFull), 0, abort_flag + 1, p.status);
        }
    } else if (warp == 17) {
        // ============================================ S^T and dP^T
        if (tiles > 0) {
            ok = mbar_wait_warp(bar(C::kKVFull), 0, abort_flag, p.status);
            const int keys = length - (blocks - 1) * kKeys, end = (keys + 15) & ~15;
            if (ok && keys < end) {      // keys behind the last one: dS of 0 times what lies there must not become NaN
                cross_zero_rows(base_ptr + C::kOffK + (blocks - 1) * C::kKeyBytes, C::kRow, keys, end, lane, 32);
                fence_proxy_async();
                __syncwarp();
            }
        }
        int b = 0;
        Place unit{0u, 0u}, scores{0u, 1u}, pair{0u, 0u};      // scores.round: of the phase that frees a buffer; pair: the stage of the first of two row tiles
        for (int u = 0; u < units && ok; ++u) {
            const int h = u & 1;
            const uint32_t st = pair.at + h, buf = scores.at;
            if ((b == 0 && !mbar_wait_warp(bar(C::kFull + st), pair.round, abort_flag, p.status)) || (u >= 3 && !mbar_wait_warp(bar(C::kPFree + buf), scores.round, abort_flag, p.status))) { ok = false; break; }
            tc_fence_after();
            const uint64_t k = smem_desc_at(T::kDesc, base + C::kOffK + b * C::kKeyBytes), v = smem_desc_at(T::kDesc, base + C::kOffV + b * C::kKeyBytes);
            const uint64_t q = smem_desc_at(T::kDesc, base + C::kOffQ + st * C::kRowBytes), go = smem_desc_at(T::kDesc, base + C::kOffDO + st * C::kRowBytes);
            constexpr uint32_t kIdesc = idesc_bf16_f32(kKeys, kRowTile, false);
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk) mma_ss(tmem + buf * kRowTile, k + T::kStepK * kk, q + T::kStepK * kk, kIdesc, kk ? 1u : 0u);
            }
            __syncwarp();
            if (!third && u >= 2 && !mbar_wait_warp(bar(C::kDPFree + h), (u / 2 - 1) & 1, abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk) mma_ss(column_dp(buf, h), v + T::kStepK * kk, go + T::kStepK * kk, kIdesc, kk ? 1u : 0u);
                mma_commit(bar(C::kSFull + unit.at));
            }
            __syncwarp();
            unit.step(1, 6);
            scores.step(1, 3);
            if (h && ++b == blocks) { b = 0; pair.step(2, kStages); }
        }
    } else if (warp == 18) {
        // ============================================ dV and dK
        int b = 0;
        Place unit{0u, 0u}, scores{0u, 0u}, pair{0u, 0u};
        for (int u = 0; u < units; ++u) {
            const int h = u & 1, w = u >> 1;
            const uint32_t st = pair.at + h, buf = scores.at;
            if (!mbar_wait_warp(bar(C::kReady + unit.at), unit.round, abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t q = smem_desc_at(T::kDesc, base + C::kOffQ + st * C::kRowBytes), go = smem_desc_at(T::kDesc, base + C::kOffDO + st * C::kRowBytes);
                const uint64_t ds = smem_desc_at(smem_desc_const(16, 1024, kSwizzle128B), base + C::kOffDS + ((w & 1) * 2 + h) * C::kDSHalf);      // 128-byte lines of a key's 64 rows
                constexpr uint32_t kIdesc = idesc_bf16_f32(kKeys, DP, true);
                const uint32_t acc = tmem + kColAcc + 2 * DP * b, more = u >= 2 * blocks || h;      // (a block's first tile begins the sums)
#pragma unroll
                for (int kk = 0; kk < kRowTile / 16; ++kk) mma_ts(acc, tmem + buf * kRowTile + 32 * (kk >> 1) + 8 * (kk & 1), go + T::kStepRows * kk, kIdesc, more | (kk ? 1u : 0u));
                mma_commit(bar(C::kPFree + buf));
#pragma unroll
                for (int kk = 0; kk < kRowTile / 16; ++kk) mma_ss(acc + DP, ds + 2 * kk, q + T::kStepRows * kk, kIdesc, more | (kk ? 1u : 0u));
                if (h) mma_commit(bar(C::kDSFree + (w & 1)));
                if (b == blocks - 1) mma_commit(bar(C::kEmpty + st));
                if (u == units - 1) mma_commit(bar(C::kAccFull));
            }
            __syncwarp();
            unit.step(1, 6);
            scores.step(1, 3);
            if (h && ++b == blocks) { b = 0; pair.step(2, kStages); }
        }
    } else if (warp == 19) {
        // ============================================ dQ
        int b = 0, g = 0;
        Place unit{0u, 0u};
        for (int w = 0; 2 * w < units; ++w, unit.step(2, 6)) {
            const int acc = g % C::kDQs;
            if (!mbar_wait_warp(bar(C::kReady + unit.at), unit.round, abort_flag, p.status) || !mbar_wait_warp(bar(C::kReady + unit.at + 1), unit.round, abort_flag, p.status) ||
                (b == 0 && g >= C::kDQs && !mbar_wait_warp(bar(C::kDQFree + acc), (g / C::kDQs - 1) & 1, abort_flag, p.status))) { ok = false; break; }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t k = smem_desc_at(T::kDesc, base + C::kOffK + b * C::kKeyBytes);
                const uint64_t ds = smem_desc_at(smem_desc_const(C::kDSHalf, 1024, kSwizzle128B), base + C::kOffDS + (w & 1) * 2 * C::kDSHalf);      // MN-major: the tiles of 64 rows one leading step apart
                constexpr uint32_t kIdesc = idesc_bf16_f32_ab(2 * kRowTile, DP, true, true);
                const int steps = (min(kKeys, length - b * kKeys) + 15) / 16;
                for (int kk = 0; kk < steps; ++kk) mma_ss(tmem + kColDQ + acc * DP, ds + 128 * kk, k + T::kStepRows * kk, kIdesc, (b || kk) ? 1u : 0u);
                mma_commit(bar(C::kDSFree + (w & 1)));
                if (b == blocks - 1) mma_commit(bar(C::kDQFull + acc));
            }
            __syncwarp();
            if (++b == blocks) { b = 0; ++g; }
        }
    } else if (warp < 16) {
        // ============================================ P^T and dS^T: a warp 32 keys and 32 rows
        // in four pieces of 16 x 16 (piece c: lanes 16 (c % 2) .., rows 16 (c / 2) ..), read as 16-lane fragments: a thread has 2 keys and 4 rows of a piece, and takes 16 words of statistics a unit.
        const int h = warp >> 3, part = (warp >> 2) & 1, quarter = warp & 3;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
        const uint32_t line = base + C::kOffDS + h * C::kDSHalf + (quarter * 32 + 8 * ((lane >> 3) & 1) + (lane & 7)) * 128;
        int b = 0;
        uint32_t w = 0;
        Place unit{(uint32_t)h, 0u}, tile{(uint32_t)h, 0u}, scores{(uint32_t)h, 0u};
        for (int u = h; u < units; u += 2, ++w) {
            const uint32_t t_s = tmem + lanes + scores.at * kRowTile + 32 * part, t_dp = column_dp(scores.at, h) + lanes + 32 * part, ds = line + (w & 1) * 2 * C::kDSHalf, ready = bar(C::kReady + unit.at), ds_free = bar(C::kDSFree + (w & 1)), ds_round = ((w >> 1) - 1) & 1;
            if (!mbar_wait_warp(bar(C::kSFull + unit.at), unit.round, abort_flag, p.status) || (b == 0 && !mbar_wait_warp(bar(C::kStats + tile.at), tile.round, abort_flag, p.status))) { ok = false; break; }
            tc_fence_after();
            const int here = length - b * kKeys - quarter * 32;      // of the warp's keys; where there are none, dS is zero for good
            if (here > 0) {
                auto load = [&](int c, uint32_t (&s)[8], uint32_t (&dp)[8]) {
                    const uint32_t at = ((uint32_t)(16 * (c & 1)) << 16) + 16 * (c >> 1);
                    tmem_ld_16x256b_x2(t_s + at, s);
                    tmem_ld_16x256b_x2(t_dp + at, dp);
                };
                const float4* stats = reinterpret_cast<const float4*>(base_ptr + C::kOffStats + tile.at * C::kStatBytes) + 16 * part + (lane & 3);      // (-lse, -lse', -D, -D') of rows 8 i + 2 (lane mod 4), + 1: 4 i on
                auto work = [&](int c, const uint32_t (&s)[8], const uint32_t (&dp)[8], const float4 (&x)[2], uint32_t (&pp)[4], uint32_t (&dd)[4]) {
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {                     // keys lane / 4 and lane / 4 + 8 of the fragment
                            const int i = 4 * q + 2 * r;
                            const float2 y = __ffma2_rn(make_float2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), scale2, make_float2(x[q].x, x[q].y));
                            const float2 e = make_float2(ex2_approx(min_nan(y.x, 0.f)), ex2_approx(min_nan(y.y, 0.f)));      // (held to 1 whatever the roundings of large scores and lse make of it)
                            const float2 z = __fmul2_rn(e, __fadd2_rn(make_float2(__uint_as_float(dp[i]), __uint_as_float(dp[i + 1])), make_float2(x[q].z, x[q].w)));
                            pp[2 * q + r] = pack_bf16x2(e.x, e.y);
                            dd[2 * q + r] = pack_bf16x2(z.x, z.y);
                        }
                    if (here < 32) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (here - (lane >> 2) <= 16 * (c & 1) + 8 * (i & 1)) dd[i] = 0u;
                    }
                };
                auto store = [&](int c, const uint32_t (&pp)[4], const uint32_t (&dd)[4]) {      // P over scores that this warp has read; dS: lanes 8 m .. 8 m + 7 name the rows of block m
                    tmem_st_16x128b_x2(t_s + ((uint32_t)(16 * (c & 1)) << 16) + 8 * (c >> 1), pp);
                    stmatrix_x4(ds + 16 * (c & 1) * 128 + (((part * 4 + 2 * (c >> 1) + (lane >> 4)) ^ (lane & 7)) << 4), dd[0], dd[1], dd[2], dd[3]);
                };
                uint32_t s0[8], dp0[8], s1[8], dp1[8], pp[4], dd[4];
                float4 xa[2], xb[2];
                const bool free_yet = w < 2 || mbar_try_wait(ds_free, ds_round);      // (who read the dS before the last one)
                load(0, s0, dp0);
                load(1, s1, dp1);
                xa[0] = stats[0]; xa[1] = stats[4];
                tmem_wait_ld();
                work(0, s0, dp0, xa, pp, dd);
                if (!__all_sync(0xffffffffu, free_yet) && !mbar_wait_warp(ds_free, ds_round, abort_flag, p.status)) { ok = false; break; }
                load(2, s0, dp0);
                store(0, pp, dd);
                xb[0] = stats[8]; xb[1] = stats[12];
                work(1, s1, dp1, xa, pp, dd);
                tmem_wait_ld();
                load(3, s1, dp1);
                store(1, pp, dd);
                work(2, s0, dp0, xb, pp, dd);
                tmem_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(C::kDPFree + h));
                store(2, pp, dd);
                work(3, s1, dp1, xb, pp, dd);
                store(3, pp, dd);
                tmem_wait_st();
                fence_proxy_async();
            } else if (lane == 0) mbar_arrive(bar(C::kDPFree + h));
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ready);
            unit.step(2, 6);
            scores.step(2, 3);
            if (++b == blocks) { b = 0; tile.step(2, kStages); }
        }
        // eight warps store dV and dK
        if (ok && h == 0) {
            if (tiles > 0) {
                ok = mbar_wait_warp(bar(C::kAccFull), 0, abort_flag, p.status);
                tc_fence_after();
            }
            const float scale = part == 0 ? 1.f : p.inv_sqrt_d;
            for (int kb = 0; kb * kKeys < p.L && ok; ++kb) {
                const int key = kb * kKeys + quarter * 32 + lane;
                const bool mine = key < p.L, zero = tiles <= 0 || key >= length;
                __nv_bfloat16* dst = (part == 0 ? p.dv : p.dk) + (((long long)context * p.L + key) * p.kv_heads + kv) * p.d;
                float* sums = (part == 0 ? p.part_dv : p.part_dk) + (((long long)split * p.groups + group) * p.L + key) * DP;
#pragma unroll
                for (int c = 0; c < DP / 32; ++c) {
                    uint32_t o[32];
                    float x[32];
                    tmem_ld32(tmem + lanes + kColAcc + 2 * DP * kb + part * DP + 32 * c, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = zero ? 0.f : __uint_as_float(o[e]) * scale;
                    if (mine && p.splits > 1) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(sums + 32 * c + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                    } else if (mine) {
                        cross_store_row(dst, 32 * c, p.d, x, p.vector != 0);
                    }
                    __syncwarp();
                }
            }
        }
    } else if (warp < 24) {
        // ============================================ stores of dQ: lane r of the accumulator is row r mod 64 of the pair's tile r / 64
        const int quarter = warp & 3, row = quarter * 32 + lane, within = row & (kRowTile - 1);
        int row_token, row_head;
        p.by_group.divmod(within, row_token, row_head);
        const int head = kv * p.G + row_head;
        uint8_t* const stage = base_ptr + C::kOffOut + row * C::kRow;
        const int swizzle = DP == 32 ? (lane >> 1) & 3 : lane & 7;
        for (int g = 0; g < pairs; ++g) {
            const int acc = g % C::kDQs, token = (first + 2 * g + (row >= kRowTile ? 1 : 0)) * p.tokens_per_tile + row_token;
            const bool mine = within < p.rows_per_tile && token < p.tokens;
            if (tiles > 0) {
                if (!mbar_wait_warp(bar(C::kDQFull + acc), (g / C::kDQs) & 1, abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
            }
            if (p.tma_out) {
                if (lane == 0) bulk_wait_group_read<0>();      // the rows of before have left
                __syncwarp();
            }
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
                uint32_t o[32];
                float x[32];
                tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + kColDQ + acc * DP + 32 * c, o);
                tmem_wait_ld();
                if (c == DP / 32 - 1 && tiles > 0) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::kDQFree + acc));
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = tiles > 0 ? __uint_as_float(o[e]) * p.inv_sqrt_d : 0.f;
                if (p.tma_out) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        *reinterpret_cast<uint4*>(stage + (((4 * c + k) ^ swizzle) << 4)) = make_uint4(pack_bf16x2(x[8 * k], x[8 * k + 1]), pack_bf16x2(x[8 * k + 2], x[8 * k + 3]),
                                                                                                   pack_bf16x2(x[8 * k + 4], x[8 * k + 5]), pack_bf16x2(x[8 * k + 6], x[8 * k + 7]));
                } else if (mine) {
                    cross_store_row(p.dq + (((long long)context * p.tokens + token) * p.heads + head) * p.d, 32 * c, p.d, x, p.vector != 0);
                }
                __syncwarp();
            }
            if (p.tma_out) {
                fence_proxy_async();
                __syncwarp();
                if (lane == 0 && mine) {                  // (of the warp's first row; if that is no token, none is)
                    tma_store_4d(&tm_dq, base + C::kOffOut + quarter * 32 * C::kRow, 0, kv * p.G, token, context);
                    bulk_commit_group();
                }
            }
        }
        if (p.tma_out && lane == 0) bulk_wait_group_read<0>();
    } else {
        // ============================================ lse and D of the row tiles: two warps to a tile, a row to a thread; lse asked for two of its tiles ahead
        const int h = (warp - 24) >> 1, row = ((warp - 24) & 1) * 32 + lane;
        int row_token, row_head;
        p.by_group.divmod(row, row_token, row_head);
        const int head = kv * p.G + row_head, swizzle = DP == 32 ? (lane >> 1) & 3 : lane & 7;
        auto ask = [&](int t) {
            const int token = (first + t) * p.tokens_per_tile + row_token;
            if (t >= tiles || row >= p.rows_per_tile || token >= p.tokens) return INFINITY;      // an entry that is no row: a weight of 0 (and rows of zeros)
            int image = context, pixel = token;
            if (p.shared) p.by_pixels.divmod(token, image, pixel);
            return p.lse[((long long)image * p.heads + head) * p.pixels + pixel];
        };
        float lse = ask(h), next = ask(h + 2);
        for (int t = h; t < tiles; t += 2) {
            const float behind = ask(t + 4);
            const uint32_t st = t % kStages;
            if (!mbar_wait_warp(bar(C::kFull + st), (t / kStages) & 1, abort_flag, p.status)) { ok = false; break; }
            const uint8_t* line = base_ptr + C::kOffDO + st * C::kRowBytes + row * C::kRow;
            float2 sum[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) {
                const uint4 x = *reinterpret_cast<const uint4*>(line + (C::kOffO - C::kOffDO) + ((i ^ swizzle) << 4)), y = *reinterpret_cast<const uint4*>(line + ((i ^ swizzle) << 4));
                const uint32_t o[4] = {x.x, x.y, x.z, x.w}, g[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum[e] = __ffma2_rn(make_float2(__uint_as_float(o[e] << 16), __uint_as_float(o[e] & 0xffff0000u)), make_float2(__uint_as_float(g[e] << 16), __uint_as_float(g[e] & 0xffff0000u)), sum[e]);
            }
            float* at = reinterpret_cast<float*>(base_ptr + C::kOffStats + st * C::kStatBytes) + 4 * (row >> 1) + (row & 1);
            at[0] = -lse * kLog2e;
            at[2] = -(((sum[0].x + sum[1].x) + (sum[2].x + sum[3].x)) + ((sum[0].y + sum[1].y) + (sum[2].y + sum[3].y)));
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::kStats + st));
            lse = next;
            next = behind;
        }
    }
    if (warp >= 17 && warp < 20) {
        // everything issued by this warp has finished before the tensor memory is released
        if (elect_one()) mma_commit(bar(C::kDrain + warp - 17));
        __syncwarp();
        mbar_wait_warp(bar(C::kDrain + warp - 17), 0, abort_flag + 1, p.status);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 18) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

template <int DP, bool kLongFirst>
cudaError_t launch(const CrossProblem& p, const CrossPlan& plan, float* part_dk, float* part_dv, cudaStream_t stream)
{
    if (!encode_fn()) return cudaErrorNotSupported;
    CUtensorMap tm_q, tm_do, tm_out, tm_k, tm_v;
    const auto rows = [&](CUtensorMap* m, const void* x) { return cross_rows_map(m, x, p.contexts, p.tokens, p.heads, p.width, DP, plan.G, plan.kv_tokens_per_tile); };
    const auto keys = [&](CUtensorMap* m, const void* x) { return cross_rows_map(m, x, p.contexts, p.L, p.kv_heads, p.width, DP, 1, kKeys); };
    if (!rows(&tm_q, p.q) || !rows(&tm_do, p.dout) || !rows(&tm_out, p.out) || !keys(&tm_k, p.k) || !keys(&tm_v, p.v)) return cudaErrorInvalidValue;
    // rows of 16-byte words whose tokens fill whole warps: dQ leaves by TMA, a warp's rows at a time
    const bool tma_out = p.d % 8 == 0 && 32 % plan.G == 0;
    CUtensorMap tm_dq = tm_q;
    if (tma_out && !cross_rows_map(&tm_dq, p.dq, p.contexts, p.tokens, p.heads, p.d, DP, plan.G, 32 / plan.G)) return cudaErrorInvalidValue;
    static KernelSetup setup;
    int sms = 0;
    if (cudaError_t e = setup.prepare(rib_cross_short_bwd_kernel<DP, kLongFirst>, Cfg<DP>::kSmem, &sms)) return e;
    Params a{};
    a.lengths = p.lengths; a.lse = p.lse_in; a.dq = p.dq; a.dk = p.dk; a.dv = p.dv; a.part_dk = part_dk; a.part_dv = part_dv; a.status = p.status;
    a.d = p.d; a.L = p.L; a.heads = p.heads; a.kv_heads = p.kv_heads; a.G = plan.G; a.splits = plan.row_splits; a.pairs = plan.dq_tiles; a.pairs_per_split = plan.row_tiles_per_split / 2;
    a.rows_per_tile = plan.kv_rows_per_tile; a.tokens_per_tile = plan.kv_tokens_per_tile; a.vector = p.d % 8 == 0; a.tma_out = tma_out; a.tokens = (int)p.tokens; a.pixels = (int)p.pixels;
    a.shared = p.tokens != p.pixels; a.contexts = p.contexts; a.groups = plan.groups; a.scale_log2 = kLog2e / sqrtf((float)p.d); a.inv_sqrt_d = 1.f / sqrtf((float)p.d);
    a.by_group = make_fast_div(plan.G); a.by_pixels = make_fast_div((int)p.pixels);
    ProfileScope scope(RIB_KERNEL_CROSS_BWD_DKV, stream);
    const int grid = plan.groups * plan.row_splits;
    return launch_overtaking(rib_cross_short_bwd_kernel<DP, kLongFirst>, grid, kThreads, Cfg<DP>::kSmem, stream, tm_q, tm_do, tm_out, tm_k, tm_v, tm_dq, a);
}

}  // namespace

cudaError_t cross_bwd_short(const CrossProblem& p, const CrossPlan& plan, float* part_dk, float* part_dv, cudaStream_t stream)
{
    // One or two blocks of keys, as the contexts' lengths have it: CTAs of two first, so that none of them begins last.  Every CTA ranks the contexts for itself, which costs more than it gives when they are many.
    // Us of the call alone, two blocks first / as they come, lengths spread evenly up to 256 in no order: 4 contexts of 128 x 128 tokens, 6 heads of 32 78 / 77, 16 of 96 x 96 126 / 152, 32 of 48 x 48 88 / 95,
    // 64 of 48 x 48, 4 heads, 93 / 111, 96 of 32 x 32, 6 heads, 104 / 108, 128 of 32 x 32, 4 heads, 98 / 96, 256 of 24 x 24 133 / 127, 512 of 16 x 16 190 / 152.
    const bool long_first = p.lengths && p.L > kKeys && p.contexts > 1 && p.contexts <= 64;
    return p.d > 32 ? launch<64, false>(p, plan, part_dk, part_dv, stream) : long_first ? launch<32, true>(p, plan, part_dk, part_dv, stream) : launch<32, false>(p, plan, part_dk, part_dv, stream);
}

}  // namespace rib
