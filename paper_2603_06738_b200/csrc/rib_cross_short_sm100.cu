// Forward pass of the attention to short sequences of states (rib_cross.cuh), a text or a learned dictionary: up to 128 of them, so that a row's scores are there at once and its largest one is known
// before the first exponential.
//     S = Q K^T (M128, N = the keys rounded up to 16),   P = exp2((S - max) log2e / sqrt(d)), written over S as bf16,   O = P V
// P is rounded once before its product, and the row's sum adds what was there before; maxima, sums and O are fp32.
//
// A persistent CTA walks a run of tiles of up to 128 rows, groups one after the other, so that K and V of a group stay in shared memory for its tiles.  Four slots of 128 columns of tensor memory, each
// with four softmax warps of its own that have a row to a thread, take the tiles in turn; inside a slot everything runs one after the other (scores, softmax, product, output), and the
// four fill one another's waits.  P lies in the first half of the scores' columns, O from column 64 on, where scores have been read.
// What bounds it is the instructions of a row beside its exponentials (waits, masks, output) and the 64-byte rows of its loads and stores, not the bytes, which would take 7 us on 180 x 320 tokens, 6 heads
// of 32, to 77 states.  That takes 18 here, and 34 in the kernel for long sequences, whose items are two tiles and whose rows have two threads that have to meet; 128 states 21 and 35, 64 x 64 x 64
// tokens to 128 74 and 127, a small map of 16 x 16 4 and 6.
//
// Roles (640 threads): warps 4 s .. 4 s + 3 softmax and output of slot s, warp 16 loads, warp 17 issues S, warp 18 P V (and owns the tensor memory).  Every wait is bounded
// (tests/test_cross_short_barriers.py is a model of them).
#include "rib_cross.cuh"

namespace rib {
namespace {

using namespace sm100;

constexpr int kThreads = 640, kRows = 128, kSlots = 4;
constexpr uint32_t kTmemCols = 512, kSlotCols = 128, kColO = 64;
constexpr float kBits = 7.f;             // weights are held down by 2^7 >= kCrossShort
static_assert(kCrossShort <= 128, "2^kBits states");

template <int DP> struct Cfg {
    static constexpr uint32_t kTiles = DP == 32 ? 6 : 4;                                           // ring of row tiles
    static constexpr uint32_t kRow = DP * 2, kTileBytes = kRows * kRow;                            // 128 rows, or 128 keys
    static constexpr uint32_t kOffQ = 0, kOffK = kTiles * kTileBytes, kOffV = kOffK + 2 * kTileBytes, kOffOut = kOffV + 2 * kTileBytes, kOffBar = kOffOut + kSlots * kTileBytes;
    // barriers: row tiles there, free; keys and values there, free; of a slot: scores there, P there, O there, O read; all products of a warp done
    static constexpr int kQFull = 0, kQEmpty = kTiles, kKVFull = 2 * kTiles, kKVEmpty = kKVFull + 2, kSFull = kKVEmpty + 2, kPReady = kSFull + kSlots, kPVDone = kPReady + kSlots,
                         kFree = kPVDone + kSlots, kDrain = kFree + kSlots, kBars = kDrain + 2;
    static constexpr uint32_t kOffMisc = kOffBar + kBars * 8, kSmem = kOffMisc + 16 + 1024;
    static_assert(kSmem <= 232448, "shared memory of a CTA");
};

struct Params {
    const int* lengths;
    __nv_bfloat16* out;
    float* lse;
    int* status;
    int d, L, heads, kv_heads, G, rows_per_tile, tokens_per_tile, tiles, all_tiles, vector, tma_out, tokens, shared, pixels;      // tiles: of a group
    float scale_log2, inv_sqrt_d;
    FastDiv by_tiles, by_kv, by_pixels, by_group;
};

// The tiles of a CTA, one after the other: those of all_tiles that its share of the run covers.  Tiles without keys are walked like the others, without products.
struct Walk {
    int tile, group, context, kv, length, left;
    uint32_t number, kvs;                // tiles before this one; groups with keys up to this one, itself included
    __device__ __forceinline__ void enter(const Params& p)
    {
        p.by_kv.divmod(group, context, kv);
        length = p.lengths ? min(max(p.lengths[context], 0), p.L) : p.L;
        if (length) ++kvs;
    }
    __device__ __forceinline__ Walk(const Params& p) : number(0), kvs(0)
    {
        const int first = (int)((long long)p.all_tiles * blockIdx.x / gridDim.x), last = (int)((long long)p.all_tiles * (blockIdx.x + 1) / gridDim.x);
        left = last - first;
        p.by_tiles.divmod(first, group, tile);
        if (left) enter(p);
    }
    __device__ __forceinline__ bool there() const { return left > 0; }
    __device__ __forceinline__ bool ends_group(const Params& p) const { return left == 1 || tile + 1 == p.tiles; }
    __device__ __forceinline__ void advance(const Params& p, int by = 1)
    {
        number += by;
        left -= by;
        tile += by;
        if (left <= 0 || tile < p.tiles) return;
        do { tile -= p.tiles; ++group; } while (tile >= p.tiles);      // (kvs counts only for those that go one by one)
        enter(p);
    }
    __device__ __forceinline__ int columns() const { return (length + 15) & ~15; }
};

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
rib_cross_short_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_out,
                           const __grid_constant__ Params p)
{
    using C = Cfg<DP>;
    using T = CrossTile<DP>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
    auto bar = [&](int i) { return base + C::kOffBar + 8u * i; };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + C::kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + C::kOffMisc + 4);      // [1] stays 0: used by the drain waits
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        abort_flag[0] = 0; abort_flag[1] = 0;
        for (int i = 0; i < C::kBars; ++i) mbar_init(bar(i), (i >= C::kPReady && i < C::kPVDone) || (i >= C::kFree && i < C::kDrain) ? 4 : 1);
        fence_barrier_init();
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
    }
    if (warp == 18) {
        tmem_alloc(base + C::kOffMisc, kTmemCols);
        tmem_relinquish();
    }
    // rows that the boxes of Q do not reach (G does not divide 128)
    for (uint32_t i = 0; i < C::kTiles; ++i) cross_zero_rows(base_ptr + C::kOffQ + i * C::kTileBytes, C::kRow, p.rows_per_tile, kRows, threadIdx.x, kThreads);
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    cudaGridDependencySynchronize();                      // it may have overtaken the kernel before
    Walk at(p);

    if (warp == 16) {
        // ============================================ loads
        uint32_t kv_asked = 0, q_asked = 0;
        for (; ok && at.there(); at.advance(p)) {
            if (at.kvs > kv_asked) {                      // a group's first tile here
                const uint32_t n = at.kvs - 1, buf = n & 1;
                if (n >= 2 && !mbar_wait_warp(bar(C::kKVEmpty + buf), ((n >> 1) - 1) & 1, abort_flag, p.status)) { ok = false; break; }
                if (elect_one()) {
                    mbar_arrive_expect_tx(bar(C::kKVFull + buf), 2 * C::kTileBytes);
                    tma_load_4d(base + C::kOffK + buf * C::kTileBytes, &tm_k, bar(C::kKVFull + buf), 0, at.kv, 0, at.context);
                    tma_load_4d(base + C::kOffV + buf * C::kTileBytes, &tm_v, bar(C::kKVFull + buf), 0, at.kv, 0, at.context);
                }
                __syncwarp();
                kv_asked = at.kvs;
            }
            const uint32_t slot = at.number % C::kTiles, use = at.number / C::kTiles;
            if (use > 0 && !mbar_wait_warp(bar(C::kQEmpty + slot), (use - 1) & 1, abort_flag, p.status)) { ok = false; break; }
            if (elect_one()) {
                mbar_arrive_expect_tx(bar(C::kQFull + slot), (uint32_t)p.rows_per_tile * C::kRow);
                tma_load_4d(base + C::kOffQ + slot * C::kTileBytes, &tm_q, bar(C::kQFull + slot), 0, at.kv * p.G, at.tile * p.tokens_per_tile, at.context);
            }
            __syncwarp();
            ++q_asked;
        }
        if (!ok) {      // gave up: copies in flight land before the CTA may exit
            for (uint32_t i = kv_asked > 2 ? kv_asked - 2 : 0; i < kv_asked; ++i) mbar_wait_warp(bar(C::kKVFull + (i & 1)), (i >> 1) & 1, abort_flag + 1, p.status);
            for (uint32_t i = q_asked > C::kTiles ? q_asked - C::kTiles : 0; i < q_asked; ++i) mbar_wait_warp(bar(C::kQFull + i % C::kTiles), (i / C::kTiles) & 1, abort_flag + 1, p.status);
        }
    } else if (warp == 17) {
        // ============================================ S
        uint32_t kv_seen = 0;
        for (; ok && at.there(); at.advance(p)) {
            const uint32_t buf = (at.kvs - 1) & 1, q_slot = at.number % C::kTiles, slot = at.number % kSlots, use = at.number / kSlots;
            if (at.kvs > kv_seen) {
                if (!mbar_wait_warp(bar(C::kKVFull + buf), ((at.kvs - 1) >> 1) & 1, abort_flag, p.status)) { ok = false; break; }
                kv_seen = at.kvs;
            }
            if (!mbar_wait_warp(bar(C::kQFull + q_slot), (at.number / C::kTiles) & 1, abort_flag, p.status) ||
                (use > 0 && !mbar_wait_warp(bar(C::kFree + slot), (use - 1) & 1, abort_flag, p.status))) { ok = false; break; }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t q = smem_desc_at(T::kDesc, base + C::kOffQ + q_slot * C::kTileBytes), k = smem_desc_at(T::kDesc, base + C::kOffK + buf * C::kTileBytes);
                const uint32_t idesc = idesc_bf16_f32(kRows, at.columns(), false);
                if (at.length)
#pragma unroll
                    for (int kk = 0; kk < DP / 16; ++kk) mma_ss(tmem + slot * kSlotCols, q + T::kStepK * kk, k + T::kStepK * kk, idesc, kk ? 1u : 0u);
                mma_commit(bar(C::kSFull + slot));
                mma_commit(bar(C::kQEmpty + q_slot));
            }
            __syncwarp();
        }
    } else if (warp == 18) {
        // ============================================ P V
        uint32_t kv_seen = 0;
        for (; ok && at.there(); at.advance(p)) {
            const uint32_t buf = (at.kvs - 1) & 1, slot = at.number % kSlots;
            const int columns = at.columns();
            if (at.kvs > kv_seen) {
                if (!mbar_wait_warp(bar(C::kKVFull + buf), ((at.kvs - 1) >> 1) & 1, abort_flag, p.status)) { ok = false; break; }
                kv_seen = at.kvs;
                if (at.length < columns) {      // values behind the last key: weights of 0 times what lies there must not become NaN
                    cross_zero_rows(base_ptr + C::kOffV + buf * C::kTileBytes, C::kRow, at.length, columns, lane, 32);
                    fence_proxy_async();
                    __syncwarp();
                }
            }
            if (!mbar_wait_warp(bar(C::kPReady + slot), (at.number / kSlots) & 1, abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t v = smem_desc_at(T::kDesc, base + C::kOffV + buf * C::kTileBytes);
                constexpr uint32_t kIdesc = idesc_bf16_f32(kRows, DP, true);
                for (int kk = 0; kk < columns / 16; ++kk) mma_ts(tmem + slot * kSlotCols + kColO, tmem + slot * kSlotCols + 8 * kk, v + T::kStepRows * kk, kIdesc, kk ? 1u : 0u);
                mma_commit(bar(C::kPVDone + slot));
                if (at.length && at.ends_group(p)) mma_commit(bar(C::kKVEmpty + buf));
            }
            __syncwarp();
        }
    } else if (warp < 16) {
        // ============================================ softmax and output: a row to a thread
        const uint32_t slot = warp >> 2;
        const int quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t t_s = tmem + ((uint32_t)(quarter * 32) << 16) + slot * kSlotCols;
        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
        int row_token, row_head;
        p.by_group.divmod(row, row_token, row_head);
        const int warp_token = __shfl_sync(0xffffffffu, row_token, 0);
        uint8_t* const stage = base_ptr + C::kOffOut + warp * 32 * C::kRow + lane * C::kRow;
        const int swizzle = DP == 32 ? (lane >> 1) & 3 : lane & 7;
        if (slot) at.advance(p, slot);
        for (; ok && at.there(); at.advance(p, kSlots)) {
            const int token = at.tile * p.tokens_per_tile + row_token, head = at.kv * p.G + row_head;
            const bool mine = row < p.rows_per_tile && token < p.tokens;
            const uint32_t phase = (at.number / kSlots) & 1;
            // (rows of a warp that are no tokens take part in the waits alone; what they leave behind is nobody's)
            const bool idle = at.tile * p.tokens_per_tile + warp_token >= p.tokens || quarter * 32 >= p.rows_per_tile;
            if (!mbar_wait_warp(bar(C::kSFull + slot), phase, abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            float most = kCrossLowest, l = 0.f;
            if (!idle) {
                // 32 keys at a time, and the last 16 or 32 with what lies behind them masked
                const int whole = at.length & ~31, rest = at.length - whole;
                float mx[4] = {kCrossLowest, kCrossLowest, kCrossLowest, kCrossLowest};
                float2 neg2, sum_a = make_float2(0.f, 0.f), sum_b = make_float2(0.f, 0.f);
                auto mask = [&](auto& a) {
#pragma unroll
                    for (int e = 0; e < (int)(sizeof(a) / 4); ++e)
                        if (e >= rest) a[e] = 0xff800000u;
                };
                auto maximum = [&](const auto& a) {
#pragma unroll
                    for (int e = 0; e < (int)(sizeof(a) / 4); e += 2) mx[e / 2 % 4] = max3(mx[e / 2 % 4], __uint_as_float(a[e]), __uint_as_float(a[e + 1]));
                };
                auto weights = [&](const auto& a, auto& packed) {
#pragma unroll
                    for (int i = 0; i < (int)(sizeof(a) / 8); ++i) {
                        const float2 x = __ffma2_rn(__fadd2_rn(make_float2(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1])), neg2), scale2, make_float2(-kBits, -kBits));
                        const float2 e = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                        if (i & 1) sum_b = __fadd2_rn(sum_b, e); else sum_a = __fadd2_rn(sum_a, e);
                        packed[i] = pack_bf16x2(e.x, e.y);
                    }
                };
#pragma unroll 1
                for (int g = 0; g < whole; g += 32) {
                    uint32_t a[32];
                    tmem_ld32(t_s + g, a);
                    tmem_wait_ld();
                    maximum(a);
                }
                if (rest > 16) {
                    uint32_t a[32];
                    tmem_ld32(t_s + whole, a);
                    tmem_wait_ld();
                    mask(a);
                    maximum(a);
                } else if (rest) {
                    uint32_t a[16];
                    tmem_ld16(t_s + whole, a);
                    tmem_wait_ld();
                    mask(a);
                    maximum(a);
                }
                most = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
                neg2 = make_float2(-most, -most);
                // the weights go where scores lie that have been read
#pragma unroll 1
                for (int g = 0; g < whole; g += 32) {
                    uint32_t a[32], packed[16];
                    tmem_ld32(t_s + g, a);
                    tmem_wait_ld();
                    weights(a, packed);
                    tmem_st16(t_s + g / 2, packed);
                }
                if (rest > 16) {
                    uint32_t a[32], packed[16];
                    tmem_ld32(t_s + whole, a);
                    tmem_wait_ld();
                    mask(a);
                    weights(a, packed);
                    tmem_st16(t_s + whole / 2, packed);
                } else if (rest) {
                    uint32_t a[16], packed[8];
                    tmem_ld16(t_s + whole, a);
                    tmem_wait_ld();
                    mask(a);
                    weights(a, packed);
                    tmem_st8(t_s + whole / 2, packed);
                }
                l = (sum_a.x + sum_a.y) + (sum_b.x + sum_b.y);
                tmem_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::kPReady + slot));
            if (p.tma_out) {
                if (lane == 0) bulk_wait_group_read<0>();      // the rows of before have left
                __syncwarp();
            }
            if (!mbar_wait_warp(bar(C::kPVDone + slot), phase, abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            const float inverse = __fdividef(1.f, l);            // (without keys the output is 0, and -inf its logarithm)
#pragma unroll
            for (int g = 0; g < DP / 32; ++g) {
                uint32_t o[32];
                float x[32];
                tmem_ld32(t_s + kColO + 32 * g, o);
                tmem_wait_ld();
                if (g == DP / 32 - 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::kFree + slot));
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = at.length ? __uint_as_float(o[e]) * inverse : 0.f;
                if (p.tma_out) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        *reinterpret_cast<uint4*>(stage + (((4 * g + k) ^ swizzle) << 4)) = make_uint4(pack_bf16x2(x[8 * k], x[8 * k + 1]), pack_bf16x2(x[8 * k + 2], x[8 * k + 3]),
                                                                                                   pack_bf16x2(x[8 * k + 4], x[8 * k + 5]), pack_bf16x2(x[8 * k + 6], x[8 * k + 7]));
                } else if (mine) {
                    cross_store_row(p.out + ((long long)(at.context * p.tokens + token) * p.heads + head) * p.d, 32 * g, p.d, x, p.vector != 0);
                }
                __syncwarp();
            }
            if (p.tma_out) {
                fence_proxy_async();
                __syncwarp();
                if (lane == 0 && mine) {                  // (of the warp's first row; if that is no token, none is)
                    tma_store_4d(&tm_out, base + C::kOffOut + warp * 32 * C::kRow, 0, at.kv * p.G, token, at.context);
                    bulk_commit_group();
                }
            }
            if (p.lse && mine) {
                int image = at.context, pixel = token;
                if (p.shared) p.by_pixels.divmod(token, image, pixel);
                p.lse[(long long)(image * p.heads + head) * p.pixels + pixel] = most * p.inv_sqrt_d + (__logf(l) + kBits * 0.6931471805599453f);
            }
            __syncwarp();
        }
        if (p.tma_out && lane == 0) bulk_wait_group_read<0>();      // (the CTA's shared memory is read until then)
    }
    if (warp == 17 || warp == 18) {
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

template <int DP>
cudaError_t launch(const CrossProblem& p, const CrossPlan& plan, cudaStream_t stream)
{
    if (!encode_fn()) return cudaErrorNotSupported;
    CUtensorMap tm_q, tm_k, tm_v;
    if (!cross_rows_map(&tm_q, p.q, p.contexts, p.tokens, p.heads, p.width, DP, plan.G, plan.tokens_per_tile) || !cross_rows_map(&tm_k, p.k, p.contexts, p.L, p.kv_heads, p.width, DP, 1, kRows) ||
        !cross_rows_map(&tm_v, p.v, p.contexts, p.L, p.kv_heads, p.width, DP, 1, kRows))
        return cudaErrorInvalidValue;
    // rows of 16-byte words whose tokens fill whole warps: the output leaves by TMA, a warp's rows at a time
    const bool tma_out = p.d % 8 == 0 && 32 % plan.G == 0;
    CUtensorMap tm_out = tm_q;
    if (tma_out && !cross_rows_map(&tm_out, p.out_w, p.contexts, p.tokens, p.heads, p.d, DP, plan.G, 32 / plan.G)) return cudaErrorInvalidValue;
    static KernelSetup setup;
    int sms = 0;
    if (cudaError_t e = setup.prepare(rib_cross_short_fwd_kernel<DP>, Cfg<DP>::kSmem, &sms)) return e;
    Params a{};
    a.lengths = p.lengths; a.out = p.out_w; a.lse = p.lse_w; a.status = p.status;
    a.d = p.d; a.L = p.L; a.heads = p.heads; a.kv_heads = p.kv_heads; a.G = plan.G; a.rows_per_tile = plan.rows_per_tile; a.tokens_per_tile = plan.tokens_per_tile; a.tiles = plan.tiles;
    a.all_tiles = plan.groups * plan.tiles; a.vector = p.d % 8 == 0; a.tma_out = tma_out; a.tokens = (int)p.tokens; a.shared = p.tokens != p.pixels; a.pixels = (int)p.pixels;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)p.d); a.inv_sqrt_d = 1.f / sqrtf((float)p.d);
    a.by_tiles = make_fast_div(plan.tiles); a.by_kv = make_fast_div(p.kv_heads); a.by_pixels = make_fast_div((int)p.pixels); a.by_group = make_fast_div(plan.G);
    const int grid = a.all_tiles < kCrossSms ? a.all_tiles : kCrossSms;
    ProfileScope scope(RIB_KERNEL_CROSS_FWD, stream);
    return launch_overtaking(rib_cross_short_fwd_kernel<DP>, grid, kThreads, Cfg<DP>::kSmem, stream, tm_q, tm_k, tm_v, tm_out, a);
}

}  // namespace

cudaError_t cross_fwd_short(const CrossProblem& p, const CrossPlan& plan, cudaStream_t stream) { return p.d <= 32 ? launch<32>(p, plan, stream) : launch<64>(p, plan, stream); }

}  // namespace rib
