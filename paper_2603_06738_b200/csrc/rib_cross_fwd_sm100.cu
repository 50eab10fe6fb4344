// Forward pass of the attention to states (rib_cross.cuh) for B200 (sm_100a): TMA loads, tcgen05 products with accumulators in tensor memory,
// softmax in registers.
//
// Work item = up to 128 rows of one (context, kv head) group x one run of its key blocks of 64.  A CTA of five warps walks items:
//     S = Q K^T           (M128, N = 64, or what the last block has rounded up to 16; K = 32 or 64 channels)
//     P = exp2((S - m) log2e / sqrt(d)), a row to a thread, written over S as bf16
//     O (+)= P V          (A from tensor memory, V an MN-major tile)
// with a running maximum m per row that moves, and rescales O and the row's sum, only when a block exceeds it by more than 2^8 in the exponentials.  Inside a CTA
// everything runs one after the other - scores, exponentials, product, next scores -; what fills the pipes is that 4 CTAs share an SM (128 columns of tensor
// memory each: S 64, O 32 or 64; 3 CTAs with rows of 64 channels, whose tiles take 66 KB of shared memory).  The exponentials bound it: 128 x 64 of them take 512 cycles
// of the SM's special-function units, the products about 130 (d = 32) to 260 cycles.
//
// Roles: warps 0-3 softmax and output of rows 32 w .. 32 w + 31; warp 4 loads (two query tiles, a ring of key blocks) and issues the products.  Every wait is bounded.
#include "rib_cross.cuh"

namespace rib {
namespace {

using namespace sm100;

constexpr int kThreads = 160, kRows = 128;
constexpr uint32_t kTmemCols = 128, kColO = 64;

template <int DP> struct Cfg {
    static constexpr int kStages = DP == 32 ? 4 : 2, kBlocksPerSm = DP == 32 ? 4 : 3;
    static constexpr uint32_t kRow = DP * 2, kQBytes = kRows * kRow, kKBytes = kCrossBlock * kRow;
    static constexpr uint32_t kOffQ = 0, kOffK = 2 * kQBytes, kOffV = kOffK + kStages * kKBytes, kOffBar = kOffV + kStages * kKBytes;
    // barriers: query tiles, key blocks, scores there, P there, P V done, all products done
    static constexpr int kQFull = 0, kKFull = 2, kSFull = kKFull + kStages, kPReady = kSFull + 1, kPVDone = kSFull + 2, kDrain = kSFull + 3, kBars = kSFull + 4;
    static constexpr uint32_t kOffMisc = kOffBar + kBars * 8, kSmem = kOffMisc + 16 + 1024;
    static_assert(kQBytes % 1024 == 0 && kKBytes % 1024 == 0, "swizzle atoms need aligned tiles");
    static_assert(kBlocksPerSm * (kSmem + 1024) <= 233472, "shared memory of an SM");
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

template <int DP>
__global__ void __launch_bounds__(kThreads, Cfg<DP>::kBlocksPerSm)
rib_cross_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ Params p)
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
        for (int i = 0; i < C::kBars; ++i) mbar_init(bar(i), i == C::kPReady ? 4 : 1);
        fence_barrier_init();
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
    }
    if (warp == 4) {
        tmem_alloc(base + C::kOffMisc, kTmemCols);
        tmem_relinquish();
    }
    // rows that the boxes of Q do not reach (G does not divide 128)
    for (int i = 0; i < 2; ++i) cross_zero_rows(base_ptr + C::kOffQ + i * C::kQBytes, C::kRow, p.rows_per_tile, kRows, threadIdx.x, kThreads);
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;

    if (warp == 4) {
        // ============================================ loads and products: the whole warp walks, one elected lane issues
        uint32_t step = 0, live = 0;                      // key blocks and items (with blocks) whose products are complete
        uint32_t loaded = 0, q_loaded = 0;                // key blocks and query tiles asked for
        int next = blockIdx.x, next_block = 0;            // the load that comes next
        // Loads as far ahead as there is room: a stage is free once its block's P V is complete, a query tile once its item's last one is.
        auto load_ahead = [&]() {
            while (next < p.items) {
                const Item c = decode(p, next);
                if (c.blocks) {
                    if (next_block == 0 && q_loaded == live + 2) return;
                    if (loaded == step + kStages) return;
                    if (elect_one()) {
                        if (next_block == 0) {
                            const uint32_t buf = q_loaded & 1;
                            mbar_arrive_expect_tx(bar(C::kQFull + buf), (uint32_t)p.rows_per_tile * C::kRow);
                            tma_load_4d(base + C::kOffQ + buf * C::kQBytes, &tm_q, bar(C::kQFull + buf), 0, c.kv * p.G, c.tile * p.tokens_per_tile, c.context);
                        }
                        const uint32_t st = loaded % kStages;
                        const int key = (c.first + next_block) * kCrossBlock;
                        mbar_arrive_expect_tx(bar(C::kKFull + st), 2 * C::kKBytes);
                        tma_load_4d(base + C::kOffK + st * C::kKBytes, &tm_k, bar(C::kKFull + st), 0, c.kv, key, c.context);
                        tma_load_4d(base + C::kOffV + st * C::kKBytes, &tm_v, bar(C::kKFull + st), 0, c.kv, key, c.context);
                    }
                    __syncwarp();
                    if (next_block == 0) ++q_loaded;
                    ++loaded;
                    if (++next_block < c.blocks) continue;
                }
                next += gridDim.x;
                next_block = 0;
            }
        };
        for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            const Item c = decode(p, item);
            if (!c.blocks) continue;
            for (int j = 0; j < c.blocks; ++j, ++step) {
                load_ahead();
                const uint32_t st = step % kStages;
                const int keys = min(kCrossBlock, c.length - (c.first + j) * kCrossBlock), columns = (keys + 15) & ~15;
                if ((j == 0 && !mbar_wait_warp(bar(C::kQFull + (live & 1)), (live >> 1) & 1, abort_flag, p.status)) ||
                    !mbar_wait_warp(bar(C::kKFull + st), (step / kStages) & 1, abort_flag, p.status)) { ok = false; break; }
                if (keys < columns) {      // values behind the last key: weights of 0 times what lies there must not become NaN
                    cross_zero_rows(base_ptr + C::kOffV + st * C::kKBytes, C::kRow, keys, columns, lane, 32);
                    fence_proxy_async();
                    __syncwarp();
                }
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t q = smem_desc_at(T::kDesc, base + C::kOffQ + (live & 1) * C::kQBytes), k = smem_desc_at(T::kDesc, base + C::kOffK + st * C::kKBytes);
                    const uint32_t idesc = idesc_bf16_f32(kRows, columns, false);
#pragma unroll
                    for (int kk = 0; kk < DP / 16; ++kk) mma_ss(tmem, q + T::kStepK * kk, k + T::kStepK * kk, idesc, kk ? 1u : 0u);
                    mma_commit(bar(C::kSFull));
                }
                __syncwarp();
                // (the first product of an item overwrites O: the softmax warps have read it before they hand over P)
                if (!mbar_wait_warp(bar(C::kPReady), step & 1, abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t v = smem_desc_at(T::kDesc, base + C::kOffV + st * C::kKBytes);
                    constexpr uint32_t kIdesc = idesc_bf16_f32(kRows, DP, true);
                    for (int kk = 0; kk < columns / 16; ++kk) mma_ts(tmem + kColO, tmem + 8 * kk, v + T::kStepRows * kk, kIdesc, (j || kk) ? 1u : 0u);
                    mma_commit(bar(C::kPVDone));
                }
                __syncwarp();
                // the next scores go where P lies
                if (!mbar_wait_warp(bar(C::kPVDone), step & 1, abort_flag, p.status)) { ok = false; break; }
            }
            ++live;
        }
        if (!ok) {      // gave up: copies in flight land before the CTA may exit
            for (uint32_t i = step; i < loaded; ++i) mbar_wait_warp(bar(C::kKFull + i % kStages), (i / kStages) & 1, abort_flag + 1, p.status);
            for (uint32_t i = live; i < q_loaded; ++i) mbar_wait_warp(bar(C::kQFull + (i & 1)), (i >> 1) & 1, abort_flag + 1, p.status);
        }
        // what has been issued is complete before the tensor memory is released
        if (elect_one()) mma_commit(bar(C::kDrain));
        __syncwarp();
        mbar_wait_warp(bar(C::kDrain), 0, abort_flag + 1, p.status);
    } else {
        // ============================================ softmax and output: a row to a thread
        const int row = threadIdx.x;
        const uint32_t lanes = (uint32_t)(warp * 32) << 16, t_s = tmem + lanes, t_o = tmem + lanes + kColO;
        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
        const float threshold = 8.f / p.scale_log2;
        int row_token, row_head;
        p.by_group.divmod(row, row_token, row_head);
        uint32_t step = 0;
        for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            const Item c = decode(p, item);
            float m = 0.f, l = 0.f;
            for (int j = 0; j < c.blocks; ++j, ++step) {
                if (!mbar_wait_warp(bar(C::kSFull), step & 1, abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
                const int keys = c.length - (c.first + j) * kCrossBlock;
                // the scores are read twice, for their maximum and for the exponentials: 64 of them and their P do not fit the registers of a thread
                float mx0 = kCrossLowest, mx1 = kCrossLowest;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    uint32_t a[32];
                    tmem_ld32(t_s + 32 * g, a);
                    tmem_wait_ld();
                    if (keys < kCrossBlock) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (32 * g + e >= keys) a[e] = 0xff800000u;
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        mx0 = max3(mx0, __uint_as_float(a[e]), __uint_as_float(a[e + 1]));
                        mx1 = max3(mx1, __uint_as_float(a[e + 2]), __uint_as_float(a[e + 3]));
                    }
                }
                const float mx = fmaxf(mx0, mx1);
                if (j == 0) {
                    m = mx;
                } else {
                    // The reference moves, and O and l with it, only when the maximum grew by more than the threshold: the result is exact after
                    // the division since l carries the same reference.  (The last P V is complete: these scores were issued behind it.)
                    const bool need = mx > m + threshold;
                    if (__any_sync(0xffffffffu, need)) {
                        const float factor = need ? ex2_approx((m - mx) * p.scale_log2) : 1.f;
                        if (need) { l *= factor; m = mx; }
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
                // P goes where scores lie that have been read
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    uint32_t a[16], packed[8];
                    tmem_ld16(t_s + 16 * g, a);
                    tmem_wait_ld();
                    if (keys < kCrossBlock) {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (16 * g + e >= keys) a[e] = 0xff800000u;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 x = __ffma2_rn(make_float2(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1])), scale2, neg2);
                        const float2 e = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                        if (i & 1) sum_b = __fadd2_rn(sum_b, e); else sum_a = __fadd2_rn(sum_a, e);
                        packed[i] = pack_bf16x2(e.x, e.y);
                    }
                    tmem_st8(t_s + 8 * g, packed);
                }
                l += (sum_a.x + sum_a.y) + (sum_b.x + sum_b.y);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(C::kPReady));
            }
            if (!ok) break;
            if (c.blocks) {
                if (!mbar_wait_warp(bar(C::kPVDone), (step - 1) & 1, abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
            }
            const long long token = (long long)c.tile * p.tokens_per_tile + row_token;
            const bool mine = row < p.rows_per_tile && token < p.tokens;
            const bool none = c.blocks == 0;
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
            tc_fence_before();
            if (mine && p.splits > 1) {
                p.part_lse[at] = l == 0.f ? -INFINITY : lse;
            } else if (mine && p.lse) {
                int image, pixel;
                p.by_pixels.divmod((int)(c.context * p.tokens + token), image, pixel);
                p.lse[((long long)image * p.heads + head) * p.pixels + pixel] = lse;
            }
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
    const int slots = kCrossSms * Cfg<DP>::kBlocksPerSm, grid = a.items < slots ? a.items : slots;
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
    const long long items = (long long)c.groups * c.tiles, slots = (long long)kCrossSms * (p.d <= 32 ? 4 : 3);
    long long splits = items >= slots ? 1 : slots / items;
    if (splits > c.blocks) splits = c.blocks;
    c.blocks_per_split = (int)((c.blocks + splits - 1) / splits);
    c.splits = (c.blocks + c.blocks_per_split - 1) / c.blocks_per_split;
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
