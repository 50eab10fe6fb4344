// Forward window attention with a learned bias by buckets for B200 (sm_100a): tcgen05 MMAs with TMEM accumulators, TMA loads whose box
// coordinates do the window partition and the cyclic shift, softmax in registers, biases from a table in shared memory.
//
// Shapes: head width d = 8, 16, 24 or 32, window side M a multiple of 8 up to 64, shift a multiple of 8, any map.  The windows are walked as lists of
// the 8 x 8-token patches that hold tokens (LiveWindows), so that maps that are no multiples of the window, masked shifted windows and windows of
// an odd number of patches are one case; a patch that the map's edge cuts is filled up with zero rows by TMA.
//
// Work item = two query tiles of two patches each of one (head, batch item, window); it streams the window's keys in blocks of two patches:
//     S_q = Q_q K^T                                                      (M128 N128 K32)
//     P_q = exp2(S_q * log2(e) / sqrt(d) + b(key - query) - m)           softmax warps, fp32 -> bf16 written back to TMEM
//     [O_q | l_q] += P_q [V | 1]                                         (A operand from TMEM, V as an MN-major shared-memory tile)
// Pipeline, tensor memory, roles and barriers are those of the rank-r forward kernel (rib_fwd_sm100.cu): three score buffers of 128
// columns rotate among the units (block, tile), a softmax thread writes P over scores that it has read, S and PV are issued by
// warps of their own, and the row sum l is a 33rd column of the PV contraction, against a tile of ones behind V.
//
// What differs is the softmax.  Scores are read as 16-lane fragments: a thread holds four query rows of one column of their patch and, of each key
// row of the block's patch, two neighbouring keys, and finds their biases in 11 pairs of the table (rib_bias_sm100.cuh).
// There is no reference m: fp32 and bf16 carry 8 exponent bits, so the exponentials of scores (with bias) up to 69 are as exact as those of
// small ones, and a score costs one multiply-add, one exponential and half a conversion.  A row whose sum of exponentials leaves
// [2^-64, 2^100) or whose output overflows - large scores of either sign or values, rows without any key, scores that are not finite - is noted, and its item redone in the same launch
// by the exact form: running maximum, accumulators per key half, a merge.  (A reference from the window's first 32 keys, as in the rank-r kernel: 302
// us against 278 on 16 x 96 x 96 tokens in windows of 32.)  Every eighth pair of exponentials (kPolyMask) is evaluated on the FMA and integer pipes
// instead of the MUFU.  Keys beyond the map's edge have zero rows of V and, for l, zeros in the tile of ones: five half tiles for
// a whole patch, none, and one cut below, right or both.
#include "rib_bias_sm100.cuh"

namespace rib {
namespace {

using namespace sm100;

// Of every 8 pairs of scores: which go to the FMA pipe.  256 x 256 tokens in windows of 64: none 444 us, the fourth 407, the eighth 418, two 417 to 425.
constexpr uint32_t kPolyMask = 0x08u;

// 2^x for a pair of arguments on the FMA and integer pipes.  x = n + f with n = round(x), |f| <= 1/2, n read off the low mantissa bits of
// x + 1.5 * 2^23; the cubic in f (relative error 7.5e-5) times 2^n, whose exponent field n + 127 is bounded to [0, 254]: arguments below -127 (masked keys among them)
// yield 0, and those from 127 on, as some around -2^24, at least 2^126, which the epilogue sees in the row sum.  (With 2^n added to the exponent of a cubic that is scaled by 2^-120, an
// instruction less, masked keys kept a weight of 2^-120, and arguments around -2^46, whose f is large, one of up to 2^-55; with two of eight pairs 404 us.)
__device__ __forceinline__ float2 ex2_poly2_bounded(float2 x)
{
    const float2 t = __fadd2_rn(x, make_float2(12582912.f, 12582912.f));
    const float2 n = __fadd2_rn(t, make_float2(-12582912.f, -12582912.f));
    const float2 f = __fadd2_rn(x, make_float2(-n.x, -n.y));
    float2 q = __ffma2_rn(make_float2(0.05517084f, 0.05517084f), f, make_float2(0.24260935f, 0.24260935f));
    q = __ffma2_rn(q, f, make_float2(0.69326097f, 0.69326097f));
    q = __ffma2_rn(q, f, make_float2(0.99992818f, 0.99992818f));
    // bits(t) = 0x4B400000 + n for |x| < 2^22
    const int vx = __vimin_s32_relu(__float_as_int(t.x) + (127 - 0x4B400000), 254), vy = __vimin_s32_relu(__float_as_int(t.y) + (127 - 0x4B400000), 254);
    return __fmul2_rn(q, make_float2(__int_as_float(vx << 23), __int_as_float(vy << 23)));
}

constexpr int kStages = 4;            // K/V ring depth
constexpr int kThreads = 640;
constexpr int kSoftmaxThreads = 512;
constexpr int kMaxRedo = 64;          // notes a CTA takes for the exact pass, one of each softmax warp with such a row: up to 16 an item (more: all of its items are redone;
                                      // 256 x 256 tokens in windows of 64 with every row redone: 2150 us, 410 with none)

// kSFull, kPReady, kPVDone: 2 * tile + parity of the block (on_block); kDrain: one per issuing warp; kMerge: 4 * tile + quarter of the rows; kTabDone,
// kTabReady: all softmax warps are through with the old table, have written the new one
enum Bar { kQFull = 0, kQEmpty = 2, kSFull = 4, kPReady = 8, kPVDone = 12, kDrain = 16, kMerge = 19, kTabDone = 27, kTabReady, kItems, kKFull,
           kKEmpty = kKFull + kStages, kVFull = kKEmpty + kStages, kVEmpty = kVFull + kStages, kNumBars = kVEmpty + kStages };

constexpr uint32_t kHalfOnes = kContentBytes / 2;
enum Ones { kOnesAll = 0, kOnesNone, kOnesBelow, kOnesRight, kOnesBoth, kOnesTiles };

// shared-memory map (offsets from a 1024-byte aligned base)
constexpr uint32_t kOffQ = 0;                                          // [2 items][2 tiles]
constexpr uint32_t kOffK = kOffQ + 4 * kContentBytes;                  // [kStages]
constexpr uint32_t kOffV = kOffK + kStages * kContentBytes;            // [kStages]
constexpr uint32_t kOffOnes = kOffV + kStages * kContentBytes;         // half tiles of 64 keys, column 0 = 1 where the key counts: second atom of V
constexpr uint32_t kOffBar = kOffOnes + kOnesTiles * kHalfOnes;
constexpr uint32_t kOffMisc = kOffBar + kNumBars * 8;                  // tmem base, abort flags, redo count
constexpr uint32_t kOffRedo = kOffMisc + 16;                           // [kMaxRedo] item ordinals of the exact pass
constexpr uint32_t kOffMerge = (kOffRedo + kMaxRedo * 4 + 15) & ~15u;  // [2 item parities][2 tiles][2 halves][128 rows] (max, sum)
constexpr uint32_t kOffLists = kOffMerge + 8 * kTile * 8;              // PatchLists
constexpr uint32_t kOffItems = (kOffLists + sizeof(PatchLists) + 15) & ~15u;      // ItemRing
constexpr uint32_t kOffTable = kOffItems + sizeof(ItemRing);           // [(2M-1)^2] fp32
constexpr uint32_t smem_bytes(int M) { return kOffTable + 4u * (2 * M - 1) * (2 * M - 1) + 1024; }      // + slack for manual alignment
static_assert(smem_bytes(kBiasMaxWindow) <= 232448, "shared memory of one CTA");

// tensor-memory columns.  O, exact form: [2 tiles][2 key halves][32];  fast form: [2 tiles][48] (32 value columns, the row sum, 15 unused)
constexpr int kBuffers = 3;
constexpr uint32_t kColO = kBuffers * kTile, kTmemCols = 512;
static_assert(kColO + 4 * kD <= kTmemCols, "tensor memory has 512 columns");
constexpr uint32_t kFastOCols = kD + 16;

constexpr uint32_t kIdescS = idesc_bf16_f32(kTile, kTile, false);
constexpr uint32_t kIdescPV = idesc_bf16_f32(kTile, kD, true);
constexpr uint32_t kIdescPV1 = idesc_bf16_f32(kTile, kFastOCols, true);

struct Params {
    __nv_bfloat16* out;
    float* lse;
    int* status;
    int H, W, heads, d, M, s, Hp, Wp;
    int items;
    int edges;                 // H or W is no multiple of 8: some patches are cut by the map's edge
    int out_sectors;           // 1: the 16 channels of every half row of out are one 32-byte sector
    int exact_only;            // 1: skip the fast form (every item takes the exact softmax)
    float scale_log2;          // log2(e) / sqrt(d)
    BiasSource source;
    BiasItems g;
};

// `sp` counts the patches of the window that hold tokens; beyond the last one the last one stands in
__device__ __forceinline__ void patch_origin(const Params& p, const LiveItem& c, int sp, int& py, int& px, int& Y0, int& X0)
{
    live_patch_origin(p.g.live, WindowGeom{p.Hp, p.Wp, p.M, p.s}, c, min(sp, c.patches - 1), py, px, Y0, X0);
}
// The table of head h, when all softmax warps are through with the last one's.  False when a wait ran out.
__device__ __forceinline__ bool change_table(const Params& p, uint8_t* base_ptr, uint32_t base, int h, int* table_head, uint32_t* ntable)
{
    if (h == *table_head) return true;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + kOffMisc + 4);
    const uint32_t done = base + kOffBar + 8u * kTabDone, ready = base + kOffBar + 8u * kTabReady;
    const int lane = threadIdx.x & 31, side = 2 * p.M - 1;
    __syncwarp();
    if (lane == 0) mbar_arrive(done);
    if (!mbar_wait_warp(done, *ntable & 1, abort_flag, p.status)) return false;
    gather_bias(p.source, h, side * side, kTableMasked, reinterpret_cast<float*>(base_ptr + kOffTable), threadIdx.x - 128, kSoftmaxThreads);
    __syncwarp();
    if (lane == 0) mbar_arrive(ready);
    if (!mbar_wait_warp(ready, *ntable & 1, abort_flag, p.status)) return false;
    ++*ntable;
    *table_head = h;
    return true;
}

// The softmax warps' items in the exact form: a thread has one query row and one half of the keys.  Not inlined: its registers and instructions
// beside those of the fast form cost that 463 -> 428 us on 256 x 256 tokens in windows of 64.
struct ExactState { uint32_t base, tmem, blk, sb, ntable; int table_head, count, first_item; bool all_items; };
__device__ __noinline__ void exact_items(const Params& p, uint8_t* base_ptr, ExactState st)
{
    const uint32_t base = st.base;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto bar = [&](int i) { return base + kOffBar + 8u * i; };
    auto on_block = [&](int which, int tile, uint32_t block) { return bar(which + 2 * tile + (block & 1)); };
    auto parity = [](uint32_t block) { return (block >> 1) & 1; };
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + kOffMisc + 4);
    volatile int* redo_list = reinterpret_cast<volatile int*>(base_ptr + kOffRedo);
    auto first = [&](int i) { return st.first_item + (st.all_items ? i : redo_list[i]); };
    const int qt = (warp - 4) >> 3, half = ((warp - 4) >> 2) & 1, quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t lane_base = (uint32_t)(quarter * 32) << 16, t_half = st.tmem + lane_base + half * 64;
    const uint32_t pitch = 4u * (2 * p.M - 1), table_addr = base + kOffTable;
    uint32_t nmerge = 0;
    bool ok = true;
    const uint32_t t_o = st.tmem + lane_base + kColO + qt * 2 * kD;        // both halves' accumulators
    // [half][row]; two sets, so that a warp that is an item ahead of its partner does not overwrite what that one still reads
    float2* const merge_sets = reinterpret_cast<float2*>(base_ptr + kOffMerge) + qt * 2 * kTile;
    for (int i = 0; i < st.count && ok; ++i, ++nmerge) {
        const LiveItem c = decode_bias_item(p.g, first(i));
        if (!change_table(p, base_ptr, base, c.h, &st.table_head, &st.ntable)) { ok = false; break; }
        float m_used = -INFINITY, l = 0.f;          // log2 units
        const int nb = (c.patches + 1) >> 1, sp = 2 * (2 * c.tp + qt) + (row >> 6);
        int qy, qx, QY0, QX0;
        patch_origin(p, c, sp, qy, qx, QY0, QX0);
        const uint32_t q_addr = table_addr + (p.M - 1 - qy - ((row >> 3) & 7)) * pitch + 4 * (p.M - 1 - qx - (row & 7));
        for (int j = 0; j < nb; ++j, ++st.blk) {
            // warp-uniform outcome: the TMEM loads below are warp-collective
            if (!mbar_wait_warp(on_block(kSFull, qt, st.blk), parity(st.blk), abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            const uint32_t t_s = t_half + st.sb * kTile;
            st.sb = st.sb == 0 ? 2u : st.sb - 1;
            uint32_t pa[16], pb[16];
            if (2 * j + half >= c.patches) {
                // half a block without tokens (the last one of an odd number of patches)
#pragma unroll
                for (int e = 0; e < 16; ++e) pa[e] = pb[e] = 0u;
            } else {
                int py, px, Y0, X0;
                patch_origin(p, c, 2 * j + half, py, px, Y0, X0);
                const uint32_t b_addr = q_addr + py * pitch + 4 * px;
                const int rows_there = p.H - Y0, cols_there = p.W - X0;      // of the patch: keys beyond the edge are none
                uint32_t sa[32], sc[32];
                tmem_ld32(t_s, sa);
                tmem_ld32(t_s + 32, sc);
                tmem_wait_ld();
                float mx = -INFINITY;
                auto add_bias = [&](uint32_t& s, int e) {
                    const int y = e >> 3, x = e & 7;
                    const float bias = lds_f32(b_addr + y * pitch + 4 * x);
                    float v = fmaf(__uint_as_float(s), p.scale_log2, bias);
                    if (bias == kTableMasked || y >= rows_there || x >= cols_there) v = -INFINITY;
                    s = __float_as_uint(v);
                    mx = fmaxf(mx, v);
                };
#pragma unroll
                for (int e = 0; e < 32; ++e) { add_bias(sa[e], e); add_bias(sc[e], e + 32); }
                if (j == 0) {
                    m_used = mx;
                } else {
                    // Move the reference (and rescale O, l) only when the maximum grew by more than 2^8
                    const bool need = mx > m_used + 8.f;
                    if (__any_sync(0xffffffffu, need)) {
                        if (!mbar_wait_warp(on_block(kPVDone, qt, st.blk - 1), parity(st.blk - 1), abort_flag, p.status)) { ok = false; break; }
                        tc_fence_after();
                        const float factor = need ? ex2_approx(m_used - mx) : 1.f;
                        if (need) { l *= factor; m_used = mx; }
                        for (int g = 0; g < 4; ++g) {
                            uint32_t o[8];
                            tmem_ld8(t_o + half * kD + 8 * g, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                            tmem_st8(t_o + half * kD + 8 * g, o);
                        }
                    }
                }
                const float m = m_used == -INFINITY ? 0.f : m_used;      // (no key so far: every exponential is 0)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float a0 = ex2_approx(__uint_as_float(sa[2 * e]) - m), a1 = ex2_approx(__uint_as_float(sa[2 * e + 1]) - m);
                    const float b0 = ex2_approx(__uint_as_float(sc[2 * e]) - m), b1 = ex2_approx(__uint_as_float(sc[2 * e + 1]) - m);
                    l += (a0 + a1) + (b0 + b1);
                    pa[e] = pack_bf16x2(a0, a1);
                    pb[e] = pack_bf16x2(b0, b1);
                }
            }
            tmem_st16(t_s + 32, pa);
            tmem_st16(t_s + 48, pb);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(on_block(kPReady, qt, st.blk));
        }
        if (!ok) break;
        // ---- merge the two key halves and write this thread's 16 output columns
        float2* const merge = merge_sets + (nmerge & 1) * 4 * kTile;
        merge[half * kTile + row] = make_float2(m_used, l);
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kMerge + 4 * qt + quarter));
        // The partner's (m, l) must be there and the item's last PV must have completed.
        if (!mbar_wait_warp(bar(kMerge + 4 * qt + quarter), nmerge & 1, abort_flag, p.status) ||
            !mbar_wait_warp(on_block(kPVDone, qt, st.blk - 1), parity(st.blk - 1), abort_flag, p.status)) { ok = false; break; }
        tc_fence_after();
        uint32_t oa[16], ob[16];
        tmem_ld16(t_o + half * 16, oa);
        tmem_ld16(t_o + kD + half * 16, ob);
        tmem_wait_ld();
        const float2 other = merge[(half ^ 1) * kTile + row];
        tc_fence_before();
        const float m_a = half ? other.x : m_used, l_a = half ? other.y : l;
        const float m_b = half ? m_used : other.x, l_b = half ? l : other.y;
        const float m = fmaxf(m_a, m_b);
        const bool none = m == -INFINITY && l_a == 0.f && l_b == 0.f;        // a row without any key: out 0, lse -inf (one of NaN: NaN)
        const float f_a = none ? 0.f : ex2_approx(m_a - m), f_b = none ? 0.f : ex2_approx(m_b - m);
        const float l_all = l_a * f_a + l_b * f_b;
        const float w_a = none ? 0.f : f_a / l_all, w_b = none ? 0.f : f_b / l_all;
        const int Y = QY0 + ((row >> 3) & 7), X = QX0 + (row & 7);   // the patch does not straddle the border
        if (sp >= c.patches || Y >= p.H || X >= p.W) continue;
        const size_t tok = (((size_t)c.b * p.H + Y) * p.W + X) * p.heads + c.h;
        uint4* dst = reinterpret_cast<uint4*>(p.out + tok * p.d + half * 16);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            if (half * 16 + 8 * g >= p.d) break;          // a head narrower than 32 channels: the rest of the row is padding
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int e = 8 * g + 2 * k;
                w[k] = pack_bf16x2(__uint_as_float(oa[e]) * w_a + __uint_as_float(ob[e]) * w_b,
                                   __uint_as_float(oa[e + 1]) * w_a + __uint_as_float(ob[e + 1]) * w_b);
            }
            dst[g] = make_uint4(w[0], w[1], w[2], w[3]);
        }
        if (p.lse && half == 0)
            p.lse[(((size_t)c.b * p.heads + c.h) * p.H + Y) * p.W + X] = none ? -INFINITY : m * 0.69314718f + logf(l_all);
    }
}

__global__ void __launch_bounds__(kThreads, 1)
rib_bias_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ Params p)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
    auto bar = [&](int i) { return base + kOffBar + 8u * i; };
    auto on_block = [&](int which, int tile, uint32_t block) { return bar(which + 2 * tile + (block & 1)); };
    auto parity = [](uint32_t block) { return (block >> 1) & 1; };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + kOffMisc + 4);
    int* redo_count = reinterpret_cast<int*>(base_ptr + kOffMisc + 12);      // notes taken (duplicates included)
    volatile int* redo_list = reinterpret_cast<volatile int*>(base_ptr + kOffRedo);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int side = 2 * p.M - 1;
    const WindowGeom geom{p.Hp, p.Wp, p.M, p.s};
    const long long work = p.g.work[9] * p.heads;
    const int first_item = first_bias_item(p.g, work * blockIdx.x / gridDim.x);
    const int my_items = min(first_bias_item(p.g, work * (blockIdx.x + 1) / gridDim.x), p.items) - first_item;

    if (threadIdx.x == 0) {
        abort_flag[0] = 0; abort_flag[1] = 0;   // [1] stays 0: used by the drain waits
        *redo_count = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(kQFull + i), 1); mbar_init(bar(kQEmpty + i), 1);
            for (int q4 = 0; q4 < 4; ++q4) mbar_init(bar(kMerge + 4 * i + q4), 2);
        }
        for (int i = 0; i < 4; ++i) { mbar_init(bar(kSFull + i), 1); mbar_init(bar(kPVDone + i), 1); mbar_init(bar(kPReady + i), 8); }
        mbar_init(bar(kItems), 1);
        for (int i = 0; i < 3; ++i) mbar_init(bar(kDrain + i), 1);
        mbar_init(bar(kTabDone), kSoftmaxThreads / 32); mbar_init(bar(kTabReady), kSoftmaxThreads / 32);
        for (int s = 0; s < kStages; ++s) {     // keys: one commit of the S issuer; values: one commit of each PV issuer
            mbar_init(bar(kKFull + s), 1); mbar_init(bar(kKEmpty + s), 1);
            mbar_init(bar(kVFull + s), 1); mbar_init(bar(kVEmpty + s), 2);
        }
        fence_barrier_init();
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
    }
    if (warp == 2) {
        tmem_alloc(base + kOffMisc, kTmemCols);
        tmem_relinquish();
    }
    if (warp >= 4 && warp < 14) {
        // the half tiles behind V: 64 key rows of 64 bytes, SWIZZLE_64B like V, element 0 of a row = 1 where the key counts
        const int t = threadIdx.x - 128, which = t >> 6, row = t & 63;
        const bool below = which == kOnesBelow || which == kOnesBoth, right = which == kOnesRight || which == kOnesBoth;
        const bool one = which != kOnesNone && !(below && (row >> 3) >= (p.H & 7)) && !(right && (row & 7) >= (p.W & 7));
        uint4* dst = reinterpret_cast<uint4*>(base_ptr + kOffOnes + which * kHalfOnes + row * 64);
        const int sw = (row >> 1) & 3;
#pragma unroll
        for (int ck = 0; ck < 4; ++ck) dst[ck] = make_uint4(ck == sw && one ? 0x00003F80u : 0u, 0u, 0u, 0u);
        fence_proxy_async();
    }
    PatchLists* const lists = reinterpret_cast<PatchLists*>(base_ptr + kOffLists);
    fill_patch_lists(p.g, p.M, lists, threadIdx.x, kThreads);
    ItemRing* const items = reinterpret_cast<ItemRing*>(base_ptr + kOffItems);
    auto items_ready = [&](uint32_t n) { return !ItemRing::begins(n) || mbar_wait_warp(bar(kItems), ItemRing::parity(n), abort_flag, p.status); };
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    // Role state that carries over from the first pass to the exact pass: block and item counters give the barrier phases.
    uint32_t blk = 0, io = 0, ntable = 0;
    uint32_t ni = 0;                                        // place in the ring of items: each pass begins with a new eight
    int table_head = -1;
    uint32_t sb = warp == 3 || warp >= 12 ? 1u : 0u;        // score buffer of the next unit: (2 blk + tile) mod kBuffers
    uint32_t q_armed = 0, k_armed = 0, v_armed = 0;
    bool ok = true;

    for (int pass = 0; pass < 2; ++pass) {
        const bool fast = pass == 0 && !p.exact_only;
        // pass 0: every item of this CTA; pass 1: the items noted by the fast form (all of them when the notes overflowed)
        const int noted = pass == 0 ? 0 : *redo_count;
        const bool all_items = pass == 0 || noted > kMaxRedo;
        const int count = all_items ? my_items : noted;
        auto item_at = [&](int i) { return first_item + (all_items ? i : redo_list[i]); };

        ni = (ni + ItemRing::kEight - 1) / ItemRing::kEight * ItemRing::kEight;
        if (warp == 0) {
            // ============================================================ TMA producer: one lane, the others decode items
            auto box = [&](const LiveItem& c, int sp, int& Y0, int& X0) {          // beyond the last patch lies nothing: zeros
                patch_place(geom, lists, c, sp, Y0, X0);
                if (sp >= c.patches) X0 = p.Wp;
            };
            for (int i = 0; i < count && ok; ++i, ++io, ++ni) {
                if (ItemRing::begins(ni)) {
                    if (lane < ItemRing::kEight && i + lane < count) items->at(ni + lane) = decode_bias_item(p.g, item_at(i + lane));
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(kItems));
                }
                if (lane == 0) {
                    const LiveItem c = items->at(ni);
                    const uint32_t buf = io & 1;
                    if (io >= 2) ok = mbar_wait(bar(kQEmpty + buf), ((io >> 1) - 1) & 1, abort_flag, p.status);
                    if (ok) {
                        mbar_arrive_expect_tx(bar(kQFull + buf), 2 * kContentBytes);
                        ++q_armed;
                        for (int qp = 0; qp < 4; ++qp) {
                            int Y0, X0;
                            box(c, 4 * c.tp + qp, Y0, X0);
                            tma_load_5d(base + kOffQ + 2 * buf * kContentBytes + qp * kPatchContent, &tm_q, bar(kQFull + buf), 0, c.h, X0, Y0, c.b);
                        }
                    }
                    const int nb = (c.patches + 1) >> 1;
                    for (int j = 0; j < nb && ok; ++j, ++blk) {
                        const uint32_t st = blk % kStages, use = blk / kStages;
                        if (use > 0 && !mbar_wait(bar(kKEmpty + st), (use - 1) & 1, abort_flag, p.status)) { ok = false; break; }
                        mbar_arrive_expect_tx(bar(kKFull + st), kContentBytes);
                        ++k_armed;
                        int Y0[2], X0[2];
                        for (int sub = 0; sub < 2; ++sub) {
                            box(c, 2 * j + sub, Y0[sub], X0[sub]);
                            tma_load_5d(base + kOffK + st * kContentBytes + sub * kPatchContent, &tm_k, bar(kKFull + st), 0, c.h, X0[sub], Y0[sub], c.b);
                        }
                        if (use > 0 && !mbar_wait(bar(kVEmpty + st), (use - 1) & 1, abort_flag, p.status)) { ok = false; break; }
                        mbar_arrive_expect_tx(bar(kVFull + st), kContentBytes);
                        ++v_armed;
                        for (int sub = 0; sub < 2; ++sub)
                            tma_load_5d(base + kOffV + st * kContentBytes + sub * kPatchContent, &tm_v, bar(kVFull + st), 0, c.h, X0[sub], Y0[sub], c.b);
                    }
                }
                ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
            }
            if (lane == 0 && !ok) {
                // Gave up: let the copies already in flight land before the CTA may exit.
                for (uint32_t b2 = q_armed > 2u ? q_armed - 2 : 0; b2 < q_armed; ++b2)
                    mbar_wait(bar(kQFull + (b2 & 1)), (b2 >> 1) & 1, abort_flag + 1, p.status);
                for (uint32_t b2 = k_armed > (uint32_t)kStages ? k_armed - kStages : 0; b2 < k_armed; ++b2)
                    mbar_wait(bar(kKFull + b2 % kStages), (b2 / kStages) & 1, abort_flag + 1, p.status);
                for (uint32_t b2 = v_armed > (uint32_t)kStages ? v_armed - kStages : 0; b2 < v_armed; ++b2)
                    mbar_wait(bar(kVFull + b2 % kStages), (b2 / kStages) & 1, abort_flag + 1, p.status);
            }
            __syncwarp();
        } else if (warp == 1) {
            // ===================================== issuer of S = Q K^T for both query tiles
            constexpr uint64_t kDesc64 = smem_desc_const(16, 512, kSwizzle64B);
            for (int i = 0; i < count && ok; ++i, ++io, ++ni) {
                if (!items_ready(ni)) { ok = false; break; }
                const LiveItem c = items->at(ni);
                const uint32_t buf = io & 1;
                if (!mbar_wait_warp(bar(kQFull + buf), (io >> 1) & 1, abort_flag, p.status)) { ok = false; break; }
                const int nb = (c.patches + 1) >> 1;
                for (int j = 0; j < nb && ok; ++j, ++blk) {
                    const uint32_t st = blk % kStages;
                    if (!mbar_wait_warp(bar(kKFull + st), (blk / kStages) & 1, abort_flag, p.status)) { ok = false; break; }
                    const uint64_t kc = smem_desc_at(kDesc64, base + kOffK + st * kContentBytes);
#pragma unroll
                    for (int qt = 0; qt < 2; ++qt) {
                        // The scores overwrite the columns that PV of three units before, one of the other tile, reads P from: it has completed.
                        const uint32_t before = blk - 2 + qt;
                        if (!mbar_wait_warp(on_block(kPVDone, qt ^ 1, before), parity(before), abort_flag, p.status)) { ok = false; break; }
                        tc_fence_after();
                        if (elect_one()) {
                            const uint64_t qc = smem_desc_at(kDesc64, base + kOffQ + (2 * buf + qt) * kContentBytes);
                            const uint32_t d_s = tmem + sb * kTile;
                            mma_ss(d_s, qc, kc, kIdescS, 0u);
                            mma_ss(d_s, qc + 2, kc + 2, kIdescS, 1u);          // + 32 bytes: second K16 step
                            mma_commit(on_block(kSFull, qt, blk));
                            if (qt == 1) {
                                mma_commit(bar(kKEmpty + st));
                                if (j == nb - 1) mma_commit(bar(kQEmpty + buf));
                            }
                        }
                        __syncwarp();
                        sb = sb == kBuffers - 1 ? 0u : sb + 1;
                    }
                }
            }
        } else if (warp < 4) {
            // ===================================== issuers of O_q (+)= P_q V: warp 2 for query tile 0, warp 3 for tile 1
            const int qt = warp - 2;
            constexpr uint64_t kDesc64 = smem_desc_const(16, 512, kSwizzle64B);
            const uint32_t d_o = tmem + kColO + qt * 2 * kD;              // exact form: one accumulator per key half
            const uint32_t d_o1 = tmem + kColO + qt * kFastOCols;         // fast form: one accumulator
            for (int i = 0; i < count && ok; ++i, ++ni) {
                if (!items_ready(ni)) { ok = false; break; }
                const LiveItem c = items->at(ni);
                const int nb = (c.patches + 1) >> 1;
                for (int j = 0; j < nb; ++j, ++blk) {
                    const uint32_t st = blk % kStages;
                    const uint32_t v_addr = base + kOffV + st * kContentBytes;
                    // which keys of each half count (zero rows of V do for O, the half tile of ones for l)
                    uint32_t lbo[2];
#pragma unroll
                    for (int sub = 0; sub < 2; ++sub) {
                        int which = 2 * j + sub < c.patches ? kOnesAll : kOnesNone;
                        if (p.edges && which == kOnesAll) {
                            int Y0, X0;
                            patch_place(geom, lists, c, 2 * j + sub, Y0, X0);
                            const bool below = Y0 + 8 > p.H, right = X0 + 8 > p.W;
                            which = below ? (right ? kOnesBoth : kOnesBelow) : right ? kOnesRight : kOnesAll;
                        }
                        lbo[sub] = kOffOnes + which * kHalfOnes - (kOffV + st * kContentBytes + sub * kPatchContent);
                    }
                    if (!mbar_wait_warp(bar(kVFull + st), (blk / kStages) & 1, abort_flag, p.status) ||
                        !mbar_wait_warp(on_block(kPReady, qt, blk), parity(blk), abort_flag, p.status)) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t a_p = tmem + sb * kTile + 32;       // P of a key half: the second 32 of its 64 score columns, keys 32 .. 63 first
                        if (fast) {
                            // [V | ones] as one MN-major operand of 48 columns, the second 32-column atom `lbo` bytes behind the first
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk) {
                                const uint64_t v = smem_desc(v_addr, lbo[kk >> 2], 512, kSwizzle64B);
                                mma_ts(d_o1, a_p + (kk >> 2) * 64 + 8 * ((kk + 2) & 3), v + 64 * kk, kIdescPV1, (j == 0 && kk == 0) ? 0u : 1u);
                            }
                        } else {
                            const uint64_t v = smem_desc_at(kDesc64, v_addr);
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk)     // keys 16 kk ..: key half kk / 4 has its own accumulator
                                mma_ts(d_o + (kk >> 2) * kD, a_p + (kk >> 2) * 64 + 8 * (kk & 3), v + 64 * kk, kIdescPV, (j == 0 && (kk & 3) == 0) ? 0u : 1u);
                        }
                        mma_commit(on_block(kPVDone, qt, blk));
                        mma_commit(bar(kVEmpty + st));
                    }
                    __syncwarp();
                    sb = sb == 0 ? 2u : sb - 1;
                }
            }
        } else {
            // ================ softmax + epilogue: a warp has 32 query rows (4 x 8 tokens) and one half of the keys (a patch)
            const int qt = (warp - 4) >> 3;
            const int half = ((warp - 4) >> 2) & 1;
            const int quarter = warp & 3;
            const int row = quarter * 32 + lane;                 // row of the tile == TMEM lane, in the epilogue and the exact form
            const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
            const uint32_t t_half = tmem + lane_base + half * 64;       // + buffer: own scores, own P in the second 32 columns
            const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
            const uint32_t pitch = 4u * side, table_addr = base + kOffTable;

            auto need_table = [&](int h) { return change_table(p, base_ptr, base, h, &table_head, &ntable); };

            if (fast) {
                // ------------------------------------------------------------------ fast form
                const uint32_t t_o1 = tmem + lane_base + kColO + qt * kFastOCols;
                // O and l of item i are complete (the caller has waited for its last PV): normalise, store, note overflow
                // where the thread's row goes: map, pixel of the map (-1: no query) and head
                struct Place { int b, h; long long pixel; };
                auto place_of = [&](const LiveItem& c) -> Place {
                    const int sp = 2 * (2 * c.tp + qt) + (row >> 6);
                    int Y0, X0;
                    patch_place(geom, lists, c, sp, Y0, X0);
                    const int Y = Y0 + ((row >> 3) & 7), X = X0 + (row & 7);   // the patch does not straddle the border
                    return Place{c.b, c.h, sp >= c.patches || Y >= p.H || X >= p.W ? -1 : (long long)Y * p.W + X};
                };
                auto epilogue = [&](int i) {
                    const Place place = place_of(items->at(i));
                    const bool no_query = place.pixel < 0;
                    const size_t map_pixels = (size_t)p.H * p.W, tok = (place.b * map_pixels + place.pixel) * p.heads + place.h;
                    uint32_t o[16], lsum[1];
                    tmem_ld16(t_o1 + half * 16, o);
                    tmem_ld1(t_o1 + kD, lsum);
                    tmem_wait_ld();
                    tc_fence_before();
                    const float l_all = __uint_as_float(lsum[0]);
                    float2 none = make_float2(0.f, 0.f);             // 0 times the sums: NaN where one has overflowed, weights of up to 2^100 times large values
#pragma unroll
                    for (int e = 0; e < 8; ++e) none = __ffma2_rn(make_float2(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1])), make_float2(0.f, 0.f), none);
                    const bool bad = !no_query && !(l_all > 0x1p-64f && l_all < 0x1p100f && none.x + none.y == 0.f);
                    if (__any_sync(0xffffffffu, bad) && lane == 0) {
                        const int slot = atomicAdd(redo_count, 1);
                        if (slot < kMaxRedo) redo_list[slot] = i;
                    }
                    if (no_query) return;
                    const float w_o = 1.f / l_all;
                    const int channels = min(16, p.d - 16 * half);        // (a head narrower than 32 channels: the rest is padding)
                    if (channels > 0) {
                        __nv_bfloat16* dst = p.out + tok * p.d + half * 16;
                        uint32_t w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = pack_bf16x2(__uint_as_float(o[2 * e]) * w_o, __uint_as_float(o[2 * e + 1]) * w_o);
                        if (p.out_sectors) {
                            st_global_v8(dst, w);
                        } else {
                            *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
                            if (channels > 8) reinterpret_cast<uint4*>(dst)[1] = make_uint4(w[4], w[5], w[6], w[7]);
                        }
                    }
                    if (p.lse && half == 0) p.lse[((size_t)place.b * p.heads + place.h) * map_pixels + place.pixel] = logf(l_all);
                };
                for (int i = 0; i < count && ok; ++i) {              // (the first pass: item i is the ring's i-th)
                    if (!items_ready(i)) { ok = false; break; }
                    const LiveItem c = items->at(i);
                    if (!need_table(c.h)) { ok = false; break; }
                    const int nb = (c.patches + 1) >> 1;
                    // table entry of the thread's first row and a key at the window's origin, plus its place among a key row's pairs
                    const uint16_t* const list = lists->entry + list_of(c);
                    const uint16_t* const entries = list + half;
                    const uint32_t q_addr = table_addr + (p.M - 1 - 4 * (quarter & 1)) * pitch + 4 * (p.M - 1 - (lane >> 2) + 2 * (lane & 3)) - list[2 * (2 * c.tp + qt) + (quarter >> 1)];
                    // query rows of no patch: whatever lies in their scores may stand for P (4 x 96 x 96 tokens, 12 heads of 16, masked
                    // windows of 16, a third of whose query tiles are none: 55 -> 50 us; 1 % more in larger windows)
                    const bool idle = 2 * (2 * c.tp + qt) + (quarter >> 1) >= c.patches;
                    for (int j = 0; j < nb; ++j, ++blk) {
                        const uint32_t b_addr = q_addr + entries[2 * j];
                        // biases of key row k of the patch against the thread's first row; row r of it: key row k - r.  Those of the patch's second half
                        // before the wait for the scores.
                        auto bias = [&](int k) { return make_float2(lds_f32(b_addr + k * (int)pitch), lds_f32(b_addr + k * (int)pitch + 4)); };
                        float2 bb[7];
#pragma unroll
                        for (int k = 0; k < 7; ++k) bb[k] = bias(k + 1);
                        // warp-uniform outcome: the TMEM loads below are warp-collective
                        if (!mbar_wait_warp(on_block(kSFull, qt, blk), parity(blk), abort_flag, p.status)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t t_s = t_half + sb * kTile;
                        sb = sb == 0 ? 2u : sb - 1;
                        if (!idle) {
                            uint32_t a[16], b[16];
                            // 4 key rows (k0 ..) x rows 2 f, 2 f + 1; bb[0] is key row k0 - 3
                            auto work4 = [&](const uint32_t (&s)[16], const float2 (&bb)[7], int f, uint32_t t_p) {
                                uint32_t pk[8];
#pragma unroll
                                for (int g = 0; g < 4; ++g)
#pragma unroll
                                    for (int rr = 0; rr < 2; ++rr) {
                                        const int e = 4 * g + 2 * rr;
                                        const float2 x = __ffma2_rn(make_float2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), scale2, bb[g - 2 * f - rr + 3]);
                                        const float2 v = ((kPolyMask >> (2 * g + rr)) & 1u) ? ex2_poly2_bounded(x) : make_float2(ex2_approx(x.x), ex2_approx(x.y));
                                        pk[2 * g + rr] = pack_bf16x2(v.x, v.y);
                                    }
                                tmem_st_16x128b_x4(t_p, pk);
                            };
                            // P goes to the second half of the columns, whose keys are therefore taken first
                            constexpr uint32_t kLow = 16u << 16;                // lanes 16 .. 31
                            tmem_ld_16x256b_x4(t_s + 32, a);
                            tmem_ld_16x256b_x4(t_s + 32 + kLow, b);
                            tmem_wait_ld();
                            work4(a, bb, 0, t_s + 32);
                            tmem_ld_16x256b_x4(t_s, a);
                            work4(b, bb, 1, t_s + 32 + kLow);
                            tmem_ld_16x256b_x4(t_s + kLow, b);
#pragma unroll
                            for (int k = 0; k < 3; ++k) { bb[4 + k] = bb[k]; bb[k] = bias(k - 3); }      // (rows 1, 2, 3 serve again)
                            bb[3] = bias(0);
                            tmem_wait_ld();
                            work4(a, bb, 0, t_s + 48);
                            work4(b, bb, 1, t_s + 48 + kLow);
                            tmem_wait_st();
                        }
                        if (j == 0 && i > 0) {       // that PV was the last one of the item before
                            if (!mbar_wait_warp(on_block(kPVDone, qt, blk - 1), parity(blk - 1), abort_flag, p.status)) { ok = false; break; }
                            tc_fence_after();
                            epilogue(i - 1);
                        }
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(on_block(kPReady, qt, blk));
                    }
                }
                if (ok && count > 0) {
                    // the last item of the pass
                    if (mbar_wait_warp(on_block(kPVDone, qt, blk - 1), parity(blk - 1), abort_flag, p.status)) { tc_fence_after(); epilogue(count - 1); } else ok = false;
                }
            } else {
                exact_items(p, base_ptr, ExactState{base, tmem, blk, sb, ntable, table_head, count, first_item, all_items});      // (the last pass: nothing of the state is needed after it)
            }
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
                for (int b2 = 0; b2 < kept; ++b2) seen = seen || redo_list[b2] == v;
                if (!seen) redo_list[kept++] = v;
            }
            *redo_count = kept;
        }
        __syncthreads();
    }
    if (warp >= 1 && warp < 4) {
        // everything issued by this warp's leader must have finished before TMEM is released
        if (elect_one()) mma_commit(bar(kDrain + warp - 1));
        __syncwarp();
        mbar_wait(bar(kDrain + warp - 1), 0, abort_flag + 1, p.status);
    }
    // ================================================================================ common tail
    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

}  // namespace

bool sm100_bias_fwd_supported(const Problem& p)
{
    BiasItems g;
    return bias_shape_supported(p) && make_bias_items(p, 4, &g);
}

cudaError_t sm100_bias_fwd(const Problem& p, cudaStream_t stream)
{
    if (!encode_fn()) return cudaErrorNotSupported;
    CUtensorMap tm_q, tm_k, tm_v;
    if (!encode_image_map(&tm_q, p.q, p) || !encode_image_map(&tm_k, p.k, p) || !encode_image_map(&tm_v, p.v, p)) return cudaErrorInvalidValue;
    static KernelSetup setup;
    int sm_count = 0;
    if (cudaError_t e = setup.prepare(rib_bias_fwd_kernel, smem_bytes(kBiasMaxWindow), &sm_count)) return e;
    Params fp{};
    if (!make_bias_items(p, 4, &fp.g)) return cudaErrorInvalidValue;
    fp.out = p.out_w; fp.lse = p.lse_w; fp.status = p.status;
    fp.H = p.H; fp.W = p.W; fp.heads = p.heads; fp.d = p.d; fp.M = p.M; fp.s = p.s; fp.Hp = p.Hp; fp.Wp = p.Wp;
    fp.items = fp.g.per_head * p.heads;
    fp.edges = p.H % 8 != 0 || p.W % 8 != 0;
    fp.out_sectors = p.d % 16 == 0 && (reinterpret_cast<uintptr_t>(p.out_w) & 31u) == 0;
    fp.exact_only = p.exact_softmax ? 1 : 0;
    fp.scale_log2 = kLog2e / sqrtf((float)p.d);
    fp.source = bias_source(p);
    const int grid = fp.items < sm_count ? fp.items : sm_count;
    { ProfileScope scope(RIB_KERNEL_BIAS_FWD, stream); rib_bias_fwd_kernel<<<grid, kThreads, smem_bytes(p.M), stream>>>(tm_q, tm_k, tm_v, fp); }
    return cudaGetLastError();
}

}  // namespace rib
