// Backward window attention with a learned bias by buckets for B200 (sm_100a): the chain rule of the softmax as five tcgen05 contractions
// per (query tile, key block) with TMEM accumulators and TMA loads, the probabilities recomputed from lse, and the gradient of the bias summed
// by offset on the way.
//
// Shapes and windows: as the forward (rib_bias_fwd_sm100.cu).  Work item = one key block of two patches of one (head, batch item, window); a persistent
// CTA keeps K_J and V_J in shared memory and dV_J, dK_J in tensor memory, and walks the query tiles I of the window.  The pipeline, its roles and
// its barriers are those of the rank-r backward kernel (rib_bwd_sm100.cu, rank 16), everything transposed (keys on the TMEM lanes), the unit
// a half-tile u = 2 I + h of the 64 queries of one patch:
//     S^T  = K_J Q_u^T - lse_i sqrt(d),   dP^T = V_J dO_u^T - D_i                                (M128 N64 K32 + 16)
//     P^T  = exp2(S^T * log2(e) / sqrt(d) + b(key - query)),   dS^T = P^T o dP^T                 (arithmetic warps)
//     dV_J += P^T dO_u,   dK_J += dS^T Q_u                                                       (A from TMEM, N = 32)
// and once per tile  dQ_I = dS K_J  (A = dS in shared memory, N = 32), added (fp32 red) into a workspace [pair][group of 4 columns][token][4].
//
// lse and D of the queries enter through the contractions: their negatives as three bf16 parts (24 bits) against columns of ones, one step of 16 more in
// each, so that a score costs one multiply-add, one exponential, one product and one conversion (16 x 96 x 96
// tokens, 6 heads, windows of 32: 725 -> 670 us; as floats from the ring of tiles they were read by every thread).
// Biases: an arithmetic warp has 4 x 8 keys and 4 x 8 queries of a unit, a thread 4 rows of one key column and 2 neighbouring query columns of 4
// rows: 7 pairs of the table in shared memory serve its 32 scores (rib_bias_sm100.cuh).
//
// Gradient of the bias: the sum of dS over all pairs of tokens at the same offset.  Four warps of their own take the dS tile that dQ reads from
// shared memory (bf16, as dQ and dK see it), one patch of keys against one of queries each: 64 blocks of 8 x 8 (key row, query row).
// Warp-level MMAs against constant 0/1 matrices sum the 4096 of them along both diagonals in fp32, which leaves the 15 x 15 offsets of the two
// patches, and those are added to the sums of the patches' difference (BiasGrad) eight bytes at a time.
#include "rib_bias_sm100.cuh"

namespace rib {
namespace {

using namespace sm100;

constexpr int kQStages = 3;           // ring of query-side tiles (Q, dO, rows of lse and D)
constexpr int kMaxSlots = 4;          // K and V of items in flight.  The scores are three half-tiles ahead of the drains, which in windows of 16 is an item: with two
                                      // slots the next item's K arrived too late (4 x 96 x 96 tokens, 12 heads, d = 16, windows of 16: 142 us; three 119, four 116)
constexpr int kThreads = 896;
constexpr int kArithmeticThreads = 512;

// shared-memory map (offsets from a 1024-byte aligned base)
constexpr uint32_t kOffRing = 0;
constexpr uint32_t kLdPatch = 64 * 16, kLdBytes = 2 * kLdPatch;  // per query 8 bf16: -lse sqrt(d) and -D in three parts each, 0, 0
constexpr uint32_t kRingQ = 0, kRingDO = kContentBytes, kRingLD = kRingDO + kContentBytes;
constexpr uint32_t kRingBytes = kRingLD + kLdBytes;              // 18432
constexpr uint32_t kOffDS = kOffRing + kQStages * kRingBytes;    // dS: [2 tiles][2 halves of 64 queries][128 keys][128 B], SWIZZLE_128B
constexpr uint32_t kDSHalf = kTile * 128;
constexpr uint32_t kOffDK = kOffDS + 4 * kDSHalf;                // dK rows of an item on their way out (dV rows leave through V's slot)
constexpr uint32_t kOffBar = kOffDK + kContentBytes;
// kSFull, kPReady, kPFree: unit mod 4 (on_unit); kDSFree: per dS tile buffer.  A parity wait cannot tell "two phases ahead" from "not yet", so a
// barrier's next phase must not be able to complete before every waiter has seen the current one: the next phases of kPReady of the units 2 g,
// 2 g + 1 belong to tile g + 2, whose dS buffer is released by dQ of tile g and by the four warps that sum the bias gradient.
enum Bar { kKVFull = 0, kKVEmpty = kMaxSlots, kQFull = 2 * kMaxSlots, kQEmpty = kQFull + kQStages, kSFull = kQEmpty + kQStages, kPReady = kSFull + 4, kPFree = kPReady + 4,
           kDSFree = kPFree + 4, kDQFull = kDSFree + 2, kDQFree, kAccFull, kAccFree, kTabDone, kTabReady, kItems, kDrain, kNumBars = kDrain + 3 };
constexpr uint32_t kOffMisc = kOffBar + kNumBars * 8;
constexpr uint32_t kOffMasked = kOffMisc + 16;                   // biases of a key that is none
// [S, dP] rows of 8 bf16 for all keys: 1 for the parts of -lse sqrt(d) (S) or of -D (dP).  The rows are alike, so the groups of 8 that an MMA reads
// begin one row behind each other.
constexpr uint32_t kOnesBytes = (kTile / 8 + 8) * 16;
constexpr uint32_t kOffOnes = (kOffMasked + 16 + 127) & ~127u;
constexpr uint32_t kOffZero = kOffOnes + 2 * kOnesBytes;         // zeros: columns 8 .. 15 of the queries' parts, and rows of dS that do not count
constexpr uint32_t kOffLists = kOffZero + 1024;                  // PatchLists
static_assert(kOffZero % 128 == 0, "lines of 128 bytes");
constexpr uint32_t kOffItems = (kOffLists + sizeof(PatchLists) + 15) & ~15u;      // ItemRing
constexpr uint32_t kOffTable = kOffItems + sizeof(ItemRing);     // [(2M-1)^2] fp32
// behind the table: K and V of the items in flight, as many as there is room for
constexpr uint32_t kMaxShared = 232448, kSlotBytes = 2 * kContentBytes;
constexpr uint32_t slots_offset(int M) { return (kOffTable + 4u * (2 * M - 1) * (2 * M - 1) + 1023u) & ~1023u; }
constexpr int slots_of(int M)
{
    int slots = 2;
    while (slots < kMaxSlots && slots_offset(M) + (slots + 1) * kSlotBytes + 1024 <= kMaxShared) ++slots;
    return slots;
}
constexpr uint32_t smem_bytes(int M) { return slots_offset(M) + slots_of(M) * kSlotBytes + 1024; }      // + slack for manual alignment
constexpr uint32_t most_shared()
{
    uint32_t most = 0;
    for (int M = 8; M <= kBiasMaxWindow; M += 8) most = smem_bytes(M) > most ? smem_bytes(M) : most;
    return most;
}
static_assert(most_shared() <= kMaxShared, "shared memory of one CTA");
static_assert(kOffRing % 1024 == 0 && kRingBytes % 1024 == 0 && kOffDS % 1024 == 0, "swizzle atoms need aligned tiles");

// tensor-memory columns: S^T of unit u in buffer u mod 3 (64 fp32 columns) and dP^T beside it; a warp writes P^T over its own scores and dS^T over its
// dP^T: 32 queries in the first 16 of its 32 columns
constexpr uint32_t kBuffers = 3;
constexpr uint32_t kStep = 128, kColDP = 64, kColDV = kBuffers * kStep, kColDK = kColDV + kD, kColDQ = kColDK + kD;
static_assert(kColDQ + kD <= 512, "tensor memory has 512 columns");
constexpr uint32_t kTmemCols = 512;

constexpr uint32_t kIdescSS = idesc_bf16_f32(kTile, kTile / 2, false);        // both operands K-major
constexpr uint32_t kIdescT = idesc_bf16_f32(kTile, kD, true);                 // A in TMEM, B MN-major, N = 32
constexpr uint32_t kIdescQ = idesc_bf16_f32_ab(kTile, kD, true, true);        // A and B MN-major

struct Params {
    const uint4* ld;           // [pairs][n], patches of the window in rows: per query the parts of -lse sqrt(d) and -D; then one patch of no queries
    float* dq_acc;             // [pairs][columns / 4][n][4] fp32, zeroed by the preparation kernel
    float* blocks;             // BiasGrad::blocks
    int* status;
    long long no_queries;      // element of ld where the patch of no queries begins
    int H, W, heads, columns, M, s, n, nWy, nWx, Hp, Wp;
    int items;
    int slots;                 // of K and V
    uint32_t slots_at;         // in shared memory
    float scale_log2;          // log2(e) / sqrt(d)
    float inv_sqrt_d;
    BiasSource source;
    BiasItems g;
};

__device__ __forceinline__ size_t pair_of(const Params& p, const LiveItem& c)
{
    return (((size_t)c.b * p.nWy + c.wy) * p.nWx + c.wx) * p.heads + c.h;
}

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// d (16 x 8, fp32) += a (16 x 16, bf16) * b (16 x 8, bf16), warp-level
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void red_add_f32x2(float* addr, float a, float b)
{
    asm volatile("red.relaxed.gpu.global.add.v2.f32 [%0], {%1, %2};" ::"l"(addr), "f"(a), "f"(b) : "memory");
}

// kCut: the map's edge cuts patches (H or W is no multiple of 8).  A kernel of its own: what the loops of all roles together take of the instruction cache
// decides its time, and with both forms of the arithmetic in one kernel it was 850 or 690 us, as the code happened to lie, against 715.
template <bool kCut>
__global__ void __launch_bounds__(kThreads, 1)
rib_bias_bwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_dk, const __grid_constant__ CUtensorMap tm_dv,
                    const __grid_constant__ Params p)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
    auto bar = [&](int i) { return base + kOffBar + 8u * i; };
    // of kSFull, kPReady, kPFree: the barrier of a unit and the parity of its phase.  (Units -1 to -3 have the parity that a barrier without a
    // completed phase answers yes to.)
    auto on_unit = [&](int which, uint32_t unit) { return bar(which + (int)(unit & 3)); };
    auto unit_parity = [](uint32_t unit) { return (unit >> 2) & 1; };
    auto buffer_after = [](uint32_t buffer, uint32_t units) { buffer += units; return buffer >= kBuffers ? buffer - kBuffers : buffer; };
    // an item's slot and how often the slots have gone round, odd or even
    const uint32_t slots = p.slots;
    auto k_slot = [&](uint32_t slot) { return base + p.slots_at + slot * kSlotBytes; };
    auto next_slot = [&](uint32_t& slot, uint32_t& round) { if (++slot == slots) { slot = 0; round ^= 1; } };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + kOffMisc + 4);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int side = 2 * p.M - 1;
    const WindowGeom geom{p.Hp, p.Wp, p.M, p.s};
    const long long work = p.g.work[9] * p.heads;
    const int first_item = first_bias_item(p.g, work * blockIdx.x / gridDim.x);
    const int last_item = min(first_bias_item(p.g, work * (blockIdx.x + 1) / gridDim.x), p.items);

    if (threadIdx.x == 0) {
        abort_flag[0] = 0; abort_flag[1] = 0;   // [1] stays 0: used by the drain waits
        for (int s = 0; s < kMaxSlots; ++s) { mbar_init(bar(kKVFull + s), 1); mbar_init(bar(kKVEmpty + s), 5); }     // empty: the item's last dQ, and V's slot by the four warps whose dV leaves through it
        for (int s = 0; s < kQStages; ++s) { mbar_init(bar(kQFull + s), 1); mbar_init(bar(kQEmpty + s), 1); }
        for (int h = 0; h < 2; ++h) mbar_init(bar(kDSFree + h), 5);        // dQ and the four warps of the bias gradient
        for (int i = 0; i < 4; ++i) { mbar_init(bar(kSFull + i), 1); mbar_init(bar(kPReady + i), 8); mbar_init(bar(kPFree + i), 1); }
        mbar_init(bar(kDQFull), 1); mbar_init(bar(kDQFree), 4);
        mbar_init(bar(kAccFull), 1); mbar_init(bar(kAccFree), 4);
        mbar_init(bar(kTabDone), kArithmeticThreads / 32); mbar_init(bar(kTabReady), kArithmeticThreads / 32);
        mbar_init(bar(kItems), 1);
        for (int i = 0; i < 3; ++i) mbar_init(bar(kDrain + i), 1);
        fence_barrier_init();
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
        prefetch_tensormap(&tm_do); prefetch_tensormap(&tm_dk); prefetch_tensormap(&tm_dv);
    }
    if (warp == 2) {
        tmem_alloc(base + kOffMisc, kTmemCols);
        tmem_relinquish();
    }
    PatchLists* const lists = reinterpret_cast<PatchLists*>(base_ptr + kOffLists);
    fill_patch_lists(p.g, p.M, lists, threadIdx.x, kThreads);
    ItemRing* const items = reinterpret_cast<ItemRing*>(base_ptr + kOffItems);
    auto items_ready = [&](uint32_t n) { return !ItemRing::begins(n) || mbar_wait_warp(bar(kItems), ItemRing::parity(n), abort_flag, p.status); };
    if (threadIdx.x < (2 * kOnesBytes + 1024) / 16) {
        constexpr uint32_t kTwo = 0x3F803F80u, kFirst = 0x00003F80u, kSecond = 0x3F800000u;
        const uint32_t at = threadIdx.x * 16;
        reinterpret_cast<uint4*>(base_ptr + kOffOnes)[threadIdx.x] = at < kOnesBytes ? make_uint4(kTwo, kFirst, 0u, 0u) : at < 2 * kOnesBytes ? make_uint4(0u, kSecond, kTwo, 0u) : make_uint4(0u, 0u, 0u, 0u);
    }
    if (threadIdx.x < 4) reinterpret_cast<float*>(base_ptr + kOffMasked)[threadIdx.x] = -INFINITY;
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    cudaGridDependencySynchronize();              // the preparation kernel, which this one may have overtaken: lse and D, cleared sums

    if (warp == 0) {
        // ============================================================ TMA producer: one lane, the others decode items
        uint32_t slot = 0, round = 0, kv_armed = 0, q_armed = 0;
        bool ok = true;
        for (uint32_t nitem = 0; first_item + (int)nitem < last_item && ok; ++nitem, next_slot(slot, round)) {
            if (ItemRing::begins(nitem)) {
                const int item = first_item + (int)nitem + lane;
                if (lane < ItemRing::kEight && item < last_item) items->at(nitem + lane) = decode_bias_item(p.g, item);
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kItems));
            }
            if (lane == 0) {
                const LiveItem c = items->at(nitem);
                // (a barrier that has completed no phase answers yes to parity 1)
                ok = mbar_wait(bar(kKVEmpty + slot), round ^ 1, abort_flag, p.status);
                if (ok) {
                    mbar_arrive_expect_tx(bar(kKVFull + slot), kSlotBytes);
                    ++kv_armed;
                    for (int sub = 0; sub < 2; ++sub) {
                        int Y0, X0;
                        patch_place(geom, lists, c, 2 * c.tp + sub, Y0, X0);
                        if (2 * c.tp + sub >= c.patches) X0 = p.Wp;          // beyond the last patch lies nothing: zeros
                        tma_load_5d(k_slot(slot) + sub * kPatchContent, &tm_k, bar(kKVFull + slot), 0, c.h, X0, Y0, c.b);
                        tma_load_5d(k_slot(slot) + kContentBytes + sub * kPatchContent, &tm_v, bar(kKVFull + slot), 0, c.h, X0, Y0, c.b);
                    }
                }
                const size_t pair = pair_of(p, c);
                const int tiles = (c.patches + 1) >> 1;
                for (int I = 0; I < tiles && ok; ++I, ++q_armed) {
                    const uint32_t st = q_armed % kQStages, use = q_armed / kQStages;
                    if (use > 0 && !mbar_wait(bar(kQEmpty + st), (use - 1) & 1, abort_flag, p.status)) { ok = false; break; }
                    mbar_arrive_expect_tx(bar(kQFull + st), kRingBytes);
                    const uint32_t to = base + kOffRing + st * kRingBytes;
                    for (int sub = 0; sub < 2; ++sub) {
                        int Y0, X0;
                        patch_place(geom, lists, c, 2 * I + sub, Y0, X0);
                        const int from = lists->origin[list_of(c) + 2 * I + sub];
                        const bool none = 2 * I + sub >= c.patches;
                        if (none) X0 = p.Wp;
                        tma_load_5d(to + kRingQ + sub * kPatchContent, &tm_q, bar(kQFull + st), 0, c.h, X0, Y0, c.b);
                        tma_load_5d(to + kRingDO + sub * kPatchContent, &tm_do, bar(kQFull + st), 0, c.h, X0, Y0, c.b);
                        const size_t at = none ? (size_t)p.no_queries : pair * p.n + 64 * (size_t)((from >> 11) * (p.M >> 3) + ((from & 255) >> 3));
                        bulk_load_1d(to + kRingLD + sub * kLdPatch, p.ld + at, kLdPatch, bar(kQFull + st));
                    }
                }
            }
            ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
        }
        if (lane == 0 && !ok) {
            // Gave up: let the copies already in flight land before the CTA may exit.
            for (uint32_t b2 = kv_armed > slots ? kv_armed - slots : 0; b2 < kv_armed; ++b2)
                mbar_wait(bar(kKVFull + b2 % slots), (b2 / slots) & 1, abort_flag + 1, p.status);
            for (uint32_t b2 = q_armed > (uint32_t)kQStages ? q_armed - kQStages : 0; b2 < q_armed; ++b2)
                mbar_wait(bar(kQFull + b2 % kQStages), (b2 / kQStages) & 1, abort_flag + 1, p.status);
        }
        __syncwarp();
    } else if (warp < 4) {
        // ============================================ MMA issuers: warps 1-3, the whole warp walks the
        // loops and waits (warp-uniform outcomes), one elected lane issues
        constexpr uint64_t kDesc64 = smem_desc_const(16, 512, kSwizzle64B);
        constexpr uint64_t kDescDS = smem_desc_const(kDSHalf, 1024, kSwizzle128B);    // MN-major: the two 64-query halves one leading step apart
        auto wait_all = [&](uint32_t b, uint32_t parity) { return mbar_wait_warp(b, parity, abort_flag, p.status); };
        bool ok = true;
        uint32_t g = 0, nitem = 0, buf = 0, slot = 0, round = 0;
        for (int item = first_item; item < last_item && ok; ++item, ++nitem, next_slot(slot, round)) {
            if (!items_ready(nitem)) { ok = false; break; }
            const int tiles = (items->at(nitem).patches + 1) >> 1;
            if (warp == 1) {
                // ---- S^T, dP^T of unit u as soon as dV and dK of unit u - 3 have consumed P^T, dS^T, which lie in the same columns
                if (!wait_all(bar(kKVFull + slot), round)) { ok = false; break; }
                // (columns 8 .. 15 of the ones: the same rows again, against zeros)
                const uint64_t ones_s = smem_desc(base + kOffOnes, 16, 16, kSwizzleNone), ones_dp = smem_desc(base + kOffOnes + kOnesBytes, 16, 16, kSwizzleNone);
                const uint64_t k = smem_desc_at(kDesc64, k_slot(slot)), v = smem_desc_at(kDesc64, k_slot(slot) + kContentBytes);
                for (int t = 0; t < tiles && ok; ++t, ++g) {
                    const uint32_t st = g % kQStages;
                    if (!wait_all(bar(kQFull + st), (g / kQStages) & 1)) { ok = false; break; }
#pragma unroll 1                     // (the kernel's loops together just fit the instruction cache)
                    for (uint32_t h = 0; h < 2; ++h) {
                        const uint32_t u = 2 * g + h;
                        if (!wait_all(on_unit(kPFree, u - kBuffers), unit_parity(u - kBuffers))) { ok = false; break; }
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t ring = base + kOffRing + st * kRingBytes + h * kPatchContent;   // rows of patch h
                            const uint64_t q = smem_desc_at(kDesc64, ring + kRingQ), go = smem_desc_at(kDesc64, ring + kRingDO);
                            const uint32_t d_s = tmem + kStep * buf;
                            mma_ss(d_s, k, q, kIdescSS, 0u);
                            mma_ss(d_s, k + 2, q + 2, kIdescSS, 1u);     // + 32 bytes: second K16 step
                            // - lse sqrt(d) of the query, and - D: three bf16 parts of each against ones
                            const uint32_t rows = st * kRingBytes + kOffRing + kRingLD + h * kLdPatch;
                            const uint64_t parts = smem_desc(base + rows, kOffZero - rows, 128, kSwizzleNone);
                            mma_ss(d_s, ones_s, parts, kIdescSS, 1u);
                            mma_ss(d_s + kColDP, v, go, kIdescSS, 0u);
                            mma_ss(d_s + kColDP, v + 2, go + 2, kIdescSS, 1u);
                            mma_ss(d_s + kColDP, ones_dp, parts, kIdescSS, 1u);
                            mma_commit(on_unit(kSFull, u));
                        }
                        __syncwarp();
                        buf = buffer_after(buf, 1);
                    }
                }
            } else if (warp == 2) {
                // ---- dV_J += P^T dO_u and dK_J += dS^T Q_u (A from tensor memory, 16 queries per step)
                for (int t = 0; t < tiles && ok; ++t, ++g) {
                    const uint32_t st = g % kQStages;
#pragma unroll 1                     // (the kernel's loops together just fit the instruction cache)
                    for (uint32_t h = 0; h < 2; ++h) {
                        const uint32_t u = 2 * g + h;
                        const bool first = t == 0 && h == 0, last = t == tiles - 1 && h == 1;
                        if (!wait_all(on_unit(kPReady, u), unit_parity(u)) ||
                            (first && nitem > 0 && !wait_all(bar(kAccFree), (nitem - 1) & 1))) { ok = false; break; }
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t ring = base + kOffRing + st * kRingBytes + h * kPatchContent;
                            const uint64_t go = smem_desc_at(kDesc64, ring + kRingDO), q = smem_desc_at(kDesc64, ring + kRingQ);
                            const uint32_t a_p = tmem + kStep * buf;          // 16 queries a step: the first 16 of every 32 columns
#pragma unroll
                            for (int kk = 0; kk < kTile / 32; ++kk)
                                mma_ts(tmem + kColDV, a_p + 32 * (kk >> 1) + 8 * (kk & 1), go + 64 * kk, kIdescT, (kk || !first) ? 1u : 0u);
#pragma unroll
                            for (int kk = 0; kk < kTile / 32; ++kk)
                                mma_ts(tmem + kColDK, a_p + kColDP + 32 * (kk >> 1) + 8 * (kk & 1), q + 64 * kk, kIdescT, (kk || !first) ? 1u : 0u);
                            mma_commit(on_unit(kPFree, u));
                            // the tile's query-side rows may go: S^T, dP^T of both halves finished before P^T existed
                            if (h == 1) mma_commit(bar(kQEmpty + st));
                            if (last) mma_commit(bar(kAccFull));
                        }
                        __syncwarp();
                        buf = buffer_after(buf, 1);
                    }
                }
            } else {
                // ---- dQ_I = dS K_J once both halves of dS are in shared memory (16 keys per step)
                for (int t = 0; t < tiles; ++t, ++g) {
                    if (!wait_all(on_unit(kPReady, 2 * g), unit_parity(2 * g)) || !wait_all(on_unit(kPReady, 2 * g + 1), unit_parity(2 * g)) ||
                        (g > 0 && !wait_all(bar(kDQFree), (g - 1) & 1))) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t k = smem_desc_at(kDesc64, k_slot(slot));
                        const uint64_t ds = smem_desc_at(kDescDS, base + kOffDS + (g & 1) * 2 * kDSHalf);
#pragma unroll
                        for (int kk = 0; kk < kTile / 16; ++kk)
                            mma_ss(tmem + kColDQ, ds + 128 * kk, k + 64 * kk, kIdescQ, kk ? 1u : 0u);
                        mma_commit(bar(kDSFree + (g & 1)));
                        mma_commit(bar(kDQFull));
                        // K_J and V_J may go once the item's last dQ is done (S^T, dP^T finished before it)
                        if (t == tiles - 1) mma_commit(bar(kKVEmpty + slot));
                    }
                    __syncwarp();
                }
            }
        }
        // everything issued by this warp must have finished before TMEM is released
        if (elect_one()) mma_commit(bar(kDrain + warp - 1));
        __syncwarp();
        mbar_wait(bar(kDrain + warp - 1), 0, abort_flag + 1, p.status);
    } else if (warp < 20) {
        // ===== P^T and dS^T: group h = warps 4 + 8h .. 11 + 8h takes half-tile (I, h), a warp 32 key rows (4 x 8 tokens) and 32 queries (4 x 8)
        const int h = (warp - 4) >> 3;
        const int cg = ((warp - 4) >> 2) & 1;                // queries 32 cg .. 32 cg + 31 of the half-tile
        const int quarter = warp & 3;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
        const uint32_t table_addr = base + kOffTable;
        uint32_t g = 0, buf = h, ntable = 0;
        int table_head = -1;
        bool ok = true;
        for (int item = first_item; item < last_item && ok; ++item) {
            const uint32_t nitem = (uint32_t)(item - first_item);
            if (!items_ready(nitem)) { ok = false; break; }
            const LiveItem c = items->at(nitem);
            if (c.h != table_head) {
                // the table of head h: when all arithmetic warps are through with the last one's
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kTabDone));
                if (!mbar_wait_warp(bar(kTabDone), ntable & 1, abort_flag, p.status)) { ok = false; break; }
                gather_bias(p.source, c.h, side * side, -INFINITY, reinterpret_cast<float*>(base_ptr + kOffTable), threadIdx.x - 128, kArithmeticThreads);
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kTabReady));
                if (!mbar_wait_warp(bar(kTabReady), ntable & 1, abort_flag, p.status)) { ok = false; break; }
                ++ntable;
                table_head = c.h;
            }
            const int key_patch = 2 * c.tp + (quarter >> 1);
            const bool key_exists = key_patch < c.patches;
            const int key_at = lists->origin[list_of(c) + key_patch], ky = key_at >> 8, kx = key_at & 255;
            int Y0 = 0, X0 = 0;
            if (kCut) patch_place(geom, lists, c, key_patch, Y0, X0);
            const int xk = lane >> 2, key_row0 = 4 * (quarter & 1);
            // keys of the patch beyond the map's edge get probability 0: a thread's whole column, or the rows from `rows_there` on
            const bool column_there = !kCut || X0 + xk < p.W;
            const int rows_there = p.H - Y0 - key_row0;          // of the thread's four
            // (a key that is none, in a whole patch or a column beyond the edge, finds the same two words for every query)
            const bool there = key_exists && column_there;
            const uint32_t pitch = there ? 4u * side : 0u, moves = there ? 0xffffu : 0u;
            const uint32_t k_addr = there ? table_addr + (ky + key_row0 - 4 * cg + p.M - 1) * pitch + 4 * (kx + xk + p.M - 1 - 2 * (lane & 3)) : base + kOffMasked + 4;
            const uint16_t* const entries = lists->entry + list_of(c) + h;
            const int tiles = (c.patches + 1) >> 1;
            for (int I = 0; I < tiles; ++I, ++g) {
                const uint32_t t_s = tmem + lane_base + 32 * cg + kStep * buf, t_dp = t_s + kColDP;
                buf = buffer_after(buf, 2);
                const uint32_t b_addr = k_addr - (entries[2 * I] & moves);
                // biases of key row a against query row b of the warp's rows, a - b = k (the queries' columns go up, so the offsets go down)
                auto bias = [&](int k) { return make_float2(lds_f32(b_addr + k * (int)pitch), lds_f32(b_addr + k * (int)pitch - 4)); };
                float2 bb[3] = {bias(1), bias(2), bias(3)};
                // warp-uniform outcome: the TMEM accesses below are warp-collective
                if (!mbar_wait_warp(on_unit(kSFull, 2 * g + h), unit_parity(2 * g), abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
                // Four pieces of 16 keys x 16 queries, read as 16-lane fragments: piece (o, G) has lanes 16 o .. and queries 16 G .., a thread of it 2 key rows of
                // 2 x 2 queries.  For each G first o = 1, then o = 0: their differences of rows a - b are 1 2 3 and -1 0 1, less 2 G, so that the
                // biases of the second piece are those of the next G's first one as well.
                // dS tile: row = key, 128-byte line = the unit's 64 queries, 16-byte chunks swizzled by the row
                const uint32_t ds_at = base + kOffDS + ((g & 1) * 2 + h) * kDSHalf + (quarter * 32 + 8 * ((lane >> 3) & 1) + (lane & 7)) * 128 + (((cg * 4 + (lane >> 4)) ^ (lane & 7)) << 4);
                auto load = [&](int o, int G, uint32_t (&s)[8], uint32_t (&dp)[8]) {
                    const uint32_t at = ((uint32_t)(16 * o) << 16) + 16 * G;
                    tmem_ld_16x256b_x2(t_s + at, s);
                    tmem_ld_16x256b_x2(t_dp + at, dp);
                };
                // bb[i]: a - b = that of equal fragment rows (gq == rr) + i - 1
                auto work = [&](int o, const uint32_t (&s)[8], const uint32_t (&dp)[8], const float2 (&bb)[3], uint32_t (&pp)[4], uint32_t (&dd)[4]) {
#pragma unroll
                    for (int gq = 0; gq < 2; ++gq)
#pragma unroll
                        for (int rr = 0; rr < 2; ++rr) {                  // key rows 2 o + rr of the warp's, query rows 2 G + gq
                            const int i = 4 * gq + 2 * rr;
                            const float2 x = __ffma2_rn(make_float2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), scale2, bb[1 + rr - gq]);
                            // (a probability is at most 1, however little of its digits a large lse has left; NaN stays)
                            float2 e = make_float2(ex2_approx(min_nan(x.x, 0.f)), ex2_approx(min_nan(x.y, 0.f)));
                            if (kCut && 2 * o + rr >= rows_there) e = make_float2(0.f, 0.f);
                            const float2 d = __fmul2_rn(e, make_float2(__uint_as_float(dp[i]), __uint_as_float(dp[i + 1])));
                            pp[2 * gq + rr] = pack_bf16x2(e.x, e.y);
                            dd[2 * gq + rr] = pack_bf16x2(d.x, d.y);
                        }
                };
                auto store = [&](int o, int G, const uint32_t (&pp)[4], const uint32_t (&dd)[4]) {
                    const uint32_t at = ((uint32_t)(16 * o) << 16) + 8 * G;
                    tmem_st_16x128b_x2(t_s + at, pp);
                    tmem_st_16x128b_x2(t_dp + at, dd);
                    stmatrix_x4((ds_at ^ (32 * G)) + 16 * o * 128, dd[0], dd[1], dd[2], dd[3]);
                };
                // The tile before the previous one is still read in this dS buffer.  (A barrier that has completed no phase answers yes to
                // parity 1, which the first tiles ask for.)
                const uint32_t b_ds = bar(kDSFree + (g & 1)), ds_parity = ((g >> 1) - 1) & 1;
                const bool ds_free = mbar_try_wait(b_ds, ds_parity);
                uint32_t pp[4], dd[4], s0[8], dp0[8], s1[8], dp1[8];
                load(1, 0, s1, dp1);
                load(0, 0, s0, dp0);
                // A piece is stored while the next but one is on its way, over scores that this warp has read.
#pragma unroll 1
                for (int G = 0; G < 2; ++G) {
                    tmem_wait_ld();
                    work(1, s1, dp1, bb, pp, dd);
                    if (G == 0) {
                        if (!__all_sync(0xffffffffu, ds_free) && !mbar_wait_warp(b_ds, ds_parity, abort_flag, p.status)) { ok = false; break; }
                        load(1, 1, s1, dp1);
                    }
                    store(1, G, pp, dd);
                    bb[2] = bb[0]; bb[0] = bias(-1 - 2 * G); bb[1] = bias(-2 * G);
                    work(0, s0, dp0, bb, pp, dd);
                    if (G == 0) load(0, 1, s0, dp0);
                    store(0, G, pp, dd);
                }
                if (!ok) break;
                tmem_wait_st();
                tc_fence_before();
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(on_unit(kPReady, 2 * g + h));
            }
        }
    } else if (warp < 24) {
        // ================================ drains: dQ after every tile, dV / dK after every item
        const int quarter = warp & 3;
        const int row = quarter * 32 + lane;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        auto drain_item = [&](const LiveItem& c, uint32_t nitem, uint32_t v_slot) -> bool {
            // rows leave by TMA, a warp's 32 (half a patch) at a time; rows beyond the map's edge are dropped by it
            int Y0, X0;
            const int sp = 2 * c.tp + (quarter >> 1);
            patch_place(geom, lists, c, sp, Y0, X0);
            const int Y = Y0 + 4 * (quarter & 1);
            if (!mbar_wait_warp(bar(kAccFull), nitem & 1, abort_flag, p.status)) return false;
            tc_fence_after();
            const int sw = (row >> 1) & 3;                    // SWIZZLE_64B
#pragma unroll
            for (int which = 0; which < 2; ++which) {         // dV through V's slot, dK through a tile of its own
                uint8_t* const stage = base_ptr + (which == 0 ? v_slot : kOffDK) + row * 64;
                const float f = which == 0 ? 1.f : p.inv_sqrt_d;
                uint32_t a[32];
                tmem_ld32(tmem + lane_base + (which == 0 ? kColDV : kColDK), a);
                tmem_wait_ld();
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(__uint_as_float(a[8 * q + 2 * e]) * f, __uint_as_float(a[8 * q + 2 * e + 1]) * f);
                    *reinterpret_cast<uint4*>(stage + ((q ^ sw) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            tc_fence_before();
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(bar(kAccFree));
                if (sp < c.patches && Y < p.H) {
                    tma_store_5d(&tm_dv, base + v_slot + quarter * (kPatchContent / 2), 0, c.h, X0, Y, c.b);
                    tma_store_5d(&tm_dk, base + kOffDK + quarter * (kPatchContent / 2), 0, c.h, X0, Y, c.b);
                    bulk_commit_group();
                }
            }
            return true;
        };
        uint32_t g = 0, nitem = 0, slot = 0, round = 0;
        bool ok = true;
        for (int item = first_item; item < last_item && ok; ++item, ++nitem, next_slot(slot, round)) {
            if (!items_ready(nitem)) { ok = false; break; }
            const LiveItem c = items->at(nitem);
            const int tiles = (c.patches + 1) >> 1;
            float* const acc = p.dq_acc + pair_of(p, c) * p.columns * p.n;
            for (int I = 0; I < tiles && ok; ++I, ++g) {
                // (dV and dK before the item's last dQ: those of the next item wait for the accumulators)
                if (I == tiles - 1) ok = drain_item(c, nitem, p.slots_at + slot * kSlotBytes + kContentBytes);
                if (!ok || !mbar_wait_warp(bar(kDQFull), g & 1, abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
                const int sp = 2 * I + (quarter >> 1), at = lists->origin[list_of(c) + sp];
                float* dst = acc + 4 * (64 * (size_t)((at >> 11) * (p.M >> 3) + ((at & 255) >> 3)) + (row & 63));
#pragma unroll
                for (int part = 0; part < kD / 16; ++part) {
                    uint32_t a[16];
                    tmem_ld16(tmem + lane_base + kColDQ + 16 * part, a);
                    tmem_wait_ld();
                    if (part + 1 == kD / 16) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(kDQFree));
                    }
                    if (sp < c.patches) {
#pragma unroll
                        for (int col = 0; col < 16; col += 4) {
                            if (16 * part + col >= p.columns) break;          // (a head narrower than 32 channels)
                            // The adds of a tile in one burst fill the queue that all warps' loads, stores and fences go through: a pause after each one
                            red_add_f32x4(dst, a + col);
                            dst += 4 * (size_t)p.n;
                            __nanosleep(20);
                        }
                    }
                }
            }
            if (ok) {
                // V's slot, when its dV rows have been read
                if (lane == 0) {
                    bulk_wait_group_read<0>();                // (this thread's own stores)
                    mbar_arrive(bar(kKVEmpty + slot));
                }
                __syncwarp();
            }
        }
        if (lane == 0) bulk_wait_group<0>();
        __syncwarp();
    } else {
        // ================================ gradient of the bias: warp 24 + 2 h + sub sums dS of key patch `sub` of the item and the queries of half h
        // One MMA of 16 x 8 x 16 takes, of one row of the keys' patch (a) and the 8 rows of the queries', two key columns x: its A has the difference of
        // rows t = (a - query row) mod 8 as its rows - the lines of an ldmatrix may come from anywhere - and (x, query column) as its columns; where
        // a - query row is t the row goes to the upper half of A, where it is t - 8 to the lower.  B names for every (x, query column) the
        // difference of columns.  So the 64 MMAs of 8 key rows x 4 pairs of columns x 2 halves of the 15 differences leave the sums of dS at
        // the 15 x 15 offsets of the two patches in 8 registers of the warp, and the loop is short: a first version with one product per block
        // and the diagonals by shuffles was a kilobyte of instructions too long for the instruction cache (1160 us; without any of it 798).
        const int h = (warp >> 1) & 1, sub = warp & 1;
        // Of an ldmatrix this lane names line t of matrix m: A's quarter of the upper (m even) or lower rows and of the first or second key column x.
        const int t = lane & 7, lower = (lane >> 3) & 1, second = lane >> 4;
        const int arow = lane >> 2, c2 = 2 * (lane & 3);
        // B of the pair of columns x, x + 1 and the differences 8 n - 8 .. 8 n - 1 of x - query column: rows (x, 0..7), (x + 1, 0..7); this lane has column
        // lane / 4 (difference 8 n - 8 + lane / 4) of the rows c2, c2 + 1
        uint32_t eye[4][2][2];
#pragma unroll
        for (int pr = 0; pr < 4; ++pr)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const int d = 8 * n - 8 + arow, x = 2 * pr + o;
                    eye[pr][n][o] = (x - c2 == d ? 0x3F80u : 0u) | (x - c2 - 1 == d ? 0x3F800000u : 0u);
                }
        const int across = 2 * (p.M >> 3) - 1;
        uint32_t g = 0;
        bool ok = true;
        for (int item = first_item; item < last_item && ok; ++item) {
            const uint32_t nitem = (uint32_t)(item - first_item);
            if (!items_ready(nitem)) { ok = false; break; }
            const LiveItem c = items->at(nitem);
            const int tiles = (c.patches + 1) >> 1;
            const uint16_t* const list = lists->origin + list_of(c);
            const int key_at = list[2 * c.tp + sub] + (0x100 + 1) * (p.M - 8);
            const bool key_exists = 2 * c.tp + sub < c.patches;
            float* const blocks = p.blocks + (size_t)c.h * across * across * 256 + arow * 16 + c2;
            for (int I = 0; I < tiles; ++I, ++g) {
                if (!mbar_wait_warp(on_unit(kPReady, 2 * g + h), unit_parity(2 * g), abort_flag, p.status)) { ok = false; break; }
                // dS of key (a, x): line 8 a + x of the patch, 128 bytes; the 8 queries of row b: chunk b, swizzled by the line
                uint32_t line = base + kOffDS + ((g & 1) * 2 + h) * kDSHalf + sub * 64 * 128 + second * 128;
                const uint32_t zero = base + kOffZero + second * 128;
                float sum[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};      // differences of columns -8 .. -1 and 0 .. 7; [0], [1]: rows t, [2], [3]: rows t - 8
#pragma unroll 4
                for (int a = 0; a < 8; ++a, line += 1024) {
                    const uint32_t addr = ((a < t) == (lower != 0) ? line : zero) + ((((a - t) & 7) ^ second) << 4);
                    uint32_t r[4][4];
#pragma unroll
                    for (int pr = 0; pr < 4; ++pr) ldmatrix_x4((addr ^ (pr << 5)) + 256 * pr, r[pr]);
#pragma unroll
                    for (int pr = 0; pr < 4; ++pr)
#pragma unroll
                        for (int n = 0; n < 2; ++n) mma_16816(sum[n], r[pr][0], r[pr][1], r[pr][2], r[pr][3], eye[pr][n][0], eye[pr][n][1]);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kDSFree + (g & 1)));
                if (!key_exists || 2 * I + h >= c.patches) continue;
                const int at = key_at - list[2 * I + h];              // (rows << 8) + columns, both 8 (patches' difference + M / 8 - 1) >= 0
                float* const to = blocks + ((at >> 11) * across + ((at & 255) >> 3)) * 256;
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    red_add_f32x2(to + 128 + 8 * n, sum[n][0], sum[n][1]);
                    red_add_f32x2(to + 8 * n, sum[n][2], sum[n][3]);
                }
            }
        }
    }
    // ================================================================================ common tail
    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

// ------------------------------------------------------------------ preparation and finishing
struct AuxParams {
    const __nv_bfloat16* out;
    const __nv_bfloat16* dout;
    const float* lse;
    uint4* ld;
    float* dq_acc;
    double* sums;                // BiasGrad, cleared here
    size_t sum_words;
    __nv_bfloat16* dq;
    CheckpointRows saved[4];     // kSaved: q, k, v, out
    int H, W, heads, M, s, n, patches, d, Hp, Wp;      // patches: of all pairs
    int columns;                 // of the dQ accumulators: d, or 32 where those from 16 on have dS times what the rounding of k left
    int wide;                    // kSaved: 1: q and k are restored to rows of 32 columns (restore_wide)
    FastDiv by_patches, by_heads, by_nwx, by_nwy, by_row;
    float inv_sqrt_d, sqrt_d;
};

// x as the sum of three bf16: exact to 2^-24
__device__ __forceinline__ void three_parts(float x, uint32_t (&part)[3])
{
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const __nv_bfloat16 b = __float2bfloat16_rn(x);
        part[i] = __bfloat16_as_ushort(b);
        x -= __bfloat162float(b);
    }
}

// Patch `index` of all (pair, patch of the window in rows), token `at` of its 64: false for a position beyond the map, where no token is.  The pair is
// (batch item, window row, window column, head), heads innermost.  (With plain divisions the preparation of 16 x 96 x 96 tokens, 6 heads of 32, took
// 45 us instead of 39.)
__device__ __forceinline__ bool decode_token(const AuxParams& p, int index, int at, int& pair, int& patch, size_t& tok, size_t& scalar)
{
    int rest, h, wx, wy, b, row, col;
    p.by_patches.divmod(index, pair, patch);
    p.by_heads.divmod(pair, rest, h);
    p.by_nwx.divmod(rest, rest, wx);
    p.by_nwy.divmod(rest, b, wy);
    p.by_row.divmod(patch, row, col);
    int Y = wy * p.M + 8 * row + p.s, X = wx * p.M + 8 * col + p.s;
    Y = (Y >= p.Hp ? Y - p.Hp : Y) + (at >> 3);
    X = (X >= p.Wp ? X - p.Wp : X) + (at & 7);
    tok = (((size_t)b * p.H + Y) * p.W + X) * p.heads + h;
    scalar = (((size_t)b * p.heads + h) * p.H + Y) * p.W + X;
    return Y < p.H && X < p.W;
}

// kLanes (2 for heads of up to 16 channels, else 4) per (pair, token in window order), 8 channels each: D = dO . O and lse in the layout the main kernel streams; the dQ accumulators and
// the sums of the bias gradient are cleared as flat arrays.  A query that is no token, or whose row has no key (lse = -inf), has a score far below
// all others: probability 0.
// kSaved: q, k, v and out are checkpoints; the first three are restored to where the main kernel reads them.
template <bool kSaved, int kLanes>
__global__ void __launch_bounds__(64 * kLanes) rib_bias_bwd_prepare_kernel(const AuxParams p)
{
    const size_t total = (size_t)p.patches * 64;
    const size_t thread = (size_t)blockIdx.x * blockDim.x + threadIdx.x, t = thread / kLanes;        // (a block has a patch)
    const int part = threadIdx.x % kLanes;
    const size_t nthreads = (size_t)gridDim.x * blockDim.x;
    for (size_t e = thread; e < p.sum_words; e += nthreads) p.sums[e] = 0.0;
    constexpr uint32_t kNone = 0xF149u;                    // -1e30 in bf16
    if (thread < 64) p.ld[total + thread] = make_uint4(kNone, 0u, 0u, 0u);       // the patch of no queries
    int pair, patch;
    size_t tok, scalar;
    const bool real = decode_token(p, blockIdx.x, threadIdx.x / kLanes, pair, patch, tok, scalar);
    uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x;
    float lse = -INFINITY;
    const bool wide = kSaved && kLanes == 2 && p.wide;
    if (wide && real) {
        // (logits of 8 channels; those of 16 lose less, and stay those of the call from the restored tensors)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (p.d == 8) restore_wide<true>(p.saved, tok, 8, part + 2 * half);
            else restore_wide<false>(p.saved, tok, 16, part + 2 * half);
        }
    }
    if (real && 8 * part < p.d) {
        x = __ldg(reinterpret_cast<const uint4*>(p.dout + tok * p.d) + part);
        if (kSaved) {
            uint2 c[4];
            float scale[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[i] = __ldg(reinterpret_cast<const uint2*>(p.saved[i].codes + tok * p.d) + part);
                scale[i] = __ldg(p.saved[i].scales + tok);
            }
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i == 2 || !wide) reinterpret_cast<uint4*>(p.saved[i].x + tok * p.d)[part] = restored_chunk(c[i], scale[i]);
            y = restored_chunk(c[3], scale[3]);
        } else {
            y = __ldg(reinterpret_cast<const uint4*>(p.out + tok * p.d) + part);
        }
        if (part == 0) lse = p.lse[scalar];
    }
    float4* z4 = reinterpret_cast<float4*>(p.dq_acc);      // pairs * columns * n floats
#pragma unroll
    for (int k = 0; k < (kSaved && kLanes == 2 ? 4 : 2); ++k)
        if (k * kLanes * total + thread < total * (p.columns / 4)) z4[k * kLanes * total + thread] = make_float4(0.f, 0.f, 0.f, 0.f);
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
    float acc = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        acc = fmaf(__uint_as_float(xs[k] << 16), __uint_as_float(ys[k] << 16), acc);
        acc = fmaf(__uint_as_float(xs[k] & 0xffff0000u), __uint_as_float(ys[k] & 0xffff0000u), acc);
    }
    acc += __shfl_xor_sync(0xffffffffu, acc, 1);
    if (kLanes > 2) acc += __shfl_xor_sync(0xffffffffu, acc, 2);
    if (part == 0) {
        uint32_t l[3], d[3];
        three_parts(-lse * p.sqrt_d, l);
        three_parts(-acc, d);
        p.ld[t] = lse == -INFINITY ? make_uint4(kNone, 0u, 0u, 0u) : make_uint4(l[0] | l[1] << 16, l[2] | d[0] << 16, d[1] | d[2] << 16, 0u);
    }
}

// dq = bf16(accumulator / sqrt(d)): a thread per token and half row (16 columns: four 16-byte reads, 512 bytes per warp and read).
// Blocks from dq_blocks on add up the gradient of the bias.
__global__ void __launch_bounds__(256) rib_bias_bwd_finish_kernel(const AuxParams p, const BiasScatter scatter, unsigned dq_blocks)
{
    cudaGridDependencySynchronize();
    if (blockIdx.x >= dq_blocks) { bias_scatter(scatter, (size_t)(blockIdx.x - dq_blocks) * blockDim.x + threadIdx.x); return; }
    const int index = 2 * blockIdx.x + (threadIdx.x >> 7), at = ((threadIdx.x >> 6) & 1) * 32 + (threadIdx.x & 31);        // 32 tokens x 2 halves per two warps
    const int half = (threadIdx.x >> 5) & 1;
    const int channels = min(16, p.d - 16 * half);
    if (index >= p.patches || channels <= 0) return;
    int pair, patch;
    size_t tok, scalar;
    if (!decode_token(p, index, at, pair, patch, tok, scalar)) return;
    const float4* src = reinterpret_cast<const float4*>(p.dq_acc + (size_t)pair * p.columns * p.n) + (size_t)(4 * half) * p.n + 64 * patch + at;
    uint32_t v[8];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float4 f = 4 * q < channels ? src[(size_t)q * p.n] : make_float4(0.f, 0.f, 0.f, 0.f);
        if (p.columns != p.d) {          // (16 channels)
            const float4 rest = src[(size_t)(4 + q) * p.n];
            f.x += rest.x; f.y += rest.y; f.z += rest.z; f.w += rest.w;
        }
        v[2 * q] = pack_bf16x2(f.x * p.inv_sqrt_d, f.y * p.inv_sqrt_d);
        v[2 * q + 1] = pack_bf16x2(f.z * p.inv_sqrt_d, f.w * p.inv_sqrt_d);
    }
    uint4* dst = reinterpret_cast<uint4*>(p.dq + tok * p.d) + 2 * half;
    dst[0] = make_uint4(v[0], v[1], v[2], v[3]);
    if (channels > 8) dst[1] = make_uint4(v[4], v[5], v[6], v[7]);
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t ld_bytes(long long pairs, int n) { return align256(((size_t)pairs * n + 64) * sizeof(uint4)); }

}  // namespace

bool sm100_bias_bwd_supported(const Problem& p)
{
    BiasItems g;
    return bias_shape_supported(p) && (long long)p.pairs * (p.n / 64) <= 0x7fffffffLL && make_bias_items(p, 2, &g);
}

size_t sm100_bias_bwd_workspace_bytes(long long pairs, int n) { return ld_bytes(pairs, n) + align256((size_t)pairs * kD * n * sizeof(float)); }

cudaError_t sm100_bias_bwd(const Problem& p, const BiasGrad& grad, cudaStream_t stream)
{
    if (!encode_fn()) return cudaErrorNotSupported;
    uint8_t* ws = static_cast<uint8_t*>(p.workspace);
    uint4* ld = reinterpret_cast<uint4*>(ws);
    float* dq_acc = reinterpret_cast<float*>(ws + ld_bytes(p.pairs, p.n));
    CUtensorMap tm_q, tm_k, tm_v, tm_do, tm_dk, tm_dv;
    if (!encode_qk_map(&tm_q, p.q, p) || !encode_qk_map(&tm_k, p.k, p) || !encode_image_map(&tm_v, p.v, p) || !encode_image_map(&tm_do, p.dout, p) ||
        !encode_image_map(&tm_dk, p.dk, p, 4) || !encode_image_map(&tm_dv, p.dv, p, 4))
        return cudaErrorInvalidValue;
    static KernelSetup setup[2];
    const bool cut = p.H % 8 != 0 || p.W % 8 != 0;
    const auto kernel = cut ? rib_bias_bwd_kernel<true> : rib_bias_bwd_kernel<false>;
    int sm_count = 0;
    if (cudaError_t e = setup[cut].prepare(kernel, most_shared(), &sm_count)) return e;
    Params bp{};
    if (!make_bias_items(p, 2, &bp.g)) return cudaErrorInvalidValue;
    bp.columns = p.qk_width && p.d == 16 ? 32 : p.d;
    AuxParams ap{};
    ap.out = p.out; ap.dout = p.dout; ap.lse = p.lse_in; ap.ld = ld; ap.dq_acc = dq_acc; ap.dq = p.dq;
    ap.sums = grad.offsets; ap.sum_words = grad.bytes / sizeof(double);
    ap.H = p.H; ap.W = p.W; ap.heads = p.heads; ap.M = p.M; ap.s = p.s; ap.n = p.n; ap.d = p.d; ap.columns = bp.columns;
    ap.wide = p.qk_width != 0;
    ap.patches = (int)((long long)p.pairs * (p.n / 64));
    ap.by_patches = make_fast_div(p.n / 64); ap.by_heads = make_fast_div(p.heads); ap.by_nwx = make_fast_div(p.nWx); ap.by_nwy = make_fast_div(p.nWy); ap.by_row = make_fast_div(p.M / 8);
    ap.Hp = p.Hp; ap.Wp = p.Wp;
    if (p.saved) for (int i = 0; i < 4; ++i) ap.saved[i] = p.saved[i];
    ap.sqrt_d = sqrtf((float)p.d);
    ap.inv_sqrt_d = 1.f / ap.sqrt_d;
    const size_t tokens = (size_t)p.pairs * p.n;
    const auto prepare = p.d <= 16 ? (p.saved ? rib_bias_bwd_prepare_kernel<true, 2> : rib_bias_bwd_prepare_kernel<false, 2>)
                                   : (p.saved ? rib_bias_bwd_prepare_kernel<true, 4> : rib_bias_bwd_prepare_kernel<false, 4>);
    { ProfileScope scope(RIB_KERNEL_BIAS_BWD_PREPARE, stream); prepare<<<ap.patches, p.d <= 16 ? 128 : 256, 0, stream>>>(ap); }
    if (cudaError_t e = cudaGetLastError()) return e;
    bp.ld = ld; bp.dq_acc = dq_acc; bp.blocks = grad.blocks; bp.status = p.status;
    bp.no_queries = (long long)tokens;
    bp.H = p.H; bp.W = p.W; bp.heads = p.heads; bp.M = p.M; bp.s = p.s; bp.n = p.n; bp.nWy = p.nWy; bp.nWx = p.nWx; bp.Hp = p.Hp; bp.Wp = p.Wp;
    bp.items = bp.g.per_head * p.heads;
    bp.slots = slots_of(p.M);
    bp.slots_at = slots_offset(p.M);
    bp.scale_log2 = kLog2e / sqrtf((float)p.d);
    bp.inv_sqrt_d = ap.inv_sqrt_d;
    bp.source = bias_source(p);
    const int grid = bp.items < sm_count ? bp.items : sm_count;
    // (each of the kernels behind the first may start while the one before it ends: its set-up, or at least its launch, is then over)
    {
        ProfileScope scope(RIB_KERNEL_BIAS_BWD, stream);
        if (cudaError_t e = launch_overtaking(kernel, grid, kThreads, smem_bytes(p.M), stream, tm_q, tm_k, tm_v, tm_do, tm_dk, tm_dv, bp)) return e;
    }
    const BiasScatter scatter = bias_scatter_args(p, grad, true);
    const unsigned dq_blocks = (unsigned)((tokens + 127) / 128), all = dq_blocks + (unsigned)(((size_t)p.heads * scatter.side * scatter.side + 255) / 256);
    {
        ProfileScope scope(RIB_KERNEL_BIAS_BWD_FINISH, stream);
        if (cudaError_t e = launch_overtaking(rib_bias_bwd_finish_kernel, (int)all, 256, 0, stream, ap, scatter, dq_blocks)) return e;
    }
    return bias_grad_convert(p, grad, stream);
}

}  // namespace rib
