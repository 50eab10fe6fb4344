// Shared between the tcgen05 kernels for a bias by buckets: work items with the heads outermost, and the table of a head in shared memory.
//
// The bias of a pair depends on the offset key - query only, so a CTA keeps ONE head's biases by offset, (2M-1)^2 fp32 values already times
// log2(e), in shared memory, and walks its items head by head: a new table is gathered through the bucket map once or twice in
// a launch.  A thread that holds query rows y .. y + 3 of one column x and keys (y', x'), (y', x' + 1) of the 8 x 8 patches of both finds the
// biases of 4 x 8 x 2 scores in 11 pairs of the table (y' - y takes 11 values): a third of a load per score, and the 32 lanes of a load
// (8 columns x, 4 pairs x') touch 15 neighbouring words.
#pragma once
#include "rib_sm100_common.cuh"

namespace rib {
namespace sm100 {

constexpr int kBiasMaxWindow = 64;                     // (127^2 fp32 = 64.5 KB beside the tiles)
constexpr float kLog2e = 1.4426950408889634f;
// What the forward's table holds for keys that are not attended to: finite, so that the polynomial form of the exponential takes it, and further
// below 0 than a score in log2 units can lie above it (a finite fp32 product times log2(e) / sqrt(d), at most 3.41e38 x 0.511 = 1.74e38 for d >= 8).  The sum
// is minus infinity for the lowest scores only, which the exact form takes.  The backward's table holds minus infinity: there is no polynomial there.
constexpr float kTableMasked = -1.8e38f;

struct BiasItems {
    LiveWindows live;              // of one head
    int per_head;                  // items of a head
    int weight[9];                 // of an item of each kind: key blocks (forward) or query tiles (backward) that it walks
    long long work[10];            // prefix sums of the weights over the kinds; work[9]: one head
    FastDiv by_head;
};

__device__ __forceinline__ LiveItem decode_bias_item(const BiasItems& g, int item)
{
    int h, rest;
    g.by_head.divmod(item, h, rest);
    LiveItem c = decode_live_item(g.live, rest);
    c.h = h;
    return c;
}

// The items that the roles of a CTA walk, decoded once by the producer's warp, eight at a time, instead of by every warp (a chain of divisions and of
// loads from the parameters by kind; in windows of 16 an item is some 3 us of work: 4 x 96 x 96 tokens, 12 heads, d = 16, backward
// 116 -> 105 us).  `n` counts the CTA's items; every 8th one a
// role waits for the barrier whose phases are the eights.  Nothing says that an eight may be overwritten, and nothing has to: the producer
// writes eight c + 2 when it has begun to load item 8 c + 15, and K, V (backward) or Q (forward) of that item went where those of item
// 8 c + 11 or 8 c + 13 had been, by when no role is more than six items behind.
struct ItemRing {
    static constexpr uint32_t kEight = 8;
    LiveItem items[2 * kEight];
    __device__ __forceinline__ static bool begins(uint32_t n) { return n % kEight == 0; }
    __device__ __forceinline__ static uint32_t parity(uint32_t n) { return (n / kEight) & 1; }
    __device__ __forceinline__ LiveItem& at(uint32_t n) { return items[n % (2 * kEight)]; }
};

// The patches of every kind of window, in the order of its list, in shared memory: where they begin in the window (y << 8 | x), and how far into a
// table by offset they move an entry (4 (y (2M-1) + x) bytes).  Behind the last patch of a list the last one stands in.
struct PatchLists {
    static constexpr int kPatches = (kBiasMaxWindow / 8) * (kBiasMaxWindow / 8);
    uint16_t origin[9 * kPatches], entry[9 * kPatches];
};
static_assert(4 * (kBiasMaxWindow - 8) * 2 * kBiasMaxWindow < 65536, "an entry's bytes in 16 bits");
__device__ __forceinline__ void fill_patch_lists(const BiasItems& g, int M, PatchLists* lists, int thread, int threads)
{
    for (int e = thread; e < 9 * PatchLists::kPatches; e += threads) {
        const int kind = e / PatchLists::kPatches, k = e % PatchLists::kPatches;
        const AxisKind &ay = g.live.y[kind / 3], &ax = g.live.x[kind % 3];
        int py = 0, px = 0;
        if (ay.count * ax.count > 0) {
            int r, l;
            ax.by_count.divmod(min(k, ay.count * ax.count - 1), r, l);
            py = (r < ay.len0 ? ay.start0 + r : ay.start1 + r - ay.len0) << 3;
            px = (l < ax.len0 ? ax.start0 + l : ax.start1 + l - ax.len0) << 3;
        }
        lists->origin[e] = (uint16_t)(py << 8 | px);
        lists->entry[e] = (uint16_t)(4 * (py * (2 * M - 1) + px));
    }
}
__device__ __forceinline__ int list_of(const LiveItem& c) { return (3 * c.ky + c.kx) * PatchLists::kPatches; }
// Patch `sp` of the item's window in shifted, wrapped coordinates of the (extended) map.
__device__ __forceinline__ void patch_place(const WindowGeom& g, const PatchLists* lists, const LiveItem& c, int sp, int& Y0, int& X0)
{
    const int at = lists->origin[list_of(c) + sp];
    Y0 = c.wy * g.M + (at >> 8) + g.s; if (Y0 >= g.H) Y0 -= g.H;
    X0 = c.wx * g.M + (at & 255) + g.s; if (X0 >= g.W) X0 -= g.W;
}

// The first item whose work begins at or behind `at`, all heads' items laid one behind the other.  CTA c of n takes the items that begin in
// [c / n, (c + 1) / n) of the work: equal shares to within one item, and neighbours in the order, i.e. mostly one head.
__device__ __forceinline__ int first_bias_item(const BiasItems& g, long long at)
{
    const long long h = at / g.work[9];
    const long long r = at - h * g.work[9];
    int kind = 0;
#pragma unroll
    for (int k = 1; k < 9; ++k) kind += r >= g.work[k] ? 1 : 0;
    const int w = g.weight[kind];
    return (int)h * g.per_head + g.live.offset[kind] + (int)((r - g.work[kind] + w - 1) / w);
}

// `patches_per_item`: 4 (two query tiles) or 2 (one key block).
inline bool make_bias_items(const Problem& p, int patches_per_item, BiasItems* g)
{
    Problem one = p;
    one.heads = 1;
    if (!make_live_windows(one, &g->live)) return false;
    long long at = 0;
    int offset = 0;
    for (int k = 0; k < 9; ++k) {
        const long long patches = (long long)g->live.y[k / 3].count * g->live.x[k % 3].count;
        const long long items4 = g->live.offset[k + 1] - g->live.offset[k];      // of four patches each
        const long long per4 = (patches + 3) / 4, per = (patches + patches_per_item - 1) / patches_per_item;
        const long long items = items4 ? items4 / per4 * per : 0;
        g->work[k] = at;
        g->weight[k] = patches ? (int)((patches + 1) / 2) : 1;
        at += items * g->weight[k];
        g->live.offset[k] = offset;
        g->live.items_per_window[k] = make_fast_div(per > 0 ? (int)per : 1);
        if (offset + items > 0x7fffffffLL) return false;
        offset += (int)items;
    }
    g->work[9] = at;
    g->live.offset[9] = offset;
    g->per_head = offset;
    g->by_head = make_fast_div(offset > 0 ? offset : 1);
    return offset > 0 && (long long)offset * p.heads <= 0x7fffffffLL;
}

// What the kernels read of the caller's table.
struct BiasSource { const void* bias; const int* buckets; long long head_stride; int bf16, num_buckets; };
inline BiasSource bias_source(const Problem& p) { return {p.bias, p.buckets, p.bias_head_stride, p.bias_bf16, p.num_buckets}; }

// Threads `thread` of `threads` write head h's biases by offset, times log2(e), to shared memory; `masked` for keys that are not attended to.
__device__ __forceinline__ void gather_bias(const BiasSource& s, int h, int entries, float masked, float* table, int thread, int threads)
{
    constexpr int kAhead = 4;
    for (int e0 = thread; e0 < entries; e0 += kAhead * threads) {
        int u[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) u[k] = e0 + k * threads < entries ? __ldg(s.buckets + e0 + k * threads) : -1;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (e0 + k * threads < entries) {
                const float b = (unsigned)u[k] < (unsigned)s.num_buckets ? bias_at(s.bias, s.bf16, (long long)h * s.head_stride + u[k]) : -INFINITY;
                table[e0 + k * threads] = b == -INFINITY ? masked : b * kLog2e;         // (other biases lie above -1.5e30)
            }
    }
}

// Head width, window and shift that the kernels take; any H and W.
inline bool bias_shape_supported(const Problem& p)
{
    return p.bias && p.d % 8 == 0 && p.d >= 8 && p.d <= kD && p.M % 8 == 0 && p.M <= kBiasMaxWindow && p.s % 8 == 0;
}

}  // namespace sm100
}  // namespace rib
