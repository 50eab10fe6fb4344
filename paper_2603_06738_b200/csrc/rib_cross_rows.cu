// Forward pass of the attention to states (rib_cross.cuh) for a group of few rows - single tokens that are served, each over a long context of its own - on the plain pipes.
//
// With R rows to a group (tokens x heads that share a head of keys) there are 4 R d flops for the 4 d bytes of a key and its value: memory bounds it, and a tensor-core tile of 128 rows would be
// mostly empty (a tile takes the exponentials of all its rows' warps: 64 single tokens, 6 heads of 32, to 64 to 4096 states 80 us, this kernel and the join 31).
// A block has a run of a group's keys; a key belongs to d / 8 lanes of a warp (rounded up to a power of two), 16 bytes of K and V each, kUnroll keys of a lane under way at once.  Every group of lanes
// keeps a running maximum, sum and output of its own for each row, all in 32 bits and P unrounded; lanes, warps and runs are joined at the end, in a fixed order.
#include "rib_cross.cuh"

namespace rib {
namespace {

using namespace sm100;

constexpr int kThreads = 128, kWarps = kThreads / 32;

struct RowsParams {
    const __nv_bfloat16 *q, *k, *v;
    const int* lengths;
    __nv_bfloat16* out;
    float *lse, *part_out, *part_lse;    // splits > 1: [splits][groups][rows][stride], [splits][groups][rows]
    int d, width, L, heads, kv_heads, G, tokens, rows, splits, shared, pixels, vector, stride;
    long long groups;
    float scale_log2, down, bits;        // down = 2^-bits: factor of the weights
};

__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[8])
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}

// kLanes lanes to a key, kRows rows.
template <int kLanes, int kRows>
__global__ void __launch_bounds__(kThreads) rib_cross_rows_kernel(const __grid_constant__ RowsParams p)
{
    constexpr int kKeys = 32 / kLanes, kUnroll = kRows == 1 ? 8 : 4;                   // kKeys: of a warp at once
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = lane % kLanes, which = lane / kLanes;
    const int split = blockIdx.x % p.splits, group = blockIdx.x / p.splits, context = group / p.kv_heads, kv = group - context * p.kv_heads;
    cudaGridDependencySynchronize();                      // it may have overtaken the kernel before
    const int length = p.lengths ? min(max(p.lengths[context], 0), p.L) : p.L;
    // runs of equal length of the context's own keys
    const int run = (length + p.splits - 1) / p.splits, first = min(length, split * run), last = min(length, first + run);
    const bool has = 8 * part < p.width;
    // rows of the group: token by token, its G heads
    float q[kRows][8], o[kRows][8], m[kRows], l[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        const int token = r / p.G, head = kv * p.G + r % p.G;
        if (has) w = *(reinterpret_cast<const uint4*>(p.q + ((long long)(context * p.tokens + token) * p.heads + head) * p.width) + part);
        unpack8(w, q[r]);
        m[r] = kCrossLowest; l[r] = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) { q[r][c] *= p.scale_log2; o[r][c] = 0.f; }
    }
    const long long step = (long long)p.kv_heads * p.width;      // elements from a state to the next one
    const __nv_bfloat16 *k_at = p.k + (long long)context * p.L * step + kv * p.width + 8 * part, *v_at = p.v + (k_at - p.k);
    for (int j0 = first + warp * kKeys * kUnroll; j0 < last; j0 += kWarps * kKeys * kUnroll) {
        uint4 kw[kUnroll], vw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int j = j0 + u * kKeys + which;
            const bool there = has && j < last;
            kw[u] = there ? *reinterpret_cast<const uint4*>(k_at + j * step) : make_uint4(0u, 0u, 0u, 0u);
            vw[u] = there ? *reinterpret_cast<const uint4*>(v_at + j * step) : make_uint4(0u, 0u, 0u, 0u);
        }
        float s[kRows][kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float x[8];
            unpack8(kw[u], x);
            const bool there = j0 + u * kKeys + which < last;
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                float sum = q[r][0] * x[0];
#pragma unroll
                for (int c = 1; c < 8; ++c) sum = fmaf(q[r][c], x[c], sum);
#pragma unroll
                for (int w = 1; w < kLanes; w <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
                s[r][u] = there ? sum : -INFINITY;
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            float most = m[r];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) most = fmaxf(most, s[r][u]);
            const float factor = ex2_approx(m[r] - most);
            m[r] = most;
            l[r] *= factor;
#pragma unroll
            for (int c = 0; c < 8; ++c) o[r][c] *= factor;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) { s[r][u] = ex2_approx(s[r][u] - most) * p.down; l[r] += s[r][u]; }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float x[8];
            unpack8(vw[u], x);
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int c = 0; c < 8; ++c) o[r][c] = fmaf(s[r][u], x[c], o[r][c]);
        }
    }
    // ---- lanes of a warp, then the warps
    __shared__ float sums[kWarps][kRows][kLanes * 8 + 2];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
#pragma unroll
        for (int w = kLanes; w < 32; w <<= 1) {
            const float other = __shfl_xor_sync(0xffffffffu, m[r], w), most = fmaxf(m[r], other);
            const float mine = ex2_approx(m[r] - most), theirs = ex2_approx(other - most);
            l[r] = l[r] * mine + __shfl_xor_sync(0xffffffffu, l[r], w) * theirs;
#pragma unroll
            for (int c = 0; c < 8; ++c) o[r][c] = o[r][c] * mine + __shfl_xor_sync(0xffffffffu, o[r][c], w) * theirs;
            m[r] = most;
        }
        if (which == 0) {
#pragma unroll
            for (int c = 0; c < 8; ++c) sums[warp][r][8 * part + c] = o[r][c];
            if (part == 0) { sums[warp][r][kLanes * 8] = m[r]; sums[warp][r][kLanes * 8 + 1] = l[r]; }
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.rows * kLanes * 8; e += kThreads) {
        const int r = e / (kLanes * 8), c = e - r * (kLanes * 8);
        float most = kCrossLowest, total = 0.f, x = 0.f;
        for (int w = 0; w < kWarps; ++w) most = fmaxf(most, sums[w][r][kLanes * 8]);
        for (int w = 0; w < kWarps; ++w) {
            const float factor = ex2_approx(sums[w][r][kLanes * 8] - most);
            total += sums[w][r][kLanes * 8 + 1] * factor;
            x += sums[w][r][c] * factor;
        }
        const bool none = first == last;                 // (a run of keys that all weigh nothing adds nothing either)
        const bool empty = none || (p.splits > 1 && total == 0.f);
        const float y = empty ? 0.f : x / total, lse = empty ? -INFINITY : (most + (__log2f(total) + p.bits)) * 0.6931471805599453f;
        const int token = r / p.G, head = kv * p.G + r % p.G;
        if (p.splits > 1) {
            const long long at = ((long long)split * p.groups + group) * p.rows + r;
            p.part_out[at * p.stride + c] = y;
            if (c == 0) p.part_lse[at] = lse;
        } else {
            const long long row = (long long)(context * p.tokens + token) * p.heads + head;
            if (c < p.d) p.out[row * p.d + c] = __float2bfloat16_rn(y);
            if (c == 0 && p.lse) {
                const int image = p.shared ? token / p.pixels : context, pixel = p.shared ? token % p.pixels : token;
                p.lse[((long long)image * p.heads + head) * p.pixels + pixel] = lse;
            }
        }
    }
}

template <int kLanes>
cudaError_t launch_lanes(const RowsParams& a, unsigned blocks, cudaStream_t stream)
{
    static_assert(kCrossFewRows == 2, "a kernel for every number of rows");
    const auto kernel = a.rows == 1 ? rib_cross_rows_kernel<kLanes, 1> : rib_cross_rows_kernel<kLanes, 2>;
    return launch_overtaking(kernel, blocks, kThreads, 0, stream, a);
}

}  // namespace

cudaError_t cross_fwd_rows(const CrossProblem& p, const CrossPlan& plan, float* part_out, float* part_lse, int stride, cudaStream_t stream)
{
    RowsParams a{};
    a.q = p.q; a.k = p.k; a.v = p.v; a.lengths = p.lengths; a.out = p.out_w; a.lse = p.lse_w; a.part_out = part_out; a.part_lse = part_lse;
    a.d = p.d; a.width = p.width; a.L = p.L; a.heads = p.heads; a.kv_heads = p.kv_heads; a.G = plan.G; a.tokens = (int)p.tokens; a.rows = (int)plan.rows; a.splits = plan.splits;
    a.shared = p.tokens != p.pixels; a.pixels = (int)p.pixels; a.stride = stride; a.groups = plan.groups; a.scale_log2 = 1.4426950408889634f / sqrtf((float)p.d);
    const int bits = cross_bits(p.L);
    a.bits = (float)bits; a.down = 1.f / (float)(1ll << bits);
    const unsigned blocks = (unsigned)(plan.groups * plan.splits);
    ProfileScope scope(RIB_KERNEL_CROSS_FWD, stream);
    return p.width <= 8 ? launch_lanes<1>(a, blocks, stream) : p.width <= 16 ? launch_lanes<2>(a, blocks, stream) : p.width <= 32 ? launch_lanes<4>(a, blocks, stream) : launch_lanes<8>(a, blocks, stream);
}

}  // namespace rib
