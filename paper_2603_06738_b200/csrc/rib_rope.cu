// Norms of queries and keys for each head with the rotation by position in the same pass, forward and backward, and the table of the rotation.
//
//     xhat = x / sqrt(mean_c x_c^2 + eps),   z = w o xhat,   y = R z
// for every token and head; R turns pairs of the first `rot` channels - (2 i, 2 i + 1), or (i, i + rot / 2) - by y f_y[i] + x f_x[i].  The cosine and sine of the sum are
// the complex product of an entry of the map's row and one of its column, so that a table of H + W rows, with far angles taken in 64 bits, serves the map.
// Backward, with g the gradient of y:  gz = R^T g,   dw = sum gz o xhat,   dx = (w o gz - xhat mean_c(w o gz o xhat)) / sqrt(...).
//
// Bound by memory: 4 bytes a channel forward, 6 backward.  A thread has a unit of 2 V channels - V pairs: two runs of V channels rot / 2 apart, or one of 2 V - of one row (a head of q or k)
// and walks tokens, kUnroll of them with their loads under way at once: a warp's accesses cover neighbouring rows of a token, whole lines, and weights and their gradients stay in registers.  The lanes
// of a row share its sums by shuffles.  A block takes tiles of tokens and puts their cosines and sines into shared memory first, once for all heads.
// (A thread to a token that walks the heads, table entries in registers: 32 lines touched by every access and few of them in flight, 16 x 96 x 96 tokens, 6 heads of 32, forward and backward 172 us
// against 000.)
#include "rib_common.cuh"
#include "rib_sm100_common.cuh"

namespace rib {
namespace {

using sm100::FastDiv;
using sm100::make_fast_div;

constexpr int kThreads = 256, kMaxTile = 64, kMaxBlocks = 4 * 148;

struct RopeTensor {
    const __nv_bfloat16 *x, *g;          // x: tokens x_stride elements apart; g (backward): [tokens][heads][d]
    __nv_bfloat16* y;                    // y or dx: tokens y_stride elements apart
    const float* w;                      // [d] or [heads][d]; null: no norm
    long long x_stride, y_stride;
    int heads;
};
struct RopeParams {
    RopeTensor t[2];
    const float2* table;                 // [H + W][rot / 2]
    float* part;                         // backward, sums of dw: [chunks][blocks][2 or rows_per_chunk][d]
    int tokens, tile, tiles, H, W, d, rot, pairs, interleaved, per_head, lanes, rows, rows_per_chunk, tokens_at_once;      // rows: heads of q, then of k; blockIdx.y: a chunk of them
    float eps, inverse_d;
    FastDiv by_pixels, by_w, by_pairs, by_slots;
};

template <int V> struct Word;
template <> struct Word<8> { using type = uint4; };
template <> struct Word<2> { using type = uint32_t; };
template <> struct Word<1> { using type = unsigned short; };

template <int V> __device__ __forceinline__ void unpack(const typename Word<V>::type& word, float* x)
{
    if constexpr (V == 1) {
        x[0] = __uint_as_float((uint32_t)word << 16);
    } else {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&word);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
}
template <int V> __device__ __forceinline__ typename Word<V>::type pack(const float* x)
{
    typename Word<V>::type word;
    if constexpr (V == 1) {
        word = __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
    } else {
        uint32_t* w = reinterpret_cast<uint32_t*>(&word);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) w[i] = sm100::pack_bf16x2(x[2 * i], x[2 * i + 1]);
    }
    return word;
}

template <int V, bool kBackward>
__global__ void __launch_bounds__(kThreads) rib_qk_norm_rope_kernel(const __grid_constant__ RopeParams p)
{
    constexpr int kUnroll = V == 8 ? (kBackward ? 2 : 4) : 4;
    using W = typename Word<V>::type;
    extern __shared__ __align__(16) float2 turns[];              // [tile][pairs] cosines and sines; backward, at the end: [threads][2 V] sums
    // this thread: unit of a row of the chunk, and which of the tokens that are walked at once
    int at_once, slot;
    p.by_slots.divmod(threadIdx.x, at_once, slot);               // slots: rows of a chunk x lanes of a row
    const int unit = slot & (p.lanes - 1), chunk_row = slot / p.lanes, row = blockIdx.y * p.rows_per_chunk + chunk_row;
    const bool works = at_once < p.tokens_at_once && row < p.rows;
    const bool is_k = row >= p.t[0].heads;
    const RopeTensor& t = p.t[is_k ? 1 : 0];
    const int head = is_k ? row - p.t[0].heads : row;
    // channels of the unit's two runs; beyond d: none
    const int turned = p.pairs / V;
    const bool rotates = unit < turned;
    int ca, cb;
    if (rotates) { ca = p.interleaved ? 2 * V * unit : V * unit; cb = p.interleaved ? ca + V : ca + p.rot / 2; }
    else { ca = p.rot + 2 * V * (unit - turned); cb = ca + V; }
    const bool has_a = works && ca < p.d, has_b = works && cb < p.d;
    const bool norm = works && t.w != nullptr;
    float w[2 * V], dw[2 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float* src = t.w + (p.per_head ? head * p.d : 0);
        w[i] = norm && has_a ? __ldg(src + ca + i) : 1.f;
        w[V + i] = norm && has_b ? __ldg(src + cb + i) : 1.f;
    }
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) dw[i] = 0.f;
    const __nv_bfloat16 *x_at = t.x + head * p.d, *g_at = kBackward ? t.g + head * p.d : nullptr;
    __nv_bfloat16* y_at = t.y + head * p.d;
    const long long x_stride = t.x_stride, y_stride = t.y_stride;
    const int g_stride = t.heads * p.d;

    for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
        const int token0 = tile * p.tile, here = min(p.tile, p.tokens - token0);
        if (p.rot) {
            __syncthreads();                                     // the tile before has been used
            for (int e = threadIdx.x; e < here * p.pairs; e += kThreads) {
                int token, i, image, pixel, y, x;
                p.by_pairs.divmod(e, token, i);
                p.by_pixels.divmod(token0 + token, image, pixel);
                p.by_w.divmod(pixel, y, x);
                const float2 a = __ldg(p.table + (long long)y * p.pairs + i), b = __ldg(p.table + (long long)(p.H + x) * p.pairs + i);
                turns[e] = make_float2(a.x * b.x - a.y * b.y, a.y * b.x + a.x * b.y);
            }
            __syncthreads();
        }
        // (all lanes walk alike: those of a row meet in shuffles)
        for (int k0 = 0; k0 < here; k0 += kUnroll * p.tokens_at_once) {
            W xa[kUnroll], xb[kUnroll], ga[kUnroll], gb[kUnroll];
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                const int token = k0 + k * p.tokens_at_once + at_once;
                const bool there = token < here;
                xa[k] = W{}; xb[k] = W{}; ga[k] = W{}; gb[k] = W{};
                const __nv_bfloat16* src = x_at + (token0 + token) * x_stride;
                if (there && has_a) xa[k] = __ldg(reinterpret_cast<const W*>(src + ca));
                if (there && has_b) xb[k] = __ldg(reinterpret_cast<const W*>(src + cb));
                if constexpr (kBackward) {
                    const __nv_bfloat16* grad = g_at + (long long)(token0 + token) * g_stride;
                    if (there && has_a) ga[k] = __ldg(reinterpret_cast<const W*>(grad + ca));
                    if (there && has_b) gb[k] = __ldg(reinterpret_cast<const W*>(grad + cb));
                }
            }
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                if (k0 + k * p.tokens_at_once >= here) break;    // (the same for all threads)
                const int token = k0 + k * p.tokens_at_once + at_once;
                const bool there = token < here;
                float c[V], s[V];
#pragma unroll
                for (int i = 0; i < V; ++i) { c[i] = 1.f; s[i] = 0.f; }
                if (rotates && there) {
                    if constexpr (V == 8) {
                        const float4* src = reinterpret_cast<const float4*>(turns + token * p.pairs + V * unit);
#pragma unroll
                        for (int i = 0; i < V / 2; ++i) {
                            const float4 q = src[i];
                            c[2 * i] = q.x; s[2 * i] = q.y; c[2 * i + 1] = q.z; s[2 * i + 1] = q.w;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < V; ++i) { const float2 q = turns[token * p.pairs + V * unit + i]; c[i] = q.x; s[i] = q.y; }
                    }
                }
                float x[2 * V], z[2 * V];
                unpack<V>(xa[k], x);
                unpack<V>(xb[k], x + V);
                float squares = 0.f, along = 0.f;
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) squares = fmaf(x[i], x[i], squares);
                if constexpr (kBackward) {
                    float g[2 * V];
                    unpack<V>(ga[k], g);
                    unpack<V>(gb[k], g + V);
                    // back by the transposed rotation
                    if (p.interleaved) {
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            z[2 * i] = fmaf(c[i], g[2 * i], s[i] * g[2 * i + 1]);
                            z[2 * i + 1] = fmaf(c[i], g[2 * i + 1], -s[i] * g[2 * i]);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            z[i] = fmaf(c[i], g[i], s[i] * g[V + i]);
                            z[V + i] = fmaf(c[i], g[V + i], -s[i] * g[i]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) along = fmaf(z[i] * w[i], x[i], along);
                }
                for (int o = p.lanes / 2; o; o >>= 1) {          // (rows without a norm beside rows with one: all take part)
                    squares += __shfl_xor_sync(0xffffffffu, squares, o);
                    if constexpr (kBackward) along += __shfl_xor_sync(0xffffffffu, along, o);
                }
                const float inverse = norm ? rsqrtf(fmaf(squares, p.inverse_d, p.eps)) : 1.f;
                if constexpr (kBackward) {
                    const float mean = norm ? along * inverse * p.inverse_d : 0.f;       // mean_c(w gz xhat)
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) {
                        const float unit_x = x[i] * inverse;
                        if (there) dw[i] = fmaf(z[i], unit_x, dw[i]);
                        z[i] = norm ? inverse * fmaf(-unit_x, mean, z[i] * w[i]) : z[i];
                    }
                } else {
                    float n[2 * V];
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) n[i] = norm ? x[i] * inverse * w[i] : x[i];
                    if (p.interleaved) {
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            z[2 * i] = fmaf(c[i], n[2 * i], -s[i] * n[2 * i + 1]);
                            z[2 * i + 1] = fmaf(c[i], n[2 * i + 1], s[i] * n[2 * i]);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            z[i] = fmaf(c[i], n[i], -s[i] * n[V + i]);
                            z[V + i] = fmaf(c[i], n[V + i], s[i] * n[i]);
                        }
                    }
                }
                if (there) {
                    __nv_bfloat16* dst = y_at + (token0 + token) * y_stride;
                    if (has_a) *reinterpret_cast<W*>(dst + ca) = pack<V>(z);
                    if (has_b) *reinterpret_cast<W*>(dst + cb) = pack<V>(z + V);
                }
            }
        }
    }
    if constexpr (kBackward) {
        if (!p.part) return;
        // Sums of the block in a fixed order: of a row's channel over the tokens at once, or of a tensor's over its rows of the chunk too.
        float* const sums = reinterpret_cast<float*>(turns);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) sums[threadIdx.x * 2 * V + i] = dw[i];
        __syncthreads();
        const int slots = p.rows_per_chunk * p.lanes, outputs = p.per_head ? p.rows_per_chunk : 2;
        float* const dst = p.part + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * outputs * p.d;
        for (int e = threadIdx.x; e < outputs * p.d; e += kThreads) {
            const int which = e / p.d, ch = e - which * p.d;
            // the unit and place of the channel
            int u, place;
            if (ch < p.rot) {
                const int half = p.rot / 2;
                if (p.interleaved) { u = ch / (2 * V); place = ch - u * 2 * V; }
                else { const int in = ch < half ? ch : ch - half; u = in / V; place = in - u * V + (ch < half ? 0 : V); }
            } else {
                const int in = ch - p.rot;
                u = turned + in / (2 * V); place = in % (2 * V);
            }
            const int row0 = blockIdx.y * p.rows_per_chunk;
            int first = which, end = which + 1;                  // rows of the chunk
            if (!p.per_head) {
                first = which ? max(0, p.t[0].heads - row0) : 0;
                end = which ? min(p.rows_per_chunk, p.rows - row0) : min(p.rows_per_chunk, p.t[0].heads - row0);
            }
            float total = 0.f;
            for (int r = first; r < end; ++r)
                for (int k = 0; k < p.tokens_at_once; ++k) total += sums[(k * slots + r * p.lanes + u) * 2 * V + place];
            dst[e] = total;
        }
    }
}

// dw of a tensor (or of one of its heads) from the blocks' sums: block (output of a chunk, or of all chunks), in a fixed order
struct RopeSum { const float* part; float* dw[2]; int d, blocks, chunks, outputs, per_head, rows_per_chunk, heads, rows; };
__global__ void __launch_bounds__(1024) rib_qk_norm_rope_sum_kernel(const RopeSum t)
{
    __shared__ float sums[1024];
    const int c = threadIdx.x & 63, run = threadIdx.x >> 6;
    // per head: blockIdx.x is a row, in one chunk; else a tensor, in all of them
    const int chunk = t.per_head ? blockIdx.x / t.rows_per_chunk : 0, output = t.per_head ? blockIdx.x % t.rows_per_chunk : blockIdx.x, chunks = t.per_head ? 1 : t.chunks;
    const bool is_k = t.per_head ? (int)blockIdx.x >= t.heads : blockIdx.x == 1;
    float* const dst = t.dw[is_k ? 1 : 0];
    cudaGridDependencySynchronize();                             // it may have overtaken the kernel before
    if (!dst) return;
    float total = 0.f;
    if (c < t.d)
        for (int i = run; i < chunks * t.blocks; i += 16) total += t.part[((long long)chunk * t.blocks + i) * t.outputs * t.d + output * t.d + c];
    sums[threadIdx.x] = total;
    __syncthreads();
    if (threadIdx.x < 64 && c < t.d) {
        for (int i = 1; i < 16; ++i) total += sums[64 * i + c];
        dst[(t.per_head ? (int)blockIdx.x - (is_k ? t.heads : 0) : 0) * t.d + c] = total;
    }
}

// Angles are products of whole numbers and 32-bit frequencies, exact in 64 bits; their cosine and sine are rounded once.
__global__ void __launch_bounds__(128) rib_rope_table_kernel(const float* __restrict__ frequencies, int H, int W, int pairs, long long y0, long long x0, float magnitude, float2* __restrict__ table)
{
    const long long e = (long long)blockIdx.x * 128 + threadIdx.x;
    if (e >= ((long long)H + W) * pairs) return;
    const long long row = e / pairs;
    const int i = (int)(e - row * pairs);
    const bool column = row >= H;
    double sine, cosine;
    sincos((double)(column ? x0 + row - H : y0 + row) * (double)frequencies[column ? pairs + i : i], &sine, &cosine);
    const double scale = column ? 1.0 : (double)magnitude;
    table[e] = make_float2((float)(scale * cosine), (float)(scale * sine));
}

struct Plan { int V, lanes, rows, rows_per_chunk, chunks, tokens_at_once, tile, tiles, blocks; };

int lanes_of(int units) { int l = 1; while (l < units) l *= 2; return l; }

// rows of a chunk and blocks along the tokens, for rows of `lanes` lanes
void rope_grid(const RopeProblem& p, int lanes, Plan* plan)
{
    plan->lanes = lanes;
    plan->rows = p.heads + p.kv_heads;
    const int most = kThreads / lanes;
    plan->chunks = (plan->rows + most - 1) / most;
    plan->rows_per_chunk = (plan->rows + plan->chunks - 1) / plan->chunks;
    plan->chunks = (plan->rows + plan->rows_per_chunk - 1) / plan->rows_per_chunk;
    plan->tokens_at_once = kThreads / (plan->rows_per_chunk * lanes);
    // tiles such that a small map still gives every SM two of them
    long long tile = p.tokens / (2 * 148);
    if (tile < plan->tokens_at_once) tile = plan->tokens_at_once;
    if (tile > kMaxTile) tile = kMaxTile;
    plan->tile = (int)tile;
    plan->tiles = (int)((p.tokens + tile - 1) / tile);
    const int cap = (kMaxBlocks + plan->chunks - 1) / plan->chunks;
    plan->blocks = plan->tiles < cap ? plan->tiles : cap;
}

// the widest words that every row allows
Plan rope_plan(const RopeProblem& p)
{
    auto fits = [&](int V) {
        if (p.d % V || p.rot % (2 * V)) return false;
        for (int i = 0; i < (p.kv_heads ? 2 : 1); ++i) {
            const RopeRows& t = p.t[i];
            if (t.x_stride % V || t.y_stride % V || reinterpret_cast<uintptr_t>(t.x) % (2 * V) || reinterpret_cast<uintptr_t>(t.y) % (2 * V) || reinterpret_cast<uintptr_t>(t.g) % (2 * V)) return false;
        }
        return true;
    };
    Plan plan{};
    plan.V = fits(8) ? 8 : fits(2) ? 2 : 1;
    rope_grid(p, lanes_of(p.rot / (2 * plan.V) + (p.d - p.rot + 2 * plan.V - 1) / (2 * plan.V)), &plan);
    return plan;
}

size_t part_floats(const Plan& plan, int d, bool per_head) { return (size_t)plan.chunks * plan.blocks * (per_head ? plan.rows_per_chunk : 2) * d; }

template <bool kBackward>
cudaError_t launch(const RopeProblem& p, float* part, const Plan& plan, cudaStream_t stream)
{
    RopeParams a{};
    for (int i = 0; i < 2; ++i) {
        const RopeRows& t = p.t[i];
        a.t[i] = RopeTensor{t.x, t.g, t.y, t.w, t.x_stride, t.y_stride, i ? p.kv_heads : p.heads};
    }
    a.table = reinterpret_cast<const float2*>(p.table); a.part = part; a.tokens = (int)p.tokens; a.tile = plan.tile; a.tiles = plan.tiles; a.H = p.H; a.W = p.W; a.d = p.d; a.rot = p.rot;
    a.pairs = p.rot / 2; a.interleaved = p.interleaved; a.per_head = p.per_head; a.lanes = plan.lanes; a.rows = plan.rows; a.rows_per_chunk = plan.rows_per_chunk;
    a.tokens_at_once = plan.tokens_at_once; a.eps = p.eps; a.inverse_d = 1.f / (float)p.d;
    a.by_pixels = make_fast_div((int)((long long)p.H * p.W)); a.by_w = make_fast_div(p.W); a.by_pairs = make_fast_div(p.rot ? p.rot / 2 : 1);
    a.by_slots = make_fast_div(plan.rows_per_chunk * plan.lanes);
    const dim3 grid((unsigned)plan.blocks, (unsigned)plan.chunks);
    size_t smem = sizeof(float2) * plan.tile * a.pairs;                                  // up to 16 KB
    if (kBackward && part && smem < sizeof(float) * kThreads * 2 * plan.V) smem = sizeof(float) * kThreads * 2 * plan.V;
    ProfileScope scope(kBackward ? RIB_KERNEL_QK_NORM_ROPE_BWD : RIB_KERNEL_QK_NORM_ROPE_FWD, stream);
    if (plan.V == 8) rib_qk_norm_rope_kernel<8, kBackward><<<grid, kThreads, smem, stream>>>(a);
    else if (plan.V == 2) rib_qk_norm_rope_kernel<2, kBackward><<<grid, kThreads, smem, stream>>>(a);
    else rib_qk_norm_rope_kernel<1, kBackward><<<grid, kThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t rope_table(const float* frequencies, int H, int W, int pairs, long long y0, long long x0, float magnitude, float* table, cudaStream_t stream)
{
    const long long entries = ((long long)H + W) * pairs;
    ProfileScope scope(RIB_KERNEL_ROPE_TABLE, stream);
    rib_rope_table_kernel<<<(unsigned)((entries + 127) / 128), 128, 0, stream>>>(frequencies, H, W, pairs, y0, x0, magnitude, reinterpret_cast<float2*>(table));
    return cudaGetLastError();
}

cudaError_t qk_norm_rope_fwd(const RopeProblem& p, cudaStream_t stream) { return launch<false>(p, nullptr, rope_plan(p), stream); }

// room for the sums of any alignment (a row has 1 to 32 lanes)
size_t qk_norm_rope_bwd_workspace(const RopeProblem& p)
{
    size_t most = 0;
    for (int lanes = 1; lanes <= 32; lanes *= 2) {
        Plan plan{};
        rope_grid(p, lanes, &plan);
        const size_t bytes = sizeof(float) * part_floats(plan, p.d, p.per_head != 0);
        most = bytes > most ? bytes : most;
    }
    return (most + 255) & ~(size_t)255;
}

cudaError_t qk_norm_rope_bwd(const RopeProblem& p, float* workspace, int* launches, cudaStream_t stream)
{
    const Plan plan = rope_plan(p);
    const bool weights = p.t[0].dw || p.t[1].dw;
    *launches = 1;
    if (cudaError_t e = launch<true>(p, weights ? workspace : nullptr, plan, stream)) return e;
    if (!weights) return cudaSuccess;
    const RopeSum s{workspace, {p.t[0].dw, p.t[1].dw}, p.d, plan.blocks, plan.chunks, p.per_head ? plan.rows_per_chunk : 2, p.per_head, plan.rows_per_chunk, p.heads, plan.rows};
    *launches = 2;
    ProfileScope scope(RIB_KERNEL_QK_NORM_ROPE_SUM, stream);
    return launch_overtaking(rib_qk_norm_rope_sum_kernel, p.per_head ? plan.rows : 2, 1024, 0, stream, s);
}

}  // namespace rib
