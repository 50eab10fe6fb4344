// Norms of queries and keys for each head with the rotation by position in the same pass, forward and backward, and the table of the rotation.
//
//     xhat = x / sqrt(mean_c x_c^2 + eps),   z = w o xhat,   y = R z
// for every token and head; R turns pairs of the first `rot` channels - (2 i, 2 i + 1), or (i, i + rot / 2) - by y f_y[i] + x f_x[i].  The cosine and sine of the sum are
// the complex product of an entry of the map's row and one of its column, so that a table of H + W rows, with far angles taken in 64 bits, serves the map.
// Backward, with g the gradient of y:  gz = R^T g,   dw = sum gz o xhat,   dx = (w o gz - xhat mean_c(w o gz o xhat)) / sqrt(...).
//
// Bound by memory: 4 bytes a channel forward, 6 backward.  A thread has a unit of 2 V channels of a token - V pairs: two runs of V channels rot / 2 apart, or one of
// 2 V - and walks the heads with the token's cosines and sines in registers; the lanes of a head's row share its sums by shuffles.
#include "rib_common.cuh"
#include "rib_sm100_common.cuh"

namespace rib {
namespace {

using sm100::FastDiv;
using sm100::make_fast_div;

constexpr int kThreads = 256;

struct RopeTensor {
    const __nv_bfloat16 *x, *g;          // x: tokens x_stride elements apart; g (backward): [tokens][heads][d]
    __nv_bfloat16* y;                    // y or dx: tokens y_stride elements apart
    const float* w;                      // [d] or [heads][d]; null: no norm
    float* part;                         // backward: [chunks][blocks][d] sums of dw
    long long x_stride, y_stride;
    int heads, chunks, first_chunk;      // chunks of heads_per_chunk heads: blockIdx.y
};
struct RopeParams {
    RopeTensor t[2];
    const float2* table;                 // [H + W][rot / 2]
    long long tokens;
    int H, W, d, rot, pairs, interleaved, per_head, heads_per_chunk, lanes;
    float eps, inverse_d;
    FastDiv by_pixels, by_w;
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

// kUnroll heads of a token have their loads under way at once.
template <int V, bool kBackward>
__global__ void __launch_bounds__(kThreads) rib_qk_norm_rope_kernel(const RopeParams p)
{
    constexpr int kUnroll = kBackward ? 2 : 4;
    using W = typename Word<V>::type;
    const RopeTensor& t = p.t[(int)blockIdx.y >= p.t[1].first_chunk ? 1 : 0];
    const int chunk = blockIdx.y - t.first_chunk, head0 = chunk * p.heads_per_chunk, head1 = min(head0 + p.heads_per_chunk, t.heads);
    const int unit = threadIdx.x & (p.lanes - 1), turned = p.pairs / V;
    // channels of the unit's two runs; beyond d: none
    const bool rotates = unit < turned;
    int ca, cb;
    if (rotates) { ca = p.interleaved ? 2 * V * unit : V * unit; cb = p.interleaved ? ca + V : ca + p.rot / 2; }
    else { ca = p.rot + 2 * V * (unit - turned); cb = ca + V; }
    const bool has_a = ca < p.d, has_b = cb < p.d;
    const bool norm = t.w != nullptr;
    float w[2 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) {        // (weights per head: a chunk is one head)
        const float* src = t.w + (p.per_head ? (long long)head0 * p.d : 0);
        w[i] = norm && has_a ? __ldg(src + ca + i) : 1.f;
        w[V + i] = norm && has_b ? __ldg(src + cb + i) : 1.f;
    }
    float dw[2 * V];
    if constexpr (kBackward) {
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) dw[i] = 0.f;
    }
    const long long step = (long long)gridDim.x * (kThreads / p.lanes);
    const long long rounds = (p.tokens + step - 1) / step;       // the same for all lanes: they meet in shuffles
    long long token = (long long)blockIdx.x * (kThreads / p.lanes) + threadIdx.x / p.lanes;
    for (long long round = 0; round < rounds; ++round, token += step) {
        const bool there = token < p.tokens;
        float c[V], s[V];
        if (rotates && there) {
            int image, pixel, y, x;
            p.by_pixels.divmod((int)token, image, pixel);
            p.by_w.divmod(pixel, y, x);
            const float2 *row = p.table + (long long)y * p.pairs + V * unit, *column = p.table + (long long)(p.H + x) * p.pairs + V * unit;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float2 a = __ldg(row + i), b = __ldg(column + i);
                c[i] = a.x * b.x - a.y * b.y;
                s[i] = a.y * b.x + a.x * b.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) { c[i] = 1.f; s[i] = 0.f; }
        }
        for (int h0 = head0; h0 < head1; h0 += kUnroll) {
            W xa[kUnroll], xb[kUnroll], ga[kUnroll], gb[kUnroll];
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                const int h = h0 + k;
                const bool here = there && h < head1;
                xa[k] = W{}; xb[k] = W{}; ga[k] = W{}; gb[k] = W{};
                const __nv_bfloat16* src = t.x + token * t.x_stride + h * p.d;
                if (here && has_a) xa[k] = __ldg(reinterpret_cast<const W*>(src + ca));
                if (here && has_b) xb[k] = __ldg(reinterpret_cast<const W*>(src + cb));
                if constexpr (kBackward) {
                    const __nv_bfloat16* grad = t.g + (token * t.heads + h) * p.d;
                    if (here && has_a) ga[k] = __ldg(reinterpret_cast<const W*>(grad + ca));
                    if (here && has_b) gb[k] = __ldg(reinterpret_cast<const W*>(grad + cb));
                }
            }
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                const int h = h0 + k;
                if (h >= head1) break;                       // (the same for all lanes)
                float x[2 * V], z[2 * V];
                unpack<V>(xa[k], x);
                unpack<V>(xb[k], x + V);
                float squares = 0.f;
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) squares = fmaf(x[i], x[i], squares);
                float along = 0.f;
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
                float inverse = 1.f;
                if (norm) {
                    for (int o = p.lanes / 2; o; o >>= 1) {
                        squares += __shfl_xor_sync(0xffffffffu, squares, o);
                        if constexpr (kBackward) along += __shfl_xor_sync(0xffffffffu, along, o);
                    }
                    inverse = 1.f / sqrtf(fmaf(squares, p.inverse_d, p.eps));
                }
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
                    __nv_bfloat16* dst = t.y + token * t.y_stride + h * p.d;
                    if (has_a) *reinterpret_cast<W*>(dst + ca) = pack<V>(z);
                    if (has_b) *reinterpret_cast<W*>(dst + cb) = pack<V>(z + V);
                }
            }
        }
    }
    if constexpr (kBackward) {
        // sums of the block: lanes of the same unit, then warps, in a fixed order
        if (!norm) return;                                   // (the same for the block)
        __shared__ float sums[kThreads / 32][32][2 * V];
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < 2 * V; ++i)
            for (int o = p.lanes; o < 32; o <<= 1) dw[i] += __shfl_xor_sync(0xffffffffu, dw[i], o);
        if (lane < p.lanes) {
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) sums[warp][lane][i] = dw[i];
        }
        __syncthreads();
        if ((int)threadIdx.x < p.lanes) {
            float* dst = t.part + ((long long)chunk * gridDim.x + blockIdx.x) * p.d;
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) {
                float total = 0.f;
                for (int k = 0; k < kThreads / 32; ++k) total += sums[k][threadIdx.x][i];
                if (i < V ? has_a : has_b) dst[(i < V ? ca : cb - V) + i] = total;
            }
        }
    }
}

// dw of a tensor (or of one of its heads) from the blocks' sums: block (head, tensor), in a fixed order
struct RopeSum { const float* part; float* dw; int sums, heads; };      // sums: of d floats each, behind one another
__global__ void __launch_bounds__(1024) rib_qk_norm_rope_sum_kernel(RopeSum q, RopeSum k, int d)
{
    const RopeSum& t = blockIdx.y ? k : q;
    if ((int)blockIdx.x >= t.heads || !t.dw) return;
    __shared__ float sums[1024];
    const int c = threadIdx.x & 63, run = threadIdx.x >> 6;
    const float* src = t.part + (long long)blockIdx.x * t.sums * d;
    float total = 0.f;
    if (c < d)
        for (int i = run; i < t.sums; i += 16) total += src[(long long)i * d + c];
    sums[threadIdx.x] = total;
    __syncthreads();
    if (threadIdx.x < 64 && c < d) {
        for (int i = 1; i < 16; ++i) total += sums[64 * i + c];
        t.dw[(long long)blockIdx.x * d + c] = total;
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

struct Plan { int V, lanes, heads_per_chunk, chunks[2], blocks; };

int lanes_of(int units) { int l = 1; while (l < units) l *= 2; return l; }

// the widest words that every row allows
Plan rope_plan(const RopeProblem& p)
{
    Plan plan{};
    auto fits = [&](int V) {
        if (p.d % V || p.rot % (2 * V)) return false;
        for (int i = 0; i < (p.kv_heads ? 2 : 1); ++i) {
            const RopeRows& t = p.t[i];
            if (t.x_stride % V || t.y_stride % V || reinterpret_cast<uintptr_t>(t.x) % (2 * V) || reinterpret_cast<uintptr_t>(t.y) % (2 * V) || reinterpret_cast<uintptr_t>(t.g) % (2 * V)) return false;
        }
        return true;
    };
    plan.V = fits(8) ? 8 : fits(2) ? 2 : 1;
    plan.lanes = lanes_of(p.rot / (2 * plan.V) + (p.d - p.rot + 2 * plan.V - 1) / (2 * plan.V));
    return plan;
}

// Chunks of heads: all of a tensor's where the map fills the card, fewer where it does not; one where weights are per head.  (From the shape alone: the workspace's size depends on it.)
void rope_grid(const RopeProblem& p, int lanes, Plan* plan)
{
    const int most = p.heads > p.kv_heads ? p.heads : p.kv_heads;
    const long long per_block = kThreads / lanes, blocks = (p.tokens + per_block - 1) / per_block;
    plan->heads_per_chunk = most;
    while (plan->heads_per_chunk > 1 && blocks * (2 * (most / plan->heads_per_chunk)) < 2 * 148) plan->heads_per_chunk = (plan->heads_per_chunk + 1) / 2;
    if (p.per_head) plan->heads_per_chunk = 1;
    plan->chunks[0] = (p.heads + plan->heads_per_chunk - 1) / plan->heads_per_chunk;
    plan->chunks[1] = (p.kv_heads + plan->heads_per_chunk - 1) / plan->heads_per_chunk;
    const int chunks = plan->chunks[0] + plan->chunks[1], cap = (148 * 8 + chunks - 1) / chunks;
    plan->blocks = (int)(blocks < cap ? blocks : cap);
}

template <bool kBackward>
cudaError_t launch(const RopeProblem& p, float* part, const Plan& plan, cudaStream_t stream)
{
    RopeParams a{};
    for (int i = 0; i < 2; ++i) {
        const RopeRows& t = p.t[i];
        a.t[i] = RopeTensor{t.x, t.g, t.y, t.w, part, t.x_stride, t.y_stride, i ? p.kv_heads : p.heads, plan.chunks[i], i ? plan.chunks[0] : 0};
        if (part) part += (long long)plan.chunks[i] * plan.blocks * p.d;
    }
    a.table = reinterpret_cast<const float2*>(p.table); a.tokens = p.tokens; a.H = p.H; a.W = p.W; a.d = p.d; a.rot = p.rot; a.pairs = p.rot / 2;
    a.interleaved = p.interleaved; a.per_head = p.per_head; a.heads_per_chunk = plan.heads_per_chunk; a.lanes = plan.lanes; a.eps = p.eps; a.inverse_d = 1.f / (float)p.d;
    a.by_pixels = make_fast_div((int)((long long)p.H * p.W)); a.by_w = make_fast_div(p.W);
    const dim3 grid((unsigned)plan.blocks, (unsigned)(plan.chunks[0] + plan.chunks[1]));
    ProfileScope scope(kBackward ? RIB_KERNEL_QK_NORM_ROPE_BWD : RIB_KERNEL_QK_NORM_ROPE_FWD, stream);
    if (plan.V == 8) rib_qk_norm_rope_kernel<8, kBackward><<<grid, kThreads, 0, stream>>>(a);
    else if (plan.V == 2) rib_qk_norm_rope_kernel<2, kBackward><<<grid, kThreads, 0, stream>>>(a);
    else rib_qk_norm_rope_kernel<1, kBackward><<<grid, kThreads, 0, stream>>>(a);
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

cudaError_t qk_norm_rope_fwd(const RopeProblem& p, cudaStream_t stream)
{
    Plan plan = rope_plan(p);
    rope_grid(p, plan.lanes, &plan);
    return launch<false>(p, nullptr, plan, stream);
}

// room for the largest number of blocks of any alignment (the number of lanes is at most 32)
size_t qk_norm_rope_bwd_workspace(const RopeProblem& p)
{
    size_t most = 0;
    for (int lanes = 1; lanes <= 32; lanes *= 2) {
        Plan plan{};
        rope_grid(p, lanes, &plan);
        const size_t bytes = sizeof(float) * (size_t)(plan.chunks[0] + plan.chunks[1]) * plan.blocks * p.d;
        most = bytes > most ? bytes : most;
    }
    return (most + 255) & ~(size_t)255;
}

cudaError_t qk_norm_rope_bwd(const RopeProblem& p, float* workspace, int* launches, cudaStream_t stream)
{
    Plan plan = rope_plan(p);
    rope_grid(p, plan.lanes, &plan);
    *launches = 1;
    if (cudaError_t e = launch<true>(p, workspace, plan, stream)) return e;
    if (!p.t[0].dw && !p.t[1].dw) return cudaSuccess;
    RopeSum s[2]{};
    const float* part = workspace;
    for (int i = 0; i < 2; ++i) {
        s[i] = RopeSum{part, p.t[i].dw, p.per_head ? plan.blocks : plan.chunks[i] * plan.blocks, p.per_head ? (i ? p.kv_heads : p.heads) : 1};
        part += (long long)plan.chunks[i] * plan.blocks * p.d;
    }
    const int heads = s[0].heads > s[1].heads ? s[0].heads : s[1].heads;
    *launches = 2;
    ProfileScope scope(RIB_KERNEL_QK_NORM_ROPE_SUM, stream);
    rib_qk_norm_rope_sum_kernel<<<dim3((unsigned)heads, 2), 1024, 0, stream>>>(s[0], s[1], p.d);
    return cudaGetLastError();
}

}  // namespace rib
