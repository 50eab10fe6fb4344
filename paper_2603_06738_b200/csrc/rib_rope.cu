// Norms of queries and keys for each head with the rotation by position in the same pass, forward and backward, and the table of the rotation.
//
//     xhat = x / sqrt(mean_c x_c^2 + eps),   z = w o xhat,   y = R z
// for every token and head; R turns pairs of the first `rot` channels - (2 i, 2 i + 1), or (i, i + rot / 2) - by y f_y[i] + x f_x[i].  The cosine and sine of the sum are
// the complex product of an entry of the map's row and one of its column, so that a table of H + W rows, with far angles taken in 64 bits, serves the map.
// Backward, with g the gradient of y:  gz = R^T g,   dw = sum gz o xhat,   dx = (w o gz - xhat mean_c(w o gz o xhat)) / sqrt(...).
//
// Bound by memory: 4 bytes a channel forward, 6 backward.  A thread has a unit of 2 V channels - V pairs: two runs of V channels rot / 2 apart - of one row (a head of q or k)
// and walks tokens, kUnroll of them with their loads under way at once: a warp's accesses cover neighbouring rows of a token, whole lines, and weights and their gradients stay in registers.  The lanes
// of a row share its sums by shuffles.  A block takes tiles of tokens and puts their cosines and sines into shared memory first, once for all heads.
// (Plain loads, not the read-only path: a kernel may start under the one that makes its inputs, and waits for its end.)
// (A thread to a token that walks the heads, table entries in registers: 32 lines touched by every access and few of them in flight, 16 x 96 x 96 tokens, 6 heads of 32, forward and backward 172 us
// against 137 now.)
#include "rib_common.cuh"
#include "rib_sm100_common.cuh"

namespace rib {
namespace {

using sm100::FastDiv;
using sm100::make_fast_div;

constexpr int kThreads = 256, kMaxTurns = 2048, kUnrollMost = 4;
// Blocks on an SM, which are all that are launched, and tokens of a thread under way at once; us forward / backward on 16 x 96 x 96 tokens, 6 heads.  Words of 8 channels, heads of 32: 54 / 83 (592 blocks in two
// rounds 61 / 84; two blocks and four tokens forward 60; three blocks backward, whose registers spill, 133).  Words of 4, heads of 24: 58 / 85 (words of 2 there 108 / 149; four tokens forward 67; three blocks and
// two tokens backward 96).  Words of 2, heads of 20: 97 / 142 (six blocks, whose registers spill, 135 / 220; two tokens 125 / 190).  Words of 1, heads of 30: 181 / 282.  All of these are turned as a whole;
// half of heads of 32 56 / 83, 16 of heads of 24 54 / 79, 12 of heads of 20 106 / 151.
constexpr int blocks_of(int V, bool backward) { return V == 8 ? (backward ? 2 : 3) : V == 4 && backward ? 2 : 4; }
constexpr int unroll_of(int V, bool backward) { return V == 8 || (V == 4 && !backward) ? 2 : 4; }

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
    int tokens, tile, tiles, H, W, d, rot, pairs, per_head, lanes, rows, rows_per_chunk, tokens_at_once;      // rows: heads of q, then of k; blockIdx.y: a chunk of them
    float eps, inverse_d;
    FastDiv by_pixels, by_w, by_pairs, by_slots;
};

template <int V> struct Word;
template <> struct Word<8> { using type = uint4; };
template <> struct Word<4> { using type = uint2; };
template <> struct Word<2> { using type = uint32_t; };
template <> struct Word<1> { using type = unsigned short; };

// A unit's V pairs as two vectors, the pairs' first and second channels, two by two for the packed instructions (V = 1: the second of two is 0).  Halves: the two runs as they lie; interleaved: the
// low and the high half of every word, of both runs.  (V = 1 looks the same either way.)
template <int V> struct Pairs { float2 a[(V + 1) / 2], b[(V + 1) / 2]; };
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
template <int V, bool kInterleaved> __device__ __forceinline__ Pairs<V> unpack(const typename Word<V>::type& wa, const typename Word<V>::type& wb)
{
    Pairs<V> x;
    if constexpr (V == 1) {
        x.a[0] = make_float2(low(wa), 0.f);
        x.b[0] = make_float2(low(wb), 0.f);
    } else {
        const uint32_t *p = reinterpret_cast<const uint32_t*>(&wa), *q = reinterpret_cast<const uint32_t*>(&wb);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if constexpr (kInterleaved) {
                const uint32_t u = 2 * i < V / 2 ? p[(2 * i) % (V / 2)] : q[(2 * i) % (V / 2)], v = 2 * i + 1 < V / 2 ? p[(2 * i + 1) % (V / 2)] : q[(2 * i + 1) % (V / 2)];
                x.a[i] = make_float2(low(u), low(v));
                x.b[i] = make_float2(high(u), high(v));
            } else {
                x.a[i] = make_float2(low(p[i]), high(p[i]));
                x.b[i] = make_float2(low(q[i]), high(q[i]));
            }
        }
    }
    return x;
}
template <int V, bool kInterleaved> __device__ __forceinline__ void pack(const Pairs<V>& x, typename Word<V>::type& wa, typename Word<V>::type& wb)
{
    if constexpr (V == 1) {
        wa = __bfloat16_as_ushort(__float2bfloat16_rn(x.a[0].x));
        wb = __bfloat16_as_ushort(__float2bfloat16_rn(x.b[0].x));
    } else {
        uint32_t *p = reinterpret_cast<uint32_t*>(&wa), *q = reinterpret_cast<uint32_t*>(&wb);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if constexpr (kInterleaved) {
                const uint32_t u = sm100::pack_bf16x2(x.a[i].x, x.b[i].x), v = sm100::pack_bf16x2(x.a[i].y, x.b[i].y);
                if (2 * i < V / 2) p[(2 * i) % (V / 2)] = u; else q[(2 * i) % (V / 2)] = u;
                if (2 * i + 1 < V / 2) p[(2 * i + 1) % (V / 2)] = v; else q[(2 * i + 1) % (V / 2)] = v;
            } else {
                p[i] = sm100::pack_bf16x2(x.a[i].x, x.a[i].y);
                q[i] = sm100::pack_bf16x2(x.b[i].x, x.b[i].y);
            }
        }
    }
}
__device__ __forceinline__ float2 twice(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 negated(float2 x) { return make_float2(-x.x, -x.y); }
// x = c x + t where the unit is turned; where it is not, x stays as it is, whatever t holds: the zeros of such a unit times an infinite neighbour are NaN.  (Predicated: no instruction more.)
template <bool kWhole> __device__ __forceinline__ void turn(float2& x, float2 c, float2 t, bool turned)
{
    if constexpr (kWhole) { x = __ffma2_rn(c, x, t); return; }
    asm("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %3, 0;\n\t@p fma.rn.f32x2 %0, %1, %0, %2;\n\t}"
        : "+l"(reinterpret_cast<unsigned long long&>(x)) : "l"(reinterpret_cast<const unsigned long long&>(c)), "l"(reinterpret_cast<const unsigned long long&>(t)), "r"((int)turned));
}

// kWhole: every channel is turned (rot = d); units that are not are lanes without channels.
template <int V, bool kInterleaved, bool kBackward, bool kWhole>
__global__ void __launch_bounds__(kThreads, blocks_of(V, kBackward)) rib_qk_norm_rope_kernel(const __grid_constant__ RopeParams p)
{
    constexpr int kUnroll = unroll_of(V, kBackward), kTwos = (V + 1) / 2, kFill = V == 8 && !kBackward ? 3 : 1;      // kFill: entries of the tile's cosines and sines that a thread has under way
    constexpr bool kOddPairs = kInterleaved && V == 1;           // a pair's channels are neighbours, and not in one word
    using W = typename Word<V>::type;
    extern __shared__ __align__(16) float turns[];               // [tile][pairs] cosines, then sines; backward, at the end: [threads][2 V] sums
    // this thread: unit of a row of the chunk, and which of the tokens that are walked at once
    int at_once, slot;
    p.by_slots.divmod(threadIdx.x, at_once, slot);               // slots: rows of a chunk x lanes of a row
    const bool spare = at_once >= p.tokens_at_once;               // (threads that are left over go along with the first token's)
    if (spare) at_once = 0;
    const int unit = slot & (p.lanes - 1), chunk_row = slot / p.lanes, row = blockIdx.y * p.rows_per_chunk + chunk_row;
    const bool works = !spare && row < p.rows;
    const bool is_k = row >= p.t[0].heads;
    const RopeTensor& t = p.t[is_k ? 1 : 0];
    const int head = is_k ? row - p.t[0].heads : row;
    // channels of the unit's two runs; beyond d: none
    const int turned = p.pairs / V;
    const bool rotates = unit < turned;
    int ca, cb;
    if (rotates) { ca = kOddPairs ? 2 * unit : V * unit; cb = kOddPairs ? ca + 1 : ca + p.rot / 2; }
    else { ca = p.rot + 2 * V * (unit - turned); cb = ca + V; }
    const bool has_a = works && ca < p.d, has_b = works && cb < p.d;
    const bool norm = works && t.w != nullptr;
    cudaGridDependencySynchronize();                             // it may have overtaken the kernel before
    // place of a pair's two channels among the unit's 2 V
    auto place_a = [](int i) { return kInterleaved && V > 1 ? 2 * i : i; };
    auto place_b = [](int i) { return kInterleaved && V > 1 ? 2 * i + 1 : V + i; };
    Pairs<V> w, dw;
    {
        const float* src = t.w + (p.per_head ? head * p.d : 0);
        auto weight = [&](int place) { return norm && (place < V ? has_a : has_b) ? src[place < V ? ca + place : cb + place - V] : 1.f; };
#pragma unroll
        for (int i = 0; i < kTwos; ++i) {
            w.a[i] = make_float2(weight(place_a(2 * i)), V > 1 ? weight(place_a(2 * i + 1)) : 0.f);
            w.b[i] = make_float2(weight(place_b(2 * i)), V > 1 ? weight(place_b(2 * i + 1)) : 0.f);
            dw.a[i] = dw.b[i] = make_float2(0.f, 0.f);
        }
    }
    const __nv_bfloat16 *x_at = t.x + head * p.d, *g_at = kBackward ? t.g + head * p.d : nullptr;
    __nv_bfloat16* y_at = t.y + head * p.d;
    const long long x_stride = t.x_stride, y_stride = t.y_stride;
    const int g_stride = t.heads * p.d;
    // Where the cosines of the unit's pairs lie - V that follow one another, or (interleaved) V / 2 of each run, `second` apart -, and the sines, and how far from a token to the next one.  Units that are not turned have
    // ones and zeros of their own, so that all threads go the same way.
    constexpr bool kTwoRuns = kInterleaved && V > 1;
    const int second = kTwoRuns ? p.rot / 4 : V / 2, span = kTwoRuns ? p.rot / 4 + V / 2 : V;
    float* const unturned = turns + 2 * p.tile * p.pairs;
    const float* const cosines = rotates ? turns + (kTwoRuns ? V / 2 * unit : V * unit) : unturned;
    const int to_sines = rotates ? p.tile * p.pairs : span, turns_step = rotates ? p.pairs : 0;
    for (int i = threadIdx.x; i < 2 * span; i += kThreads) unturned[i] = i < span ? 1.f : 0.f;
    if (!p.rot) __syncthreads();                                 // (else behind the first tile's cosines and sines)

    // (what is not there is not loaded, and stays the zero that it is here, or a token's of before, whose results are not kept)
    W xa[kUnroll], xb[kUnroll], ga[kUnroll], gb[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) { xa[k] = W{}; xb[k] = W{}; ga[k] = W{}; gb[k] = W{}; }

    for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
        const int token0 = tile * p.tile, here = min(p.tile, p.tokens - token0);
        auto load = [&](int k0) {
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                const int token = k0 + k * p.tokens_at_once + at_once;
                const bool there = token < here;
                const __nv_bfloat16* src = x_at + (token0 + token) * x_stride;
                const bool needed = !kBackward || norm;          // (the gradient of a row without a norm does not depend on it)
                if (there && needed && has_a) xa[k] = *reinterpret_cast<const W*>(src + ca);
                if (there && needed && has_b) xb[k] = *reinterpret_cast<const W*>(src + cb);
                if constexpr (kBackward) {
                    const __nv_bfloat16* grad = g_at + (long long)(token0 + token) * g_stride;
                    if (there && has_a) ga[k] = *reinterpret_cast<const W*>(grad + ca);
                    if (there && has_b) gb[k] = *reinterpret_cast<const W*>(grad + cb);
                }
            }
        };
        load(0);
        if (p.rot) {                                             // (under the loads)
            __syncthreads();                                     // the tile before has been used
#pragma unroll kFill
            for (int e = threadIdx.x; e < here * p.pairs; e += kThreads) {
                int token, i, image, pixel, y, x;
                p.by_pairs.divmod(e, token, i);
                p.by_pixels.divmod(token0 + token, image, pixel);
                p.by_w.divmod(pixel, y, x);
                const float2 a = p.table[(long long)y * p.pairs + i], b = p.table[(long long)(p.H + x) * p.pairs + i];
                turns[e] = a.x * b.x - a.y * b.y;
                turns[p.tile * p.pairs + e] = a.y * b.x + a.x * b.y;
            }
            __syncthreads();
        }
        // (all lanes walk alike: those of a row meet in shuffles)
        for (int k0 = 0; k0 < here; k0 += kUnroll * p.tokens_at_once) {
            if (k0) load(k0);
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                if (k0 + k * p.tokens_at_once >= here) break;    // (the same for all threads)
                const int token = k0 + k * p.tokens_at_once + at_once;
                const bool there = token < here;
                float2 c[kTwos], s[kTwos];
                const float *cp = cosines + token * turns_step, *sp = cp + to_sines;
                if constexpr (V == 8) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float4 u = *reinterpret_cast<const float4*>(cp + i * second), v = *reinterpret_cast<const float4*>(sp + i * second);
                        c[2 * i] = make_float2(u.x, u.y); c[2 * i + 1] = make_float2(u.z, u.w);
                        s[2 * i] = make_float2(v.x, v.y); s[2 * i + 1] = make_float2(v.z, v.w);
                    }
                } else if constexpr (V == 4) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) { c[i] = *reinterpret_cast<const float2*>(cp + i * second); s[i] = *reinterpret_cast<const float2*>(sp + i * second); }
                } else {
                    c[0] = make_float2(cp[0], V > 1 ? cp[second] : 0.f);
                    s[0] = make_float2(sp[0], V > 1 ? sp[second] : 0.f);
                }
                const Pairs<V> x = unpack<V, kInterleaved>(xa[k], xb[k]);
                Pairs<V> z;
                float2 squares = twice(0.f), along = twice(0.f);
#pragma unroll
                for (int i = 0; i < kTwos; ++i) squares = __ffma2_rn(x.b[i], x.b[i], __ffma2_rn(x.a[i], x.a[i], squares));
                if constexpr (kBackward) {
                    const Pairs<V> g = unpack<V, kInterleaved>(ga[k], gb[k]);
#pragma unroll
                    for (int i = 0; i < kTwos; ++i) {            // back by the transposed rotation
                        z.a[i] = g.a[i]; z.b[i] = g.b[i];
                        turn<kWhole>(z.a[i], c[i], __fmul2_rn(s[i], g.b[i]), rotates);
                        turn<kWhole>(z.b[i], c[i], __fmul2_rn(negated(s[i]), g.a[i]), rotates);
                        along = __ffma2_rn(__fmul2_rn(z.b[i], w.b[i]), x.b[i], __ffma2_rn(__fmul2_rn(z.a[i], w.a[i]), x.a[i], along));
                    }
                }
                float of_squares = squares.x + squares.y, of_along = along.x + along.y;
                for (int o = p.lanes / 2; o; o >>= 1) {          // (rows without a norm beside rows with one: all take part)
                    of_squares += __shfl_xor_sync(0xffffffffu, of_squares, o);
                    if constexpr (kBackward) of_along += __shfl_xor_sync(0xffffffffu, of_along, o);
                }
                const float inverse = norm ? rsqrtf(fmaf(of_squares, p.inverse_d, p.eps)) : 1.f;
                const float2 inverse2 = twice(inverse);
                if constexpr (kBackward) {
                    const float2 mean = twice(norm ? -of_along * inverse * p.inverse_d : 0.f);       // - mean_c(w gz xhat)
#pragma unroll
                    for (int i = 0; i < kTwos; ++i) {
                        const float2 ua = __fmul2_rn(x.a[i], inverse2), ub = __fmul2_rn(x.b[i], inverse2);
                        if (there) { dw.a[i] = __ffma2_rn(z.a[i], ua, dw.a[i]); dw.b[i] = __ffma2_rn(z.b[i], ub, dw.b[i]); }
                        z.a[i] = __fmul2_rn(inverse2, __ffma2_rn(ua, mean, __fmul2_rn(z.a[i], w.a[i])));
                        z.b[i] = __fmul2_rn(inverse2, __ffma2_rn(ub, mean, __fmul2_rn(z.b[i], w.b[i])));
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < kTwos; ++i) {
                        z.a[i] = __fmul2_rn(__fmul2_rn(x.a[i], inverse2), w.a[i]); z.b[i] = __fmul2_rn(__fmul2_rn(x.b[i], inverse2), w.b[i]);
                        const float2 ta = __fmul2_rn(negated(s[i]), z.b[i]), tb = __fmul2_rn(s[i], z.a[i]);
                        turn<kWhole>(z.a[i], c[i], ta, rotates);
                        turn<kWhole>(z.b[i], c[i], tb, rotates);
                    }
                }
                if (there) {
                    W ya, yb;
                    if (!kWhole && !kBackward && !norm && !rotates) { ya = xa[k]; yb = xb[k]; }      // (as it was, NaN and all)
                    else pack<V, kInterleaved>(z, ya, yb);
                    __nv_bfloat16* dst = y_at + (token0 + token) * y_stride;
                    if (has_a) *reinterpret_cast<W*>(dst + ca) = ya;
                    if (has_b) *reinterpret_cast<W*>(dst + cb) = yb;
                }
            }
        }
    }
    if constexpr (kBackward) {
        if (!p.part) return;
        // Sums of the block in a fixed order: of a row's channel over the tokens at once, or of a tensor's over its rows of the chunk too.
        float* const sums = turns;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) {
            sums[threadIdx.x * 2 * V + place_a(i)] = i & 1 ? dw.a[i >> 1].y : dw.a[i >> 1].x;
            sums[threadIdx.x * 2 * V + place_b(i)] = i & 1 ? dw.b[i >> 1].y : dw.b[i >> 1].x;
        }
        __syncthreads();
        const int slots = p.rows_per_chunk * p.lanes, outputs = p.per_head ? p.rows_per_chunk : 2;
        float* const dst = p.part + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * outputs * p.d;
        for (int e = threadIdx.x; e < outputs * p.d; e += kThreads) {
            const int which = e / p.d, ch = e - which * p.d;
            // the unit and place of the channel
            int u, place;
            if (ch < p.rot) {
                const int half = p.rot / 2;
                if (kOddPairs) { u = ch / 2; place = ch & 1; }
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
__global__ void __launch_bounds__(256) rib_qk_norm_rope_sum_kernel(const RopeSum t)
{
    __shared__ float sums[256];
    // a block has eight channels, 32 threads to each, of a row, whose sums are in one chunk, or of a tensor, in all of them
    const int eights = (t.d + 7) / 8, which = blockIdx.x / eights, c = 8 * (blockIdx.x % eights) + (threadIdx.x & 7), run = threadIdx.x >> 3;
    const int chunk = t.per_head ? which / t.rows_per_chunk : 0, output = t.per_head ? which % t.rows_per_chunk : which, chunks = t.per_head ? 1 : t.chunks;
    const bool is_k = t.per_head ? which >= t.heads : which == 1;
    float* const dst = t.dw[is_k ? 1 : 0];
    cudaGridDependencySynchronize();                             // it may have overtaken the kernel before
    if (!dst) return;
    float total = 0.f;
    if (c < t.d) {
#pragma unroll 8
        for (int i = run; i < chunks * t.blocks; i += 32) total += t.part[((long long)chunk * t.blocks + i) * t.outputs * t.d + output * t.d + c];
    }
    sums[threadIdx.x] = total;
    __syncthreads();
    if (threadIdx.x < 8 && c < t.d) {
#pragma unroll
        for (int i = 1; i < 32; ++i) total += sums[8 * i + threadIdx.x];
        dst[(t.per_head ? which - (is_k ? t.heads : 0) : 0) * t.d + c] = total;
    }
}

// Angles are products of whole numbers (42 bits) and 32-bit frequencies (24 bits): the product in 64 bits (53), and beyond 2^29 what it leaves, exactly; their cosine and sine are rounded once.
__global__ void __launch_bounds__(128) rib_rope_table_kernel(const float* frequencies, int H, int W, int pairs, long long y0, long long x0, float magnitude, float2* table)
{
    const long long e = (long long)blockIdx.x * 128 + threadIdx.x;
    if (e >= ((long long)H + W) * pairs) return;
    const long long row = e / pairs;
    const int i = (int)(e - row * pairs);
    const bool column = row >= H;
    cudaGridDependencySynchronize();                             // it may have overtaken the kernel before
    const double position = (double)(column ? x0 + row - H : y0 + row), frequency = (double)frequencies[column ? pairs + i : i], angle = position * frequency;
    double sine, cosine;
    sincos(angle, &sine, &cosine);
    if (fabs(position) > 0x1p29) {
        double sine_left, cosine_left;
        sincos(fma(position, frequency, -angle), &sine_left, &cosine_left);
        const double s = sine;
        sine = s * cosine_left + cosine * sine_left;
        cosine = cosine * cosine_left - s * sine_left;
    }
    const double scale = column ? 1.0 : (double)magnitude;
    table[e] = make_float2((float)(scale * cosine), (float)(scale * sine));
}

struct Plan { int V, lanes, rows, rows_per_chunk, chunks, tokens_at_once, tile, tiles, blocks; };

int lanes_of(int units) { int l = 1; while (l < units) l *= 2; return l; }

// rows of a chunk and blocks along the tokens, for rows of `lanes` lanes
void rope_grid(const RopeProblem& p, int lanes, int blocks, Plan* plan)
{
    plan->lanes = lanes;
    plan->rows = p.heads + p.kv_heads;
    const int most = kThreads / lanes;
    plan->chunks = (plan->rows + most - 1) / most;
    plan->rows_per_chunk = (plan->rows + plan->chunks - 1) / plan->chunks;
    plan->chunks = (plan->rows + plan->rows_per_chunk - 1) / plan->rows_per_chunk;
    plan->tokens_at_once = kThreads / (plan->rows_per_chunk * lanes);
    // a tile is what a block has under way at once, as far as its cosines and sines have room, and such that a small map still gives every SM two tiles
    long long tile = p.tokens / (2 * 148), most_tokens = kUnrollMost * plan->tokens_at_once;
    if (tile > most_tokens) tile = most_tokens;
    if (tile > kMaxTurns / (p.rot > 2 ? p.rot / 2 : 1)) tile = kMaxTurns / (p.rot > 2 ? p.rot / 2 : 1);
    tile = tile < plan->tokens_at_once ? plan->tokens_at_once : tile / plan->tokens_at_once * plan->tokens_at_once;
    plan->tile = (int)tile;
    plan->tiles = (int)((p.tokens + tile - 1) / tile);
    const int cap = (148 * blocks + plan->chunks - 1) / plan->chunks;
    plan->blocks = plan->tiles < cap ? plan->tiles : cap;
}

// the widest words that every row allows
Plan rope_plan(const RopeProblem& p, bool backward)
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
    plan.V = fits(8) ? 8 : fits(4) ? 4 : fits(2) ? 2 : 1;
    rope_grid(p, lanes_of(p.rot / (2 * plan.V) + (p.d - p.rot + 2 * plan.V - 1) / (2 * plan.V)), blocks_of(plan.V, backward), &plan);
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
    a.pairs = p.rot / 2; a.per_head = p.per_head; a.lanes = plan.lanes; a.rows = plan.rows; a.rows_per_chunk = plan.rows_per_chunk;
    a.tokens_at_once = plan.tokens_at_once; a.eps = p.eps; a.inverse_d = 1.f / (float)p.d;
    a.by_pixels = make_fast_div((int)((long long)p.H * p.W)); a.by_w = make_fast_div(p.W); a.by_pairs = make_fast_div(p.rot ? p.rot / 2 : 1);
    a.by_slots = make_fast_div(plan.rows_per_chunk * plan.lanes);
    const dim3 grid((unsigned)plan.blocks, (unsigned)plan.chunks);
    size_t smem = sizeof(float2) * (plan.tile * a.pairs + p.rot / 4 + plan.V);           // up to 16 KB, or 256 tokens of one row's pairs
    if (kBackward && part && smem < sizeof(float) * kThreads * 2 * plan.V) smem = sizeof(float) * kThreads * 2 * plan.V;
    ProfileScope scope(kBackward ? RIB_KERNEL_QK_NORM_ROPE_BWD : RIB_KERNEL_QK_NORM_ROPE_FWD, stream);
    const auto kernel_of = [&](auto whole) {
        constexpr bool kWhole = decltype(whole)::value;
        return plan.V == 8 ? (p.interleaved ? rib_qk_norm_rope_kernel<8, true, kBackward, kWhole> : rib_qk_norm_rope_kernel<8, false, kBackward, kWhole>)
             : plan.V == 4 ? (p.interleaved ? rib_qk_norm_rope_kernel<4, true, kBackward, kWhole> : rib_qk_norm_rope_kernel<4, false, kBackward, kWhole>)
             : plan.V == 2 ? (p.interleaved ? rib_qk_norm_rope_kernel<2, true, kBackward, kWhole> : rib_qk_norm_rope_kernel<2, false, kBackward, kWhole>)
                           : (p.interleaved ? rib_qk_norm_rope_kernel<1, true, kBackward, kWhole> : rib_qk_norm_rope_kernel<1, false, kBackward, kWhole>);
    };
    const auto kernel = p.rot == p.d ? kernel_of(std::true_type{}) : kernel_of(std::false_type{});
    return launch_overtaking(kernel, grid, kThreads, smem, stream, a);
}

}  // namespace

cudaError_t rope_table(const float* frequencies, int H, int W, int pairs, long long y0, long long x0, float magnitude, float* table, cudaStream_t stream)
{
    const long long entries = ((long long)H + W) * pairs;
    ProfileScope scope(RIB_KERNEL_ROPE_TABLE, stream);
    return launch_overtaking(rib_rope_table_kernel, (unsigned)((entries + 127) / 128), 128, 0, stream, frequencies, H, W, pairs, y0, x0, magnitude, reinterpret_cast<float2*>(table));
}

cudaError_t qk_norm_rope_fwd(const RopeProblem& p, cudaStream_t stream) { return launch<false>(p, nullptr, rope_plan(p, false), stream); }

constexpr int kMostBlocks = 4;
// room for the sums of any alignment (a row has 1 to 32 lanes)
size_t qk_norm_rope_bwd_workspace(const RopeProblem& p)
{
    size_t most = 0;
    for (int lanes = 1; lanes <= 32; lanes *= 2) {
        Plan plan{};
        rope_grid(p, lanes, kMostBlocks, &plan);
        // (the tiles' size depends on `rot` too; they are no smaller than the tokens that are walked at once)
        const long long tiles = (p.tokens + plan.tokens_at_once - 1) / plan.tokens_at_once, cap = (148 * kMostBlocks + plan.chunks - 1) / plan.chunks;
        plan.blocks = (int)(tiles < cap ? tiles : cap);
        const size_t bytes = sizeof(float) * part_floats(plan, p.d, p.per_head != 0);
        most = bytes > most ? bytes : most;
    }
    return (most + 255) & ~(size_t)255;
}

cudaError_t qk_norm_rope_bwd(const RopeProblem& p, float* workspace, int* launches, cudaStream_t stream)
{
    const Plan plan = rope_plan(p, true);
    const bool weights = p.t[0].dw || p.t[1].dw;
    *launches = 1;
    if (cudaError_t e = launch<true>(p, weights ? workspace : nullptr, plan, stream)) return e;
    if (!weights) return cudaSuccess;
    const RopeSum s{workspace, {p.t[0].dw, p.t[1].dw}, p.d, plan.blocks, plan.chunks, p.per_head ? plan.rows_per_chunk : 2, p.per_head, plan.rows_per_chunk, p.heads, plan.rows};
    *launches = 2;
    ProfileScope scope(RIB_KERNEL_QK_NORM_ROPE_SUM, stream);
    return launch_overtaking(rib_qk_norm_rope_sum_kernel, (p.per_head ? plan.rows : 2) * ((p.d + 7) / 8), 256, 0, stream, s);
}

}  // namespace rib
