// Window attention with a bias by buckets in windows of up to 256 tokens whose shape the tcgen05 kernels do not take: odd windows, head widths and
// shifts.  A row of such a window begins anywhere (7 tokens of 20 channels: 40 bytes each), so its tiles cannot be boxes of a tensor map, and a
// window of 49 tokens would fill a third of an M = 128 tile; so a block has one window of one head at a time, its rows as bf16 in shared memory, and
// warp-level MMAs (m16n8k16) with a tile of 16 rows to a warp.
//     forward    a warp has 16 queries:  S = Q K^T over 64 keys at a time, running maximum and sum, O += P V
//     backward   a warp has 16 keys:     S^T = K Q^T, dP^T = V dO^T over 16 queries at a time, P^T = exp2(S^T + b - lse), dS^T = P^T o (dP^T - D),
//                dV += P^T dO, dK += dS^T Q;  dS^T of 64 queries goes to shared memory, and the warps share out dQ = dS K among them
// P and dS are rounded to bf16 for the contractions, as in the tcgen05 kernels; scores, sums, lse, D and the sums of the bias gradient are fp32
// (dS is added to its offset's sum before it is rounded).  A block walks a run of windows, head by head: the biases by offset are gathered to shared
// memory and their gradient leaves it once per head, not per window.
//
// What bounds it is instructions: staging, and a table entry, an exponential and (backward) an addition in shared memory for every score.
// 2 x 50 x 39 tokens, 3 heads of 20, windows of 7, forward and backward: 29 us; with a row of the window to a thread, on the plain pipes, it was 62
// (and 1030 -> 254 us for the backward pass alone of 8 x 96 x 96 tokens, 6 heads, where that form waited for 16-byte reads of shared memory that serve
// four products each).
#include "rib_sm100_common.cuh"

namespace rib {
namespace {

using namespace sm100;

constexpr int kMaxTokens = 256;
constexpr int kQueryBlock = 64, kDSPitch = kQueryBlock + 8;       // of dS^T in shared memory, bf16 (rows 144 bytes apart: eight of them in different banks)
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;
constexpr size_t kMostShared = 232448;                             // of a block
constexpr int kNoPart = 0x7fff;                                   // part of a place without a token

__device__ __forceinline__ void ldmatrix_x4(const __nv_bfloat16* at, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_u32(at)) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(const __nv_bfloat16* at, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_u32(at)) : "memory");
}
// d (16 x 8) += a (16 x 16) b (16 x 8)
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Rows of 16 kD channels in shared memory; 16 bytes behind each put the eight rows of an 8 x 8 matrix into different banks.
template <int kD> constexpr int kPitch = 16 * kD + 8;
__host__ __device__ inline int rows_of(int n) { return (n + 15) & ~15; }
__host__ __device__ inline size_t table_floats(int M) { return (size_t)((2 * M - 1) * (2 * M - 1) + 3) & ~(size_t)3; }
size_t shared_bytes(int n, int d, int M, bool backward)
{
    const size_t rows = rows_of(n), pitch = (d + 15) / 16 * 16 + 8;
    return (backward ? 4 : 3) * rows * pitch * 2 + (backward ? rows * kDSPitch * 2 : 0) + (backward ? 2 : 1) * table_floats(M) * 4 + (backward ? 5 : 3) * rows * 4;
}

// The lane's part of what an x4 load names, for a tile of 16 rows x 16 columns: matrices as the A operand has them (rows, then columns 8 ..), and as
// two B operands side by side have them (columns 8 .., then rows).
__device__ __forceinline__ int a_row(int lane) { return (lane & 7) + ((lane >> 3) & 1) * 8; }
__device__ __forceinline__ int a_col(int lane) { return (lane >> 4) * 8; }
__device__ __forceinline__ int b_row(int lane) { return (lane & 7) + (lane >> 4) * 8; }
__device__ __forceinline__ int b_col(int lane) { return ((lane >> 3) & 1) * 8; }

struct Block { int h, b, wy, wx; };
// Window `index` of p.pairs, heads outermost.
__device__ __forceinline__ Block decode_window(const Problem& p, int per_head, int index)
{
    Block w;
    w.h = index / per_head;
    int rest = index - w.h * per_head;
    w.b = rest / (p.nWy * p.nWx);
    rest -= w.b * (p.nWy * p.nWx);
    w.wy = rest / p.nWx;
    w.wx = rest - w.wy * p.nWx;
    return w;
}

// Shared memory of a block beside its rows.  place[i] = entry y side + x of window position i in the table by offset, its part of the window above
// it (kNoPart: no token), pixel[i] = its pixel in the map or -1.
struct Places { long long* pixel; int* place; };
__device__ inline void find_places(const Problem& p, const Block& w, int rows, const Places& s)
{
    for (int i = threadIdx.x; i < rows; i += blockDim.x) {
        long long pixel = -1;
        int place = kNoPart << 16;
        if (i < p.n) {
            int Y, X;
            token_pixel(p.Hp, p.Wp, p.M, p.s, w.wy, w.wx, i, Y, X);
            const int y = i / p.M, x = i - y * p.M;
            if (Y < p.H && X < p.W) {
                pixel = (long long)Y * p.W + X;
                place = y * (2 * p.M - 1) + x | (p.masked ? window_part(p.M, p.s, w.wy == p.nWy - 1, w.wx == p.nWx - 1, y, x) << 16 : 0);
            }
        }
        s.pixel[i] = pixel;
        s.place[i] = place;
    }
}
__device__ inline void gather_table(const Problem& p, int h, float* table)
{
    const int side = 2 * p.M - 1;
    for (int e = threadIdx.x; e < side * side; e += blockDim.x) {
        const int u = __ldg(p.buckets + e);
        table[e] = (unsigned)u < (unsigned)p.num_buckets ? bias_at(p.bias, p.bias_bf16, (long long)h * p.bias_head_stride + u) * kLog2e : -INFINITY;
    }
}
// The window's rows of several tensors, T at a time (the largest power of two of bytes that rows begin on); zeros where no token is.  What lies behind
// the last channel and the last row is not touched.
template <int kCount> struct Staged { const __nv_bfloat16* from[kCount]; __nv_bfloat16* to[kCount]; };
template <int kP, typename T, int kCount>
__device__ __forceinline__ void stage_as(const Problem& p, const FastDiv& by_words, const Block& w, const long long* pixel, const Staged<kCount>& x)
{
    constexpr int kPer = sizeof(T) / 2;
    const size_t origin = ((size_t)w.b * p.H * p.W * p.heads + w.h) * p.d, step = (size_t)p.heads * p.d;
    const int words = (int)by_words.d;
#pragma unroll 2
    for (int e = threadIdx.x; e < p.n * words; e += blockDim.x) {
        int row, c;
        by_words.divmod(e, row, c);
        const long long px = pixel[row];
        const size_t at = origin + px * step + c * kPer;
        T v[kCount];
#pragma unroll
        for (int k = 0; k < kCount; ++k) {
            v[k] = T{};
            if (px >= 0) v[k] = __ldg(reinterpret_cast<const T*>(x.from[k] + at));
        }
#pragma unroll
        for (int k = 0; k < kCount; ++k) *reinterpret_cast<T*>(x.to[k] + row * kP + c * kPer) = v[k];
    }
}
__host__ __device__ inline int elements_of_word(int d) { return d % 8 == 0 ? 8 : d % 4 == 0 ? 4 : d % 2 == 0 ? 2 : 1; }
template <int kP, int kCount>
__device__ __forceinline__ void stage(const Problem& p, const FastDiv& by_words, const Block& w, const long long* pixel, const Staged<kCount>& x)
{
    switch (elements_of_word(p.d)) {
    case 8: stage_as<kP, uint4>(p, by_words, w, pixel, x); break;
    case 4: stage_as<kP, uint2>(p, by_words, w, pixel, x); break;
    case 2: stage_as<kP, uint32_t>(p, by_words, w, pixel, x); break;
    default: stage_as<kP, uint16_t>(p, by_words, w, pixel, x); break;
    }
}
// two neighbouring channels c, c + 1 of a row
__device__ __forceinline__ void store_pair(const Problem& p, __nv_bfloat16* row, int c, float a, float b)
{
    if (c >= p.d) return;
    if (p.d % 2 == 0) {
        *reinterpret_cast<uint32_t*>(row + c) = pack_bf16x2(a, b);
    } else {
        row[c] = __float2bfloat16_rn(a);
        if (c + 1 < p.d) row[c + 1] = __float2bfloat16_rn(b);
    }
}
__device__ __forceinline__ __nv_bfloat16* row_at(const Problem& p, const Block& w, __nv_bfloat16* x, long long pixel)
{
    return x + (((size_t)w.b * p.H * p.W + pixel) * p.heads + w.h) * p.d;
}
__device__ __forceinline__ size_t scalar_at(const Problem& p, const Block& w, long long pixel) { return ((size_t)w.b * p.heads + w.h) * p.H * p.W + pixel; }

// zeros behind the last channel of the rows and behind the last row, which stay
__device__ inline void clear_rows(__nv_bfloat16* rows, int elements)
{
    for (int e = 8 * threadIdx.x; e < elements; e += 8 * blockDim.x) *reinterpret_cast<uint4*>(rows + e) = make_uint4(0u, 0u, 0u, 0u);
}

template <int kD>
__global__ void __launch_bounds__(2 * kMaxTokens) rib_bias_small_fwd_kernel(const Problem p, const FastDiv by_words)
{
    extern __shared__ __align__(16) uint8_t sm[];
    constexpr int kP = kPitch<kD>;
    const int rows = rows_of(p.n), side = 2 * p.M - 1, lane = threadIdx.x & 31, tile = (threadIdx.x >> 5) * 16, c2 = 2 * (lane & 3);
    __nv_bfloat16 *const qs = reinterpret_cast<__nv_bfloat16*>(sm), *const ks = qs + rows * kP, *const vs = ks + rows * kP;
    float* const table = reinterpret_cast<float*>(vs + rows * kP);
    long long* const pixels = reinterpret_cast<long long*>(table + table_floats(p.M));
    const Places s{pixels, reinterpret_cast<int*>(pixels + rows)};
    const int per_head = p.pairs / p.heads;
    const int first = (int)((long long)p.pairs * blockIdx.x / gridDim.x), last = (int)((long long)p.pairs * (blockIdx.x + 1) / gridDim.x);
    const float scale = rsqrtf((float)p.d) * kLog2e;
    const Staged<3> staged{{p.q, p.k, p.v}, {qs, ks, vs}};
    clear_rows(qs, 3 * rows * kP);
    int head = -1;
    for (int index = first; index < last; ++index) {
        const Block w = decode_window(p, per_head, index);
        __syncthreads();
        if (w.h != head) { gather_table(p, w.h, table); head = w.h; }
        find_places(p, w, rows, s);
        __syncthreads();
        stage<kP>(p, by_words, w, s.pixel, staged);
        __syncthreads();
        uint32_t qf[kD][4];
#pragma unroll
        for (int k = 0; k < kD; ++k) ldmatrix_x4(qs + (tile + a_row(lane)) * kP + 16 * k + a_col(lane), qf[k]);
        // a thread has rows lane / 4 and 8 more of the tile, and of every 8 keys two
        const int r0 = tile + (lane >> 2);
        const int place0 = s.place[r0], place1 = s.place[r0 + 8], part0 = place0 >> 16, part1 = place1 >> 16;
        const float *const bias0 = table + (p.M - 1) * (side + 1) - (place0 & 0xffff), *const bias1 = table + (p.M - 1) * (side + 1) - (place1 & 0xffff);
        float o[2 * kD][4], m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int g = 0; g < 2 * kD; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[g][e] = 0.f;
        for (int key = 0; key < rows; key += 64) {
            float x[8][4];
            float most0 = m0, most1 = m1;
#pragma unroll
            for (int sub = 0; sub < 4; ++sub) {
                if (key + 16 * sub >= rows) break;
                float (&a)[4] = x[2 * sub], (&b)[4] = x[2 * sub + 1];
#pragma unroll
                for (int e = 0; e < 4; ++e) a[e] = b[e] = 0.f;
#pragma unroll
                for (int k = 0; k < kD; ++k) {
                    uint32_t f[4];
                    ldmatrix_x4(ks + (key + 16 * sub + b_row(lane)) * kP + 16 * k + b_col(lane), f);
                    mma_16816(a, qf[k], f[0], f[1]);
                    mma_16816(b, qf[k], f[2], f[3]);
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int2 keys = *reinterpret_cast<const int2*>(s.place + key + 16 * sub + 8 * t + c2);
                    float (&y)[4] = x[2 * sub + t];
                    const int ex = keys.x & 0xffff, ey = keys.y & 0xffff, px = keys.x >> 16, py = keys.y >> 16;
                    // (a key that is not attended to counts as such whatever its own row holds)
                    auto score = [&](float y, bool same, float b) { return same && b != -INFINITY ? fmaf(y, scale, b) : -INFINITY; };
                    y[0] = score(y[0], px == part0, bias0[ex]);
                    y[1] = score(y[1], py == part0, bias0[ey]);
                    y[2] = score(y[2], px == part1, bias1[ex]);
                    y[3] = score(y[3], py == part1, bias1[ey]);
                    most0 = fmaxf(most0, fmaxf(y[0], y[1]));
                    most1 = fmaxf(most1, fmaxf(y[2], y[3]));
                }
            }
#pragma unroll
            for (int step = 1; step < 4; step <<= 1) {
                most0 = fmaxf(most0, __shfl_xor_sync(0xffffffffu, most0, step));
                most1 = fmaxf(most1, __shfl_xor_sync(0xffffffffu, most1, step));
            }
            const float ref0 = most0 == -INFINITY ? 0.f : most0, ref1 = most1 == -INFINITY ? 0.f : most1;      // (no key so far: exponentials of minus infinity)
            if (key > 0) {
                const float f0 = ex2_approx(m0 - ref0), f1 = ex2_approx(m1 - ref1);
                l0 *= f0; l1 *= f1;
#pragma unroll
                for (int g = 0; g < 2 * kD; ++g) { o[g][0] *= f0; o[g][1] *= f0; o[g][2] *= f1; o[g][3] *= f1; }
            }
            m0 = most0; m1 = most1;
#pragma unroll
            for (int sub = 0; sub < 4; ++sub) {
                if (key + 16 * sub >= rows) break;
                uint32_t pf[4];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const float (&y)[4] = x[2 * sub + t];
                    const float a = ex2_approx(y[0] - ref0), b = ex2_approx(y[1] - ref0), c = ex2_approx(y[2] - ref1), d = ex2_approx(y[3] - ref1);
                    l0 += a + b; l1 += c + d;
                    pf[2 * t] = pack_bf16x2(a, b);
                    pf[2 * t + 1] = pack_bf16x2(c, d);
                }
#pragma unroll
                for (int g = 0; g < kD; ++g) {
                    uint32_t f[4];
                    ldmatrix_x4_trans(vs + (key + 16 * sub + a_row(lane)) * kP + 16 * g + a_col(lane), f);
                    mma_16816(o[2 * g], pf, f[0], f[1]);
                    mma_16816(o[2 * g + 1], pf, f[2], f[3]);
                }
            }
        }
#pragma unroll
        for (int step = 1; step < 4; step <<= 1) { l0 += __shfl_xor_sync(0xffffffffu, l0, step); l1 += __shfl_xor_sync(0xffffffffu, l1, step); }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const long long pixel = s.pixel[r0 + 8 * half];
            if (pixel < 0) continue;
            const float l = half ? l1 : l0, f = l == 0.f ? 0.f : 1.f / l;             // a row without any key: out 0, lse minus infinity
            __nv_bfloat16* const to = row_at(p, w, p.out_w, pixel);
#pragma unroll
            for (int g = 0; g < 2 * kD; ++g) store_pair(p, to, 8 * g + c2, o[g][2 * half] * f, o[g][2 * half + 1] * f);
            if (p.lse_w && c2 == 0) p.lse_w[scalar_at(p, w, pixel)] = l == 0.f ? -INFINITY : ((half ? m1 : m0) + log2f(l)) * kLn2;
        }
    }
}

template <int kD>
__global__ void __launch_bounds__(2 * kMaxTokens) rib_bias_small_bwd_kernel(const Problem p, const FastDiv by_words, double* offset_sums)
{
    extern __shared__ __align__(16) uint8_t sm[];
    constexpr int kP = kPitch<kD>;
    const int rows = rows_of(p.n), side = 2 * p.M - 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tile = warp * 16, c2 = 2 * (lane & 3);
    __nv_bfloat16 *const qs = reinterpret_cast<__nv_bfloat16*>(sm), *const ks = qs + rows * kP, *const vs = ks + rows * kP, *const gs = vs + rows * kP;
    __nv_bfloat16* const ds = gs + rows * kP;              // [key][kDSPitch]; before that, the rows of out
    float *const table = reinterpret_cast<float*>(ds + rows * kDSPitch), *const sums = table + table_floats(p.M);
    float *const lse = sums + table_floats(p.M), *const D = lse + rows;
    long long* const pixels = reinterpret_cast<long long*>(D + rows);
    const Places s{pixels, reinterpret_cast<int*>(pixels + rows)};
    const int per_head = p.pairs / p.heads;
    const int first = (int)((long long)p.pairs * blockIdx.x / gridDim.x), last = (int)((long long)p.pairs * (blockIdx.x + 1) / gridDim.x);
    const float isd = rsqrtf((float)p.d), scale = isd * kLog2e;
    const Staged<5> staged{{p.q, p.k, p.v, p.dout, p.out}, {qs, ks, vs, gs, ds}};
    clear_rows(qs, 4 * rows * kP);
    int head = -1;
    // the sums of a head by offset to those of all blocks, in 64 bits
    auto flush = [&](int h) {
        for (int e = threadIdx.x; e < side * side; e += blockDim.x)
            if (sums[e] != 0.f) atomicAdd(offset_sums + (size_t)h * side * side + e, (double)sums[e]);
    };
    for (int index = first; index < last; ++index) {
        const Block w = decode_window(p, per_head, index);
        __syncthreads();
        if (w.h != head) {
            if (head >= 0) flush(head);
            __syncthreads();
            gather_table(p, w.h, table);
            for (int e = threadIdx.x; e < side * side; e += blockDim.x) sums[e] = 0.f;
            head = w.h;
        }
        find_places(p, w, rows, s);
        __syncthreads();
        stage<kP>(p, by_words, w, s.pixel, staged);
        // a query that is none, or whose row has no key, has probability 0: lse plus infinity
        for (int i = threadIdx.x; i < rows; i += blockDim.x) {
            const float v = s.pixel[i] >= 0 ? p.lse_in[scalar_at(p, w, s.pixel[i])] * kLog2e : INFINITY;
            lse[i] = v == -INFINITY ? INFINITY : v;
        }
        __syncthreads();
        {   // D = rowsum(out o dO), two threads to a row
            // (what stands behind the last channel and the last row of out is anything)
            const int row = threadIdx.x >> 1;
            float sum = 0.f;
            for (int c = 2 * (threadIdx.x & 1); row < p.n && c < p.d; c += 4) {
                const int at = row * kP + c;
                const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(ds + at)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(gs + at));
                sum = fmaf(a.x, b.x, sum);
                if (c + 1 < p.d) sum = fmaf(a.y, b.y, sum);
            }
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            if (!(threadIdx.x & 1)) D[row] = sum;
        }
        __syncthreads();
        const int r0 = tile + (lane >> 2);                 // a thread has key rows r0 and r0 + 8 of the warp's tile, and of every 8 queries two
        const int place0 = s.place[r0], place1 = s.place[r0 + 8];
        const int part0 = place0 >> 16, part1 = place1 >> 16;
        const int entry0 = (p.M - 1) * (side + 1) + (place0 & 0xffff), entry1 = (p.M - 1) * (side + 1) + (place1 & 0xffff);
        // (parts of places without a token are alike: such a key is none for any query)
        const bool there0 = part0 != kNoPart, there1 = part1 != kNoPart;
        uint32_t kf[kD][4], vf[kD][4];
        float dk[2 * kD][4], dv[2 * kD][4];
#pragma unroll
        for (int g = 0; g < 2 * kD; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) dk[g][e] = dv[g][e] = 0.f;
#pragma unroll
        for (int k = 0; k < kD; ++k) {
            ldmatrix_x4(ks + (tile + a_row(lane)) * kP + 16 * k + a_col(lane), kf[k]);
            ldmatrix_x4(vs + (tile + a_row(lane)) * kP + 16 * k + a_col(lane), vf[k]);
        }
        for (int block = 0; block < rows; block += kQueryBlock) {
            const int end = min(rows, block + kQueryBlock);
            for (int query = block; query < end; query += 16) {
                float x[2][4], dp[2][4];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[t][e] = dp[t][e] = 0.f;
#pragma unroll
                for (int k = 0; k < kD; ++k) {
                    uint32_t f[4];
                    ldmatrix_x4(qs + (query + b_row(lane)) * kP + 16 * k + b_col(lane), f);
                    mma_16816(x[0], kf[k], f[0], f[1]);
                    mma_16816(x[1], kf[k], f[2], f[3]);
                    ldmatrix_x4(gs + (query + b_row(lane)) * kP + 16 * k + b_col(lane), f);
                    mma_16816(dp[0], vf[k], f[0], f[1]);
                    mma_16816(dp[1], vf[k], f[2], f[3]);
                }
                uint32_t pf[4], df[4];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int at = query + 8 * t + c2;
                    const int2 places = *reinterpret_cast<const int2*>(s.place + at);
                    const float2 ls = *reinterpret_cast<const float2*>(lse + at), dd = *reinterpret_cast<const float2*>(D + at);
                    float pr[4], d[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {          // (key row r0 + 8 (e / 2), query at + e % 2)
                        const int place = e & 1 ? places.y : places.x, entry = (e & 2 ? entry1 : entry0) - (place & 0xffff);
                        const float b = table[entry];
                        const bool seen = (e & 2 ? there1 : there0) && (place >> 16) == (e & 2 ? part1 : part0) && b != -INFINITY;
                        pr[e] = seen ? ex2_approx(min_nan(fmaf(x[t][e], scale, b - (e & 1 ? ls.y : ls.x)), 0.f)) : 0.f;      // (at most 1, whatever lse has left of its digits)
                        d[e] = seen ? pr[e] * (dp[t][e] - (e & 1 ? dd.y : dd.x)) : 0.f;
                        if (seen) atomicAdd(sums + entry, d[e]);
                    }
                    pf[2 * t] = pack_bf16x2(pr[0], pr[1]);
                    pf[2 * t + 1] = pack_bf16x2(pr[2], pr[3]);
                    df[2 * t] = pack_bf16x2(d[0], d[1]);
                    df[2 * t + 1] = pack_bf16x2(d[2], d[3]);
                    __nv_bfloat16* const to = ds + r0 * kDSPitch + at - block;
                    *reinterpret_cast<uint32_t*>(to) = df[2 * t];
                    *reinterpret_cast<uint32_t*>(to + 8 * kDSPitch) = df[2 * t + 1];
                }
#pragma unroll
                for (int g = 0; g < kD; ++g) {
                    uint32_t f[4];
                    ldmatrix_x4_trans(gs + (query + a_row(lane)) * kP + 16 * g + a_col(lane), f);
                    mma_16816(dv[2 * g], pf, f[0], f[1]);
                    mma_16816(dv[2 * g + 1], pf, f[2], f[3]);
                    ldmatrix_x4_trans(qs + (query + a_row(lane)) * kP + 16 * g + a_col(lane), f);
                    mma_16816(dk[2 * g], df, f[0], f[1]);
                    mma_16816(dk[2 * g + 1], df, f[2], f[3]);
                }
            }
            __syncthreads();
            // dQ of the block's queries: 16 of them and 16 channels at a time
            const int tiles = (end - block) / 16, warps = rows / 16;
            for (int unit = warp; unit < tiles * kD; unit += warps) {
                const int g = unit / tiles, query = 16 * (unit - g * tiles);
                float a[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
                for (int key = 0; key < rows; key += 16) {
                    uint32_t f[4], kk[4];
                    ldmatrix_x4_trans(ds + (key + b_row(lane)) * kDSPitch + query + b_col(lane), f);
                    ldmatrix_x4_trans(ks + (key + a_row(lane)) * kP + 16 * g + a_col(lane), kk);
                    mma_16816(a[0], f, kk[0], kk[1]);
                    mma_16816(a[1], f, kk[2], kk[3]);
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const long long pixel = s.pixel[block + query + (lane >> 2) + 8 * half];
                    if (pixel < 0) continue;
                    __nv_bfloat16* const to = row_at(p, w, p.dq, pixel);
#pragma unroll
                    for (int t = 0; t < 2; ++t) store_pair(p, to, 16 * g + 8 * t + c2, a[t][2 * half] * isd, a[t][2 * half + 1] * isd);
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const long long pixel = s.pixel[r0 + 8 * half];
            if (pixel < 0) continue;
            __nv_bfloat16 *const to_v = row_at(p, w, p.dv, pixel), *const to_k = row_at(p, w, p.dk, pixel);
#pragma unroll
            for (int g = 0; g < 2 * kD; ++g) {
                store_pair(p, to_v, 8 * g + c2, dv[g][2 * half], dv[g][2 * half + 1]);
                store_pair(p, to_k, 8 * g + c2, dk[g][2 * half] * isd, dk[g][2 * half + 1] * isd);
            }
        }
    }
    if (head >= 0) flush(head);                            // (behind the last barrier, every sum is there)
}

// Blocks: one to a window, or as many as walk their runs well.  Of blocks of up to 128 threads (windows of up to 64 tokens) the SMs hold 512
// threads, and that many blocks are fastest (8 x 96 x 96 tokens, 6 heads of 32, windows of 7, backward 231 us; twice as many 264, one to a window 256).
// Of larger ones they hold one or two, whose ends do not meet, and twice the threads deal the work out more evenly (heads of 30, windows of 9:
// 455 us, with half as many 470; of 12: 655 and 690).
int blocks_for(const Problem& p, int sms, size_t shared)
{
    const int threads = 2 * rows_of(p.n), by_shared = (int)(kMostShared / (shared + 1024)), by_threads = (threads <= 128 ? 512 : 1024) / threads;
    const long long blocks = (long long)sms * (by_threads < by_shared ? by_threads : by_shared > 1 ? by_shared : 1);
    return (int)(p.pairs < blocks ? p.pairs : blocks);
}

}  // namespace

bool bias_small_supported(const Problem& p)
{
    return p.bias && p.n <= kMaxTokens && p.d <= 64 && shared_bytes(p.n, p.d, p.M, true) <= kMostShared;
}

cudaError_t bias_small_fwd(const Problem& p, cudaStream_t stream)
{
    const int kd = (p.d + 15) / 16;
    const auto kernel = kd == 1 ? rib_bias_small_fwd_kernel<1> : kd == 2 ? rib_bias_small_fwd_kernel<2> : kd == 3 ? rib_bias_small_fwd_kernel<3> : rib_bias_small_fwd_kernel<4>;
    static KernelSetup setup[4];
    int sms = 0;
    if (cudaError_t e = setup[kd - 1].prepare(kernel, kMostShared, &sms)) return e;
    const size_t bytes = shared_bytes(p.n, p.d, p.M, false);
    { ProfileScope scope(RIB_KERNEL_BIAS_SMALL_FWD, stream); kernel<<<blocks_for(p, sms, bytes), 2 * rows_of(p.n), bytes, stream>>>(p, make_fast_div(p.d / elements_of_word(p.d))); }
    return cudaGetLastError();
}

cudaError_t bias_small_bwd(const Problem& p, double* offset_sums, cudaStream_t stream)
{
    const int kd = (p.d + 15) / 16;
    const auto kernel = kd == 1 ? rib_bias_small_bwd_kernel<1> : kd == 2 ? rib_bias_small_bwd_kernel<2> : kd == 3 ? rib_bias_small_bwd_kernel<3> : rib_bias_small_bwd_kernel<4>;
    static KernelSetup setup[4];
    int sms = 0;
    if (cudaError_t e = setup[kd - 1].prepare(kernel, kMostShared, &sms)) return e;
    const size_t bytes = shared_bytes(p.n, p.d, p.M, true);
    { ProfileScope scope(RIB_KERNEL_BIAS_SMALL_BWD, stream); kernel<<<blocks_for(p, sms, bytes), 2 * rows_of(p.n), bytes, stream>>>(p, make_fast_div(p.d / elements_of_word(p.d)), offset_sums); }
    return cudaGetLastError();
}

}  // namespace rib
