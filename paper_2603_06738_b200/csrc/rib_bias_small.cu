// Window attention with a bias by buckets in windows of up to 256 tokens whose shape the tcgen05 kernels do not take (odd windows, head widths
// and shifts), in fp32 on the plain pipes.  A block has one window of one head: its rows lie in shared memory, a thread has one query row (or, in
// the second half of the backward pass, one key row) in registers and walks the others, which the threads of a warp read at the same time (a
// broadcast of 16 bytes per four channels); two or four threads share a row of a window that has few (a row in one thread: 147 us); the biases by
// offset are gathered to shared memory once.  dS of the whole window lies there too (up to 144 tokens; beyond, it is added by offset with
// shared-memory atomics, which on the smaller windows take REFATOMS), and a thread sums an offset's.  Such windows are small and many, and what the any-shape kernels took on them was latency: a map of
// 50 x 39 tokens in windows of 7, forward and backward 232 -> REFSMALL us.
#include "rib_common.cuh"

namespace rib {
namespace {

constexpr int kMaxTokens = 256;
constexpr float kLog2 = 1.4426950408889634f;

struct Window { int h, b, tokens, side, width; };          // width: floats per row in shared memory (d rounded up to 4)

constexpr int kMatrixTokens = 144;          // windows whose dS is kept

// shared memory: two row arrays [n][width], biases [side^2], (backward) dS [n][n + 1] or its sums [side^2], then per place of the window: pixel row
// offset (-1: no token), entry y side + x, part, and (backward) lse * log2(e) and D
struct Shared {
    float *rows0, *rows1, *bias, *ds, *lse, *D;
    int *pixel, *entry, *part;
};
__host__ __device__ inline size_t ds_floats(int n, int side) { return n <= kMatrixTokens ? (size_t)(n * (n + 1) + 3) & ~3 : (size_t)(side * side + 3) & ~3; }
__host__ __device__ inline size_t shared_bytes(int n, int d, int side, bool backward)
{
    const size_t width = (d + 3) & ~3;
    return sizeof(float) * (2 * n * width + (size_t)((side * side + 3) & ~3) + (backward ? ds_floats(n, side) + 5 * (size_t)n : 3 * (size_t)n));
}
__device__ inline Shared carve(float* sm, int n, int width, int side, bool backward)
{
    Shared s;
    const int table = (side * side + 3) & ~3;
    s.rows0 = sm; s.rows1 = s.rows0 + n * width;
    s.bias = s.rows1 + n * width;
    s.ds = s.bias + table;
    float* rest = s.ds + (backward ? ds_floats(n, side) : 0);
    s.pixel = reinterpret_cast<int*>(rest); s.entry = s.pixel + n; s.part = s.entry + n;
    s.lse = rest + 3 * n; s.D = s.lse + n;
    return s;
}

// Places, biases (times log2(e); minus infinity: not attended to) and the window of this block.
__device__ inline Window set_up(const Problem& p, const Shared& s, bool backward)
{
    int pid = blockIdx.x;
    Window w;
    w.h = pid % p.heads; pid /= p.heads;
    const int wx = pid % p.nWx; pid /= p.nWx;
    const int wy = pid % p.nWy; w.b = pid / p.nWy;
    w.side = 2 * p.M - 1;
    w.width = (p.d + 3) & ~3;
    for (int i = threadIdx.x; i < p.n; i += blockDim.x) {
        int Y, X;
        token_pixel(p.Hp, p.Wp, p.M, p.s, wy, wx, i, Y, X);
        const int y = i / p.M, x = i - y * p.M;
        s.pixel[i] = Y < p.H && X < p.W ? Y * p.W + X : -1;
        s.entry[i] = y * w.side + x;
        s.part[i] = p.masked ? window_part(p.M, p.s, wy == p.nWy - 1, wx == p.nWx - 1, y, x) : 0;
    }
    for (int e = threadIdx.x; e < w.side * w.side; e += blockDim.x) {
        const int u = __ldg(p.buckets + e);
        s.bias[e] = (unsigned)u < (unsigned)p.num_buckets ? bias_at(p.bias, p.bias_bf16, (long long)w.h * p.bias_head_stride + u) * kLog2 : -INFINITY;
        if (backward && p.n > kMatrixTokens) s.ds[e] = 0.f;
    }
    return w;
}
__device__ inline size_t row_offset(const Problem& p, const Window& w, int pixel)
{
    return (((size_t)w.b * p.H * p.W + pixel) * p.heads + w.h) * p.d;
}
__device__ inline size_t scalar_offset(const Problem& p, const Window& w, int pixel)
{
    return ((size_t)w.b * p.heads + w.h) * p.H * p.W + pixel;
}
// The window's rows of x as fp32, zeros behind the last channel and where there is no token; a warp per row, two at a time.
__device__ inline void stage(const Problem& p, const Window& w, const Shared& s, const __nv_bfloat16* x, float* rows)
{
    const int per_row = w.width;
#pragma unroll 4
    for (int e = threadIdx.x; e < p.n * per_row; e += blockDim.x) {
        const int i = e / per_row, c = e - i * per_row, pixel = s.pixel[i];
        rows[e] = pixel >= 0 && c < p.d ? __bfloat162float(x[row_offset(p, w, pixel) + c]) : 0.f;
    }
}
template <int kMax>
__device__ inline void load_row(const Problem& p, const __nv_bfloat16* x, size_t at, float (&r)[kMax])
{
#pragma unroll
    for (int c = 0; c < kMax; ++c) r[c] = c < p.d ? __bfloat162float(x[at + c]) : 0.f;
}
template <int kMax>
__device__ inline float dot(const float (&a)[kMax], const float* row, int groups)
{
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);          // (four short chains instead of a long one)
#pragma unroll
    for (int g = 0; g < kMax / 4; ++g)
        if (g < groups) {
            const float4 v = reinterpret_cast<const float4*>(row)[g];
            sum.x = fmaf(a[4 * g], v.x, sum.x); sum.y = fmaf(a[4 * g + 1], v.y, sum.y); sum.z = fmaf(a[4 * g + 2], v.z, sum.z); sum.w = fmaf(a[4 * g + 3], v.w, sum.w);
        }
    return (sum.x + sum.y) + (sum.z + sum.w);
}
template <int kMax>
__device__ inline void add_scaled(float (&a)[kMax], float f, const float* row, int groups)
{
#pragma unroll
    for (int g = 0; g < kMax / 4; ++g)
        if (g < groups) {
            const float4 v = reinterpret_cast<const float4*>(row)[g];
            a[4 * g] = fmaf(f, v.x, a[4 * g]); a[4 * g + 1] = fmaf(f, v.y, a[4 * g + 1]); a[4 * g + 2] = fmaf(f, v.z, a[4 * g + 2]); a[4 * g + 3] = fmaf(f, v.w, a[4 * g + 3]);
        }
}
// the sum over the `share` neighbouring lanes that have a row together
__device__ inline float shared_sum(float v, int share)
{
    for (int o = 1; o < share; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int kMax>
__device__ inline void share_row(float (&r)[kMax], int share)
{
    if (share == 1) return;
#pragma unroll
    for (int c = 0; c < kMax; ++c) r[c] = shared_sum(r[c], share);
}
template <int kMax>
__device__ inline void store_row(const Problem& p, __nv_bfloat16* x, size_t at, const float (&r)[kMax], float f)
{
#pragma unroll
    for (int c = 0; c < kMax; ++c)
        if (c < p.d) x[at + c] = __float2bfloat16_rn(r[c] * f);
}

template <int kMax>
__global__ void __launch_bounds__(kMaxTokens) rib_bias_small_fwd_kernel(const Problem p, int share)
{
    extern __shared__ float sm[];
    const Shared s = carve(sm, p.n, (p.d + 3) & ~3, 2 * p.M - 1, false);
    const Window w = set_up(p, s, false);
    __syncthreads();
    stage(p, w, s, p.k, s.rows0);
    stage(p, w, s, p.v, s.rows1);
    __syncthreads();
    const int i = min((int)threadIdx.x / share, p.n - 1), groups = w.width / 4;
    const bool mine = (int)threadIdx.x < p.n * share && s.pixel[i] >= 0;
    const size_t at = mine ? row_offset(p, w, s.pixel[i]) : 0;
    float q[kMax], o[kMax], m = -INFINITY, l = 0.f;
    load_row(p, p.q, at, q);
    const float scale = rsqrtf((float)p.d) * kLog2;
#pragma unroll
    for (int c = 0; c < kMax; ++c) { q[c] *= scale; o[c] = 0.f; }
    const float* bias = s.bias + (p.M - 1) * w.side + p.M - 1 - s.entry[i];
    const int part = s.part[i];
    for (int j = threadIdx.x % share; mine && j < p.n; j += share) {
        const float b = bias[s.entry[j]];
        if (s.pixel[j] < 0 || s.part[j] != part || b == -INFINITY) continue;
        const float x = dot(q, s.rows0 + j * w.width, groups) + b;
        if (x > m) {                                   // a new maximum: what there is so far shrinks
            const float f = exp2f(m - x);
            l *= f;
#pragma unroll
            for (int c = 0; c < kMax; ++c) o[c] *= f;
            m = x;
        }
        const float e = exp2f(x - m);
        l += e;
        add_scaled(o, e, s.rows1 + j * w.width, groups);
    }
    if (share > 1) {                                   // the lanes of a row: the larger of their references, then sums
        float most = m;
        for (int step = 1; step < share; step <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, step));
        const float f = m == -INFINITY ? 0.f : exp2f(m - most);
        l = shared_sum(l * f, share);
#pragma unroll
        for (int c = 0; c < kMax; ++c) o[c] *= f;
        share_row(o, share);
        m = most;
    }
    if (!mine || threadIdx.x % share) return;
    store_row(p, p.out_w, at, o, l > 0.f ? 1.f / l : 0.f);
    if (p.lse_w) p.lse_w[scalar_offset(p, w, s.pixel[i])] = l > 0.f ? (m + log2f(l)) / kLog2 : -INFINITY;
}

template <int kMax>
__global__ void __launch_bounds__(kMaxTokens, kMax <= 24 ? 2 : 1) rib_bias_small_bwd_kernel(const Problem p, double* offset_sums, int share)
{
    extern __shared__ float sm[];
    const Shared s = carve(sm, p.n, (p.d + 3) & ~3, 2 * p.M - 1, true);
    const Window w = set_up(p, s, true);
    __syncthreads();
    stage(p, w, s, p.k, s.rows0);
    stage(p, w, s, p.v, s.rows1);
    __syncthreads();
    const int i = min((int)threadIdx.x / share, p.n - 1), groups = w.width / 4, centre = (p.M - 1) * w.side + p.M - 1, first = threadIdx.x % share;
    const bool mine = (int)threadIdx.x < p.n * share && s.pixel[i] >= 0;
    const size_t at = mine ? row_offset(p, w, s.pixel[i]) : 0;
    const float isd = rsqrtf((float)p.d);
    {
        // ---- a query row: dq and the sums of dS by offset
        float q[kMax], g[kMax], dq[kMax];
        load_row(p, p.out, at, q);
        load_row(p, p.dout, at, g);
        float D = 0.f;
#pragma unroll
        for (int c = 0; c < kMax; ++c) D = fmaf(q[c], g[c], D);
        load_row(p, p.q, at, q);
#pragma unroll
        for (int c = 0; c < kMax; ++c) { q[c] *= isd * kLog2; dq[c] = 0.f; }
        const float lse = mine ? p.lse_in[scalar_offset(p, w, s.pixel[i])] * kLog2 : 0.f;
        if (mine && first == 0) { s.lse[i] = lse; s.D[i] = D; }
        const int part = s.part[i], origin = centre - s.entry[i];
        for (int j = first; j < p.n; j += share) {
            const int e = origin + s.entry[j];
            const float b = s.bias[e];
            const bool seen = mine && s.pixel[j] >= 0 && s.part[j] == part && b != -INFINITY;
            float ds = 0.f;
            if (seen) {
                ds = exp2f(dot(q, s.rows0 + j * w.width, groups) + b - lse) * (dot(g, s.rows1 + j * w.width, groups) - D);
                add_scaled(dq, ds, s.rows0 + j * w.width, groups);
            }
            if (p.n > kMatrixTokens) { if (seen) atomicAdd(s.ds + e, ds); }
            else if ((int)threadIdx.x < p.n * share) s.ds[i * (p.n + 1) + j] = ds;
        }
        share_row(dq, share);
        if (mine && first == 0) store_row(p, p.dq, at, dq, isd);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < w.side * w.side; e += blockDim.x) {
        float sum = 0.f;
        if (p.n > kMatrixTokens) {
            sum = s.ds[e];
        } else {
            const int dy = e / w.side - p.M + 1, dx = e % w.side - p.M + 1;          // key - query
            const int x0 = max(0, -dx), x1 = p.M - max(0, dx);
            for (int y = max(0, -dy); y < p.M - max(0, dy); ++y)
                for (int x = x0; x < x1; ++x) sum += s.ds[(y * p.M + x) * (p.n + 1) + (y + dy) * p.M + x + dx];
        }
        if (sum != 0.f) atomicAdd(offset_sums + (size_t)w.h * w.side * w.side + e, (double)sum);
    }
    stage(p, w, s, p.q, s.rows0);
    stage(p, w, s, p.dout, s.rows1);
    __syncthreads();
    {
        // ---- a key row: dk and dv
        float k[kMax], v[kMax], dk[kMax], dv[kMax];
        load_row(p, p.k, at, k);
        load_row(p, p.v, at, v);
#pragma unroll
        for (int c = 0; c < kMax; ++c) { k[c] *= isd * kLog2; dk[c] = dv[c] = 0.f; }
        const int part = s.part[i], origin = centre + s.entry[i];
        for (int j = first; mine && j < p.n; j += share) {
            const float b = s.bias[origin - s.entry[j]];
            if (s.pixel[j] < 0 || s.part[j] != part || b == -INFINITY) continue;
            const float prob = exp2f(dot(k, s.rows0 + j * w.width, groups) + b - s.lse[j]);
            const float ds = prob * (dot(v, s.rows1 + j * w.width, groups) - s.D[j]);
            add_scaled(dv, prob, s.rows1 + j * w.width, groups);
            add_scaled(dk, ds, s.rows0 + j * w.width, groups);
        }
        share_row(dv, share);
        share_row(dk, share);
        if (mine && first == 0) {
            store_row(p, p.dv, at, dv, 1.f);
            store_row(p, p.dk, at, dk, isd);
        }
    }
}

int share_of(const Problem& p) { return p.n <= kMaxTokens / 4 ? 4 : p.n <= kMaxTokens / 2 ? 2 : 1; }         // threads to a row
int threads_of(const Problem& p) { return (p.n * share_of(p) + 31) / 32 * 32; }

template <typename Kernel>
cudaError_t room_for(Kernel kernel, size_t bytes)
{
    return bytes > 48 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) : cudaSuccess;
}

}  // namespace

bool bias_small_supported(const Problem& p)
{
    return p.bias && p.n <= kMaxTokens && p.d <= 64 && shared_bytes(p.n, p.d, 2 * p.M - 1, true) <= 200 * 1024;
}

cudaError_t bias_small_fwd(const Problem& p, cudaStream_t stream)
{
    const auto kernel = p.d <= 16 ? rib_bias_small_fwd_kernel<16> : p.d <= 24 ? rib_bias_small_fwd_kernel<24> : p.d <= 32 ? rib_bias_small_fwd_kernel<32> : rib_bias_small_fwd_kernel<64>;
    const size_t bytes = shared_bytes(p.n, p.d, 2 * p.M - 1, false);
    if (cudaError_t e = room_for(kernel, bytes)) return e;
    { ProfileScope scope(RIB_KERNEL_BIAS_SMALL_FWD, stream); kernel<<<p.pairs, threads_of(p), bytes, stream>>>(p, share_of(p)); }
    return cudaGetLastError();
}

cudaError_t bias_small_bwd(const Problem& p, double* offset_sums, cudaStream_t stream)
{
    const auto kernel = p.d <= 16 ? rib_bias_small_bwd_kernel<16> : p.d <= 24 ? rib_bias_small_bwd_kernel<24> : p.d <= 32 ? rib_bias_small_bwd_kernel<32> : rib_bias_small_bwd_kernel<64>;
    const size_t bytes = shared_bytes(p.n, p.d, 2 * p.M - 1, true);
    if (cudaError_t e = room_for(kernel, bytes)) return e;
    { ProfileScope scope(RIB_KERNEL_BIAS_SMALL_BWD, stream); kernel<<<p.pairs, threads_of(p), bytes, stream>>>(p, offset_sums, share_of(p)); }
    return cudaGetLastError();
}

}  // namespace rib
