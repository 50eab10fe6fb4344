// Activation checkpoints in 8 bits: a row of d channels of one token and head becomes d whole numbers -127 .. 127 and one fp32 scale,
//     scale = max_c |x_c| * (1/127),   code_c = round(x_c / scale),   restored x_c = bf16(code_c * scale),
// rounding half to even, division and products as IEEE fp32.  A row of zeros has scale 0; a row with an infinity or a NaN gets the scale
// NaN and comes back as NaN, so that an overflow is not lost on the way through the checkpoint.
//
// Both directions are bound by memory: 2 d bytes on one side, d + 4 on the other.  Rows of 8, 16, ... 64 channels (16-byte aligned): a thread has 8
// channels of a row, or 16 to store those of whole 32 bytes - one or two 16-byte accesses to x, one of as many codes, neighbours side by side -
// and the lanes of a row share its maximum by shuffles.  Other widths: a block takes 64 rows, whose bytes are whole 16-byte words on both sides, through
// shared memory.
#include "rib_common.cuh"

namespace rib {
namespace {

constexpr int kThreads = 256;
constexpr int kStagedRows = 64;
constexpr int kStoreUnroll = 4, kRestoreUnroll = 8, kRestoreBlocks = 2;

// Quotients decide codes, so they are those of the IEEE division.  With y the reciprocal of the scale, t = x y is off by an ulp or so; the remainder
// x - t scale is exact, and adding y times it leaves a quotient (Markstein's method) that names the same code for every pair of bf16 mantissas and
// every distance of their exponents: they are few enough to try them all, and a test does.  Three operations without a branch: a test
// whether t lies near a border, with the division behind it, took 108 to 116 us
// where this took 96, since half the maximum is a border and half of the warps met one.
// A scale below 2^-100, whose remainders could vanish, takes the division.
// The nearest whole number is read off the low bits of t + 1.5 x 2^23 (half to even, as round() does): conversions between floating and whole
// numbers have an eighth of the rate of additions, and were what these kernels waited for.  Both return a word with the code in its low byte.
__device__ __forceinline__ uint32_t code_of(float x, float scale, float inverse)
{
    const float t = x * inverse;
    return __float_as_uint(fmaf(fmaf(-t, scale, x), inverse, t) + 12582912.f);
}
__device__ __forceinline__ uint32_t quotient_code(float x, float scale) { return (uint32_t)__float2int_rn(__fdiv_rn(x, scale)); }
// the low bytes of four words
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
struct RowScale { float scale, inverse; bool zero, tiny; };
__device__ __forceinline__ RowScale row_scale(float most, bool bad)
{
    RowScale r;
    r.scale = bad ? __int_as_float(0x7fffffff) : most * (1.f / 127.f);
    r.zero = bad || r.scale == 0.f;
    r.inverse = 1.f / r.scale;
    r.tiny = r.scale < 0x1p-100f;
    return r;
}

// kLanes lanes to a row (a power of two, the last ones without channels where d is none), four runs of kThreads / kLanes rows per block (a layer of
// 16 x 96 x 96 tokens, 6 heads, d = 32: 85 us for four tensors, 4.2 TB/s; two runs or one 91.  Blocks that walk runs with the next one's loads under
// way, as restore has them, took 8 us more: the shuffles and the reciprocal of a row wait for one another, and what hides that is other warps)
// kWords: 16-byte words of a thread, 2 where rows are whole 32 bytes (a reciprocal and shuffles for sixteen channels: 85 us where
// one word took 94).
template <int kLanes, int kWords>
__global__ void __launch_bounds__(kThreads) rib_checkpoint_store_kernel(const __nv_bfloat16* __restrict__ x, long long rows, int d, int8_t* __restrict__ codes, float* __restrict__ scales)
{
    constexpr int kUnroll = kStoreUnroll, kRowsAtOnce = kThreads / kLanes;
    const int part = threadIdx.x % kLanes;
    const bool mine = 8 * kWords * part < d;
    const long long row0 = (long long)blockIdx.x * (kUnroll * kRowsAtOnce) + threadIdx.x / kLanes;
    uint4 v[kUnroll][kWords];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
        const long long row = row0 + k * kRowsAtOnce;
#pragma unroll
        for (int j = 0; j < kWords; ++j) v[k][j] = mine && row < rows ? __ldg(reinterpret_cast<const uint4*>(x + row * d) + kWords * part + j) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
        const long long row = row0 + k * kRowsAtOnce;
        uint32_t w[4 * kWords];
#pragma unroll
        for (int j = 0; j < kWords; ++j) { w[4 * j] = v[k][j].x; w[4 * j + 1] = v[k][j].y; w[4 * j + 2] = v[k][j].z; w[4 * j + 3] = v[k][j].w; }
        // the largest magnitude as an integer: magnitudes of bf16 are ordered like their bits, infinity and NaN behind all others
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 4 * kWords; ++i) most = max(most, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
#pragma unroll
        for (int o = kLanes / 2; o; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
        const RowScale s = row_scale(__uint_as_float(most << 16), most >= 0x7f80u);
        uint32_t c[2 * kWords];
#pragma unroll
        for (int i = 0; i < 2 * kWords; ++i) c[i] = 0u;
        if (!s.zero) {
#pragma unroll
            for (int i = 0; i < 2 * kWords; ++i)
                c[i] = low_bytes(code_of(__uint_as_float(w[2 * i] << 16), s.scale, s.inverse), code_of(__uint_as_float(w[2 * i] & 0xffff0000u), s.scale, s.inverse),
                                 code_of(__uint_as_float(w[2 * i + 1] << 16), s.scale, s.inverse), code_of(__uint_as_float(w[2 * i + 1] & 0xffff0000u), s.scale, s.inverse));
            if (s.tiny) {
#pragma unroll
                for (int i = 0; i < 2 * kWords; ++i)
                    c[i] = low_bytes(quotient_code(__uint_as_float(w[2 * i] << 16), s.scale), quotient_code(__uint_as_float(w[2 * i] & 0xffff0000u), s.scale),
                                     quotient_code(__uint_as_float(w[2 * i + 1] << 16), s.scale), quotient_code(__uint_as_float(w[2 * i + 1] & 0xffff0000u), s.scale));
            }
        }
        if (row < rows) {
            if (mine) {
                if constexpr (kWords == 2) *reinterpret_cast<uint4*>(codes + row * d + 16 * part) = make_uint4(c[0], c[1], c[2], c[3]);
                else *reinterpret_cast<uint2*>(codes + row * d + 8 * part) = make_uint2(c[0], c[1]);
            }
            if (part == 0) scales[row] = s.scale;
        }
    }
}

// any d: 64 rows of a block through shared memory
__global__ void __launch_bounds__(kThreads) rib_checkpoint_store_staged_kernel(const __nv_bfloat16* __restrict__ x, long long rows, int d, int8_t* __restrict__ codes, float* __restrict__ scales)
{
    __shared__ __align__(16) __nv_bfloat16 xs[kStagedRows * 64];
    __shared__ __align__(16) int8_t cs[kStagedRows * 64];
    const long long row0 = (long long)blockIdx.x * kStagedRows;
    const int here = (int)min((long long)kStagedRows, rows - row0), elements = here * d;
    const __nv_bfloat16* src = x + row0 * d;
    for (int e = 8 * threadIdx.x; e < elements; e += 8 * kThreads) {
        if (e + 8 <= elements) *reinterpret_cast<uint4*>(xs + e) = __ldg(reinterpret_cast<const uint4*>(src + e));
        else for (int i = e; i < elements; ++i) xs[i] = src[i];
    }
    __syncthreads();
    // four lanes to a row
    const int r = threadIdx.x >> 2, part = threadIdx.x & 3;
    float most = 0.f;
    bool bad = false;
    if (r < here)
        for (int c = part; c < d; c += 4) {
            const float a = fabsf(__bfloat162float(xs[r * d + c]));
            bad = bad || !isfinite(a);
            most = fmaxf(most, a);
        }
    for (int o = 1; o < 4; o <<= 1) {
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        bad = __shfl_xor_sync(0xffffffffu, bad ? 1 : 0, o) != 0 || bad;
    }
    const RowScale s = row_scale(most, bad);
    if (r < here) {
        for (int c = part; c < d; c += 4) {
            const float v = __bfloat162float(xs[r * d + c]);
            cs[r * d + c] = s.zero ? 0 : (int8_t)(s.tiny ? quotient_code(v, s.scale) : code_of(v, s.scale, s.inverse));
        }
        if (part == 0) scales[row0 + r] = s.scale;
    }
    __syncthreads();
    int8_t* dst = codes + row0 * d;
    for (int e = 16 * threadIdx.x; e < elements; e += 16 * kThreads) {
        if (e + 16 <= elements) *reinterpret_cast<uint4*>(dst + e) = *reinterpret_cast<const uint4*>(cs + e);
        else for (int i = e; i < elements; ++i) dst[i] = cs[i];
    }
}

struct RestoreArgs { CheckpointRows t[4]; };

// A block walks runs of rows and has the next run's loads under way while it writes one (the same layer: 64 us for four tensors, 5.5 TB/s; a run per block 100)
template <int kLanes>
__global__ void __launch_bounds__(kThreads) rib_checkpoint_restore_kernel(const RestoreArgs args, long long rows, int d)
{
    constexpr int kRowsAtOnce = kThreads / kLanes;
    const CheckpointRows t = args.t[blockIdx.y];
    const int part = threadIdx.x % kLanes;
    if (8 * part >= d) return;
    const long long step = (long long)gridDim.x * kRestoreUnroll * kRowsAtOnce;
    long long row0 = (long long)blockIdx.x * (kRestoreUnroll * kRowsAtOnce) + threadIdx.x / kLanes;
    const uint2* src = reinterpret_cast<const uint2*>(t.codes + 8 * part);
    uint4* dst = reinterpret_cast<uint4*>(t.x + 8 * part);
    const int words = d / 8;
    uint2 c[kRestoreUnroll], ahead[kRestoreUnroll];
    float scale[kRestoreUnroll], ahead_scale[kRestoreUnroll];
    auto load = [&](uint2 (&c)[kRestoreUnroll], float (&scale)[kRestoreUnroll]) {
#pragma unroll
        for (int k = 0; k < kRestoreUnroll; ++k) {
            const long long row = row0 + k * kRowsAtOnce;
            c[k] = row < rows ? __ldg(src + row * words) : make_uint2(0u, 0u);
            scale[k] = row < rows ? __ldg(t.scales + row) : 0.f;
        }
    };
    load(c, scale);
    while (row0 < rows) {
        const long long here = row0;
        row0 += step;
        load(ahead, ahead_scale);
#pragma unroll
        for (int k = 0; k < kRestoreUnroll; ++k) {
            const long long row = here + k * kRowsAtOnce;
            if (row < rows) dst[row * words] = restored_chunk(c[k], scale[k]);
            c[k] = ahead[k];
            scale[k] = ahead_scale[k];
        }
    }
}

__global__ void __launch_bounds__(kThreads) rib_checkpoint_restore_staged_kernel(const RestoreArgs args, long long rows, int d)
{
    __shared__ float scale[kStagedRows];
    const CheckpointRows t = args.t[blockIdx.y];
    const long long row0 = (long long)blockIdx.x * kStagedRows;
    const int here = (int)min((long long)kStagedRows, rows - row0), elements = here * d;
    if (threadIdx.x < here) scale[threadIdx.x] = __ldg(t.scales + row0 + threadIdx.x);
    __syncthreads();
    const int8_t* src = t.codes + row0 * d;
    __nv_bfloat16* dst = t.x + row0 * d;
    for (int e = 8 * threadIdx.x; e < elements; e += 8 * kThreads) {
        if (e + 8 <= elements) {
            const uint2 c = __ldg(reinterpret_cast<const uint2*>(src + e));
            const uint32_t w[2] = {c.x, c.y};
            __nv_bfloat162 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = __floats2bfloat162_rn((float)(int8_t)(w[i >> 1] >> (16 * (i & 1))) * scale[(e + 2 * i) / d],
                                             (float)(int8_t)(w[i >> 1] >> (16 * (i & 1) + 8)) * scale[(e + 2 * i + 1) / d]);
            *reinterpret_cast<uint4*>(dst + e) = *reinterpret_cast<const uint4*>(v);
        } else {
            for (int i = e; i < elements; ++i) dst[i] = __float2bfloat16_rn((float)src[i] * scale[i / d]);
        }
    }
}

// q, k, v and out of a layer with heads of 8 or 16 channels: four lanes to a row, q and k to rows of 32 columns
__global__ void __launch_bounds__(kThreads) rib_checkpoint_restore_wide_kernel(const RestoreArgs args, long long rows, int d)
{
    const long long thread = (long long)blockIdx.x * kThreads + threadIdx.x, row = thread >> 2;
    const int part = (int)(thread & 3);
    if (row >= rows) return;
    restore_wide<true>(args.t, (size_t)row, d, part);
    if (8 * part >= d) return;
#pragma unroll
    for (int i = 2; i < 4; ++i)
        reinterpret_cast<uint4*>(args.t[i].x + row * d)[part] =
            restored_chunk(__ldg(reinterpret_cast<const uint2*>(args.t[i].codes + row * d) + part), __ldg(args.t[i].scales + row));
}

// 8 channels to a thread: lanes to a row as a power of two
int lanes_of(int d) { return d <= 8 ? 1 : d <= 16 ? 2 : d <= 32 ? 4 : 8; }
// restore: blocks of a run each, or as many as kRestoreBlocks to an SM (of 148: the same number everywhere, so that a call's shape decides the launch)
unsigned restore_blocks(long long rows, int lanes, int tensors)
{
    const long long per = (long long)kRestoreUnroll * kThreads / lanes, all = (rows + per - 1) / per, most = kRestoreBlocks * 148 / tensors;
    return (unsigned)(all < most ? all : most);
}

}  // namespace

cudaError_t checkpoint_store(const __nv_bfloat16* x, long long rows, int d, int8_t* codes, float* scales, cudaStream_t stream)
{
    ProfileScope scope(RIB_KERNEL_CHECKPOINT_STORE, stream);
    if (d % 8) {
        rib_checkpoint_store_staged_kernel<<<(unsigned)((rows + kStagedRows - 1) / kStagedRows), kThreads, 0, stream>>>(x, rows, d, codes, scales);
    } else {
        const bool wide = d % 16 == 0;
        const int lanes = wide ? lanes_of(d / 2) : lanes_of(d);
        const auto kernel = wide ? (lanes == 1 ? rib_checkpoint_store_kernel<1, 2> : lanes == 2 ? rib_checkpoint_store_kernel<2, 2> : rib_checkpoint_store_kernel<4, 2>)
                                 : (lanes == 1 ? rib_checkpoint_store_kernel<1, 1> : lanes == 4 ? rib_checkpoint_store_kernel<4, 1> : rib_checkpoint_store_kernel<8, 1>);
        const long long per = (long long)kStoreUnroll * kThreads / lanes;
        kernel<<<(unsigned)((rows + per - 1) / per), kThreads, 0, stream>>>(x, rows, d, codes, scales);
    }
    return cudaGetLastError();
}

cudaError_t checkpoint_restore(const CheckpointRows* tensors, int count, long long rows, int d, cudaStream_t stream)
{
    RestoreArgs args{};
    for (int i = 0; i < count; ++i) args.t[i] = tensors[i];
    ProfileScope scope(RIB_KERNEL_CHECKPOINT_RESTORE, stream);
    if (d % 8) {
        rib_checkpoint_restore_staged_kernel<<<dim3((unsigned)((rows + kStagedRows - 1) / kStagedRows), (unsigned)count), kThreads, 0, stream>>>(args, rows, d);
    } else {
        const int lanes = lanes_of(d);
        const auto kernel = lanes == 1 ? rib_checkpoint_restore_kernel<1> : lanes == 2 ? rib_checkpoint_restore_kernel<2> : lanes == 4 ? rib_checkpoint_restore_kernel<4> : rib_checkpoint_restore_kernel<8>;
        kernel<<<dim3(restore_blocks(rows, lanes, count), (unsigned)count), kThreads, 0, stream>>>(args, rows, d);
    }
    return cudaGetLastError();
}

cudaError_t checkpoint_restore_wide(const CheckpointRows* tensors, long long rows, int d, cudaStream_t stream)
{
    RestoreArgs args{};
    for (int i = 0; i < 4; ++i) args.t[i] = tensors[i];
    ProfileScope scope(RIB_KERNEL_CHECKPOINT_RESTORE, stream);
    rib_checkpoint_restore_wide_kernel<<<(unsigned)((4 * rows + kThreads - 1) / kThreads), kThreads, 0, stream>>>(args, rows, d);
    return cudaGetLastError();
}

}  // namespace rib
