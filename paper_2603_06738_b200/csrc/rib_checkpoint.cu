// Activation checkpoints in 8 bits: a row of d channels of one token and head becomes d whole numbers -127 .. 127 and one fp32 scale,
//     scale = max_c |x_c| * (1/127),   code_c = round(x_c / scale),   restored x_c = bf16(code_c * scale),
// rounding half to even, division and products as IEEE fp32.  A row of zeros has scale 0; a row with an infinity or a NaN gets the scale
// NaN and comes back as NaN, so that an overflow is not lost on the way through the checkpoint.
#include "rib_common.cuh"

namespace rib {
namespace {

constexpr int kThreads = 256;

// One warp per row, a lane per two channels (d <= 64).
__global__ void __launch_bounds__(kThreads) rib_checkpoint_store_kernel(const __nv_bfloat16* x, long long rows, int d, int8_t* codes, float* scales)
{
    const long long row = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    if (row >= rows) return;
    const float a = lane < d ? __bfloat162float(x[row * d + lane]) : 0.f;
    const float b = lane + 32 < d ? __bfloat162float(x[row * d + lane + 32]) : 0.f;
    float most = fmaxf(fabsf(a), fabsf(b));
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    const bool bad = __any_sync(0xffffffffu, !isfinite(a) || !isfinite(b));
    const float scale = bad ? __int_as_float(0x7fffffff) : most * (1.f / 127.f);
    const bool zero = bad || scale == 0.f;
    if (lane < d) codes[row * d + lane] = zero ? 0 : (int8_t)__float2int_rn(__fdiv_rn(a, scale));
    if (lane + 32 < d) codes[row * d + lane + 32] = zero ? 0 : (int8_t)__float2int_rn(__fdiv_rn(b, scale));
    if (lane == 0) scales[row] = scale;
}

struct RestoreArgs { CheckpointRows t[4]; };

__global__ void __launch_bounds__(kThreads) rib_checkpoint_restore_kernel(const RestoreArgs args, long long rows, int d)
{
    const CheckpointRows t = args.t[blockIdx.y];
    const long long row = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    if (row >= rows) return;
    const float scale = t.scales[row];
    for (int c = lane; c < d; c += 32) t.x[row * d + c] = __float2bfloat16_rn((float)t.codes[row * d + c] * scale);
}

}  // namespace

cudaError_t checkpoint_store(const __nv_bfloat16* x, long long rows, int d, int8_t* codes, float* scales, cudaStream_t stream)
{
    const unsigned blocks = (unsigned)((rows * 32 + kThreads - 1) / kThreads);
    { ProfileScope scope(RIB_KERNEL_CHECKPOINT_STORE, stream); rib_checkpoint_store_kernel<<<blocks, kThreads, 0, stream>>>(x, rows, d, codes, scales); }
    return cudaGetLastError();
}

cudaError_t checkpoint_restore(const CheckpointRows* tensors, int count, long long rows, int d, cudaStream_t stream)
{
    RestoreArgs args{};
    for (int i = 0; i < count; ++i) args.t[i] = tensors[i];
    const dim3 grid((unsigned)((rows * 32 + kThreads - 1) / kThreads), (unsigned)count);
    { ProfileScope scope(RIB_KERNEL_CHECKPOINT_RESTORE, stream); rib_checkpoint_restore_kernel<<<grid, kThreads, 0, stream>>>(args, rows, d); }
    return cudaGetLastError();
}

}  // namespace rib
