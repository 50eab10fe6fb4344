// Gradient of a learned bias by buckets.  The backward kernels sum dS by offset (key minus query position); here the sums of a
// bucket's offsets are added up, over all heads where they share one table, and rounded once to the table's type.  The adds are made in 64 bits, in
// which their order changes nothing that is left after the rounding to 32 or 16.
#include "rib_common.cuh"

namespace rib {
namespace {

constexpr int kThreads = 256;

__global__ void __launch_bounds__(kThreads) rib_bias_scatter_kernel(const BiasScatter s) 
{
    cudaGridDependencySynchronize();
    bias_scatter(s, (size_t)blockIdx.x * kThreads + threadIdx.x);
}

__global__ void __launch_bounds__(kThreads) rib_bias_convert_kernel(const double* tables, int num_buckets, size_t entries, void* dbias, int bf16, long long head_stride)
{
    cudaGridDependencySynchronize();              // (it may have overtaken the kernel that sums)
    const size_t e = (size_t)blockIdx.x * kThreads + threadIdx.x;
    if (e >= entries) return;
    const size_t to = (e / num_buckets) * (size_t)head_stride + e % num_buckets;
    if (bf16) static_cast<__nv_bfloat16*>(dbias)[to] = __double2bfloat16(tables[e]);
    else static_cast<float*>(dbias)[to] = (float)tables[e];
}

}  // namespace

BiasGrad bias_grad_layout(int heads, int tables, int M, int num_buckets, void* base)
{
    const size_t side = 2 * M - 1, across = M % 8 ? 0 : 2 * (M / 8) - 1;
    const size_t by_offset = sizeof(double) * heads * side * side, by_block = sizeof(float) * 256 * heads * across * across;
    BiasGrad g;
    const size_t area = by_offset > by_block ? by_offset : by_block;
    g.offsets = static_cast<double*>(base);
    g.blocks = static_cast<float*>(base);
    g.tables = reinterpret_cast<double*>(static_cast<unsigned char*>(base) + area);
    g.bytes = area + sizeof(double) * (size_t)tables * num_buckets;
    return g;
}

cudaError_t bias_grad_clear(const BiasGrad& g, cudaStream_t stream) { return cudaMemsetAsync(g.offsets, 0, g.bytes, stream); }

cudaError_t bias_grad_scatter(const Problem& p, const BiasGrad& g, cudaStream_t stream)
{
    const BiasScatter s = bias_scatter_args(p, g, false);
    const size_t threads = (size_t)p.heads * s.side * s.side;
    ProfileScope scope(RIB_KERNEL_BIAS_FINISH, stream);
    return launch_overtaking(rib_bias_scatter_kernel, (int)((threads + kThreads - 1) / kThreads), kThreads, 0, stream, s);
}

cudaError_t bias_grad_convert(const Problem& p, const BiasGrad& g, cudaStream_t stream)
{
    const size_t entries = (size_t)bias_tables(p) * p.num_buckets;
    ProfileScope scope(RIB_KERNEL_BIAS_FINISH, stream);
    return launch_overtaking(rib_bias_convert_kernel, (int)((entries + kThreads - 1) / kThreads), kThreads, 0, stream, static_cast<const double*>(g.tables), p.num_buckets, entries,
                             p.dbias, p.bias_bf16, p.bias_head_stride);
}

}  // namespace rib
