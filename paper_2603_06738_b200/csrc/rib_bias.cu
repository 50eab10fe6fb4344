// Gradient of a learned bias by buckets.  The backward kernels sum dS by offset (key minus query position); here the sums of a
// bucket's offsets are added up, over all heads where they share one table, and rounded once to the table's type.
#include "rib_common.cuh"

namespace rib {
namespace {

constexpr int kThreads = 256;

// One thread per (head, offset).  The sums are kept in 64 bits, in which the order of the adds changes nothing that is left after
// the rounding to 32 or 16; the block that is through last converts the tables.
__global__ void __launch_bounds__(kThreads) rib_bias_finish_kernel(const int* buckets, int num_buckets, int offsets, int heads, int tables, BiasGrad g,
                                                                   void* dbias, int bf16, long long head_stride)
{
    const size_t t = (size_t)blockIdx.x * kThreads + threadIdx.x;
    if (t < (size_t)heads * offsets) {
        const int h = (int)(t / offsets), u = buckets[t % offsets];
        if ((unsigned)u < (unsigned)num_buckets) atomicAdd(g.tables + (size_t)(tables > 1 ? h : 0) * num_buckets + u, g.offsets[t]);
    }
    __shared__ bool last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(g.done, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    for (size_t e = threadIdx.x; e < (size_t)tables * num_buckets; e += kThreads) {
        const size_t to = (e / num_buckets) * (size_t)head_stride + e % num_buckets;
        const double sum = __ldcg(g.tables + e);
        if (bf16) static_cast<__nv_bfloat16*>(dbias)[to] = __double2bfloat16(sum);
        else static_cast<float*>(dbias)[to] = (float)sum;
    }
}

}  // namespace

BiasGrad bias_grad_layout(int heads, int tables, int M, int num_buckets, void* base)
{
    const size_t offsets = (size_t)heads * (2 * M - 1) * (2 * M - 1), entries = (size_t)tables * num_buckets;
    BiasGrad g;
    g.offsets = static_cast<double*>(base);
    g.tables = g.offsets + offsets;
    g.done = reinterpret_cast<unsigned*>(g.tables + entries);
    g.bytes = sizeof(double) * (offsets + entries + 1);
    return g;
}

cudaError_t bias_grad_clear(const BiasGrad& g, cudaStream_t stream) { return cudaMemsetAsync(g.offsets, 0, g.bytes, stream); }

cudaError_t bias_grad_finish(const Problem& p, const BiasGrad& g, cudaStream_t stream)
{
    const int offsets = (2 * p.M - 1) * (2 * p.M - 1);
    const unsigned blocks = (unsigned)(((size_t)p.heads * offsets + kThreads - 1) / kThreads);
    { ProfileScope scope(RIB_KERNEL_BIAS_FINISH, stream);
      rib_bias_finish_kernel<<<blocks, kThreads, 0, stream>>>(p.buckets, p.num_buckets, offsets, p.heads, bias_tables(p), g, p.dbias, p.bias_bf16, p.bias_head_stride); }
    return cudaGetLastError();
}

}  // namespace rib
