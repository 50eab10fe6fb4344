// Shared declarations of the RIB window-attention CUDA library (internal; the public surface is
// include/rib_window_attn.h).
#pragma once
#include "../../include/rib_window_attn.h"
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <stddef.h>
#include <stdint.h>

namespace rib {

// A tensor of rows kept in 8 bits (codes, a scale per row) and where its bf16 form goes.
struct CheckpointRows { const int8_t* codes; const float* scales; __nv_bfloat16* x; };

// One problem instance.  Image tensors are bf16 [B][H][W][heads][d]; pq/pk bf16 [n][r];
// lse / rowdot fp32 [B][heads][H][W]; dpq/dpk fp32 [n][r].
struct Problem {
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    const __nv_bfloat16* pq;
    const __nv_bfloat16* pk;
    const __nv_bfloat16* gate;  // forward: optional CLA gate multiplied into the output (Eq. 9), layout of out
    const __nv_bfloat16* out;   // forward result (input of the backward pass)
    const __nv_bfloat16* dout;
    const float* lse_in;        // backward
    __nv_bfloat16* out_w;       // forward output
    float* lse_w;               // forward output, may be null
    __nv_bfloat16* dq;
    __nv_bfloat16* dk;
    __nv_bfloat16* dv;
    float* dpq;
    float* dpk;
    float* rowdot;              // any-shape backward: D_i = sum_c dout_ic * out_ic, image layout of lse
    void* workspace;            // caller's scratch (backward), 256-byte aligned
    size_t workspace_bytes;
    long long pos_head_stride;        // elements between the heads' tables in pq/pk/dpq/dpk; 0 = one table for all heads
    int B, H, W, heads, d, r, M, s;   // M = window side, s = cyclic shift
    int Hp, Wp;                       // sides of the map the windows are laid over: H, W rounded up to multiples of M
                                      // (positions with Y >= H or X >= W are not tokens); equal to H, W in the plain calls
    int n, nWy, nWx, pairs;           // n = M*M, windows per image, B*nWy*nWx*heads
    int* status;                      // device status word (bounded waits report here)
    bool exact_softmax;               // tcgen05 forward: every item takes the exact (running-maximum) softmax form
    bool masked;                      // shifted windows: the wrapped parts of a border window do not attend to each other
    int d_true, r_true;               // tcgen05 kernels on zero-padded copies (rib_repack.cu): the widths the scales 1/sqrt(d),
                                      // 1/sqrt(r) are taken from; 0 = d, r themselves
    // learned bias by buckets in place of the rank-r tables (then r = 0); null: none
    const void* bias;                 // [heads][num_buckets], bias_head_stride elements apart (0: one table for all heads)
    int bias_bf16;                    // 1: bf16, 0: fp32
    long long bias_head_stride;
    const int* buckets;               // [2M-1][2M-1]: bucket of the offset (key - query); outside [0, num_buckets): not attended to
    int num_buckets;
    void* dbias;                      // gradient, layout and type of bias
    const CheckpointRows* saved;      // backward: q, k, v, out as checkpoints, which the preparation kernel restores (q, k, v) and uses (out); null: not
    int qk_width;                     // backward from checkpoints, narrow heads: q and k lie in rows of that width (restored_width); 0: d
    int narrow;                       // general tcgen05 backward on such copies: width of the rows of `out` and `dq`, which are the caller's; 0 = d
};

// Pq/Pk tables: one shared by the heads, or one per head (Sec. 3.1, after Eq. 3: head-wise projections of the shared h).
inline int pos_tables(const Problem& p) { return p.pos_head_stride ? p.heads : 1; }
// Elements from the first entry of the first table to the end of the last one.
inline size_t pos_extent(const Problem& p)
{
    return (size_t)(pos_tables(p) - 1) * (size_t)p.pos_head_stride + (size_t)p.n * p.r;
}

// Tables of a bias by buckets: one for all heads or one per head.
inline int bias_tables(const Problem& p) { return p.bias_head_stride ? p.heads : 1; }

// A bias of kBiasMasked or less takes its pair out of the softmax, as minus infinity does: the lowest value of a type, the usual stand-in for
// minus infinity, means the same, and what is left stays far from overflow when it is scaled by log2(e).
constexpr float kBiasMasked = -1e30f;

__device__ __forceinline__ float bias_at(const void* bias, int bf16, long long at)
{
    const float b = bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(bias)[at]) : static_cast<const float*>(bias)[at];
    return b <= kBiasMasked ? -INFINITY : b;
}

// The head width and the rank that the scales of Eq. 6 are taken from.
inline float scale_width_d(const Problem& p) { return (float)(p.d_true ? p.d_true : p.d); }
inline float scale_width_r(const Problem& p) { return (float)(p.r_true ? p.r_true : p.r); }

// Launchers; each returns the cudaError_t of its launches.
cudaError_t generic_fwd(const Problem& p, cudaStream_t stream);
cudaError_t generic_bwd(const Problem& p, cudaStream_t stream, double* offset_sums = nullptr);     // offset_sums: BiasGrad::offsets
cudaError_t rowdot_prepass(const Problem& p, cudaStream_t stream);

// The gradient of a bias by buckets (rib_bias.cu): its scratch lies at the end of a backward workspace and starts at zero.  The any-shape
// kernels sum dS by offset, in 64 bits; the tcgen05 kernels by the difference of 8 x 8 patches, [heads][(2M/8-1)^2] blocks of 16 x 16 fp32 with the
// differences -8 .. 7 of rows and columns inside them, of which an offset has up to four.
struct BiasGrad {
    double* offsets;      // [heads][(2M-1)^2]
    float* blocks;        // in the same place
    double* tables;       // [tables][num_buckets]
    size_t bytes;
};
BiasGrad bias_grad_layout(int heads, int tables, int M, int num_buckets, void* base);
cudaError_t bias_grad_clear(const BiasGrad& g, cudaStream_t stream);
// Adds the sums of a bucket's offsets (thread `t` of heads * (2M-1)^2).
struct BiasScatter { const int* buckets; double* tables; const double* offsets; const float* blocks; int num_buckets, side, heads, shared; };
inline BiasScatter bias_scatter_args(const Problem& p, const BiasGrad& g, bool blocked)
{
    return {p.buckets, g.tables, blocked ? nullptr : g.offsets, blocked ? g.blocks : nullptr, p.num_buckets, 2 * p.M - 1, p.heads, bias_tables(p) == 1 ? 1 : 0};
}
__device__ inline void bias_scatter(const BiasScatter& s, size_t t)
{
    const int entries = s.side * s.side;
    if (t >= (size_t)s.heads * entries) return;
    const int h = (int)(t / entries), e = (int)(t % entries), u = s.buckets[e];
    if ((unsigned)u >= (unsigned)s.num_buckets) return;
    double sum = 0.0;
    if (s.blocks) {
        const int M = (s.side + 1) / 2, across = 2 * (M / 8) - 1, oy = e / s.side + 1, ox = e % s.side + 1;       // (+ M - 1 - offset) + 1: 1 .. 2M - 1
        // oy = 8 (patches + M / 8 - 1) + row + 8 with row -8 .. 7: block oy / 8 - 1 with row oy % 8, block oy / 8 with row oy % 8 - 8
        for (int by = oy / 8 - 1; by <= oy / 8; ++by)
            for (int bx = ox / 8 - 1; bx <= ox / 8; ++bx)
                if (by >= 0 && by < across && bx >= 0 && bx < across)
                    sum += (double)s.blocks[(((size_t)h * across + by) * across + bx) * 256 + (oy - 8 * by) * 16 + ox - 8 * bx];
    } else {
        sum = s.offsets[t];
    }
    atomicAdd(s.tables + (size_t)(s.shared ? 0 : h) * s.num_buckets + u, sum);
}
cudaError_t bias_grad_scatter(const Problem& p, const BiasGrad& g, cudaStream_t stream);        // sums by offset -> tables
cudaError_t bias_grad_convert(const Problem& p, const BiasGrad& g, cudaStream_t stream);        // tables -> dbias
// Windows of up to 256 tokens outside the tcgen05 kernels' shapes (rib_bias_small.cu).
bool bias_small_supported(const Problem& p);
cudaError_t bias_small_fwd(const Problem& p, cudaStream_t stream);
cudaError_t bias_small_bwd(const Problem& p, double* offset_sums, cudaStream_t stream);
bool sm100_bias_fwd_supported(const Problem& p);
cudaError_t sm100_bias_fwd(const Problem& p, cudaStream_t stream);
bool sm100_bias_bwd_supported(const Problem& p);
size_t sm100_bias_bwd_workspace_bytes(long long pairs, int n);
cudaError_t sm100_bias_bwd(const Problem& p, const BiasGrad& grad, cudaStream_t stream);       // 4 kernels

// Rows of bf16 as whole numbers of 8 bits with a scale each, and back (rib_checkpoint.cu).
cudaError_t checkpoint_store(const __nv_bfloat16* x, long long rows, int d, int8_t* codes, float* scales, cudaStream_t stream);
cudaError_t checkpoint_restore(const CheckpointRows* tensors, int count, long long rows, int d, cudaStream_t stream);
cudaError_t checkpoint_restore_wide(const CheckpointRows* tensors, long long rows, int d, cudaStream_t stream);      // q, k (restore_wide), v, out
// byte `at` of four codes as a float: 0x4B000000 + (code + 128) is 2^23 + 128 + code
__device__ __forceinline__ float code_value(uint32_t codes_plus_128, int at)
{
    return __uint_as_float(__byte_perm(codes_plus_128, 0x4B000000u, 0x7440 + at)) - 8388736.f;
}

__device__ __forceinline__ uint32_t restored_pair(uint32_t codes, int at, float scale)       // codes at, at + 1 (bytes of the word, 128 added) as bf16
{
    const float lo = code_value(codes, at) * scale, hi = code_value(codes, at + 1) * scale;
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// eight codes of a row as bf16
__device__ __forceinline__ uint4 restored_chunk(uint2 codes, float scale)
{
    codes.x ^= 0x80808080u; codes.y ^= 0x80808080u;
    return make_uint4(restored_pair(codes.x, 0, scale), restored_pair(codes.x, 2, scale), restored_pair(codes.y, 0, scale), restored_pair(codes.y, 2, scale));
}

// Narrow heads.  A logit of 8 or 16 channels is a sum of few products, the largest logits have the largest errors, and with q and k rounded to bf16 the gradients are further
// off than a backward pass's own roundings put them (dq 5.7e-3 in relative L2 of 5e-3).  So for the tcgen05 kernels q and k are restored to rows of 32 columns, which the tiles
// have anyhow, with what the rounding leaves (lo) in the free ones.  kLogits: q = hi lo hi 0, k = hi hi lo 0 in pieces of the head's width (16 channels: the first two), so
// that a row of one times a row of the other is their product in 16 bits, or with 16 channels that with k rounded.  Else (16 channels under a bias, whose logits lose
// less): q = hi 0, k = hi lo, which leaves the logits as they are and puts the rest of dS k into columns 16 .. 31.
inline int restored_width(int d) { return d == 8 || d == 16 ? 32 : d; }
__device__ __forceinline__ void restored_parts(uint2 codes, float scale, uint4& hi, uint4& lo)
{
    hi = restored_chunk(codes, scale);
    const uint32_t c[2] = {codes.x ^ 0x80808080u, codes.y ^ 0x80808080u}, h[4] = {hi.x, hi.y, hi.z, hi.w};
    uint32_t rest[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = code_value(c[i >> 1], 2 * (i & 1)) * scale, b = code_value(c[i >> 1], 2 * (i & 1) + 1) * scale;
        const __nv_bfloat162 v = __floats2bfloat162_rn(a - __uint_as_float(h[i] << 16), b - __uint_as_float(h[i] & 0xffff0000u));
        rest[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    lo = make_uint4(rest[0], rest[1], rest[2], rest[3]);
}
// 8 channels `part` (0 .. 3) of the wide rows of token `tok` of q and k, heads of d channels
template <bool kLogits>
__device__ __forceinline__ void restore_wide(const CheckpointRows* qk, size_t tok, int d, int part)
{
    const int chunk = d == 16 ? part & 1 : 0, copy = d == 16 ? part >> 1 : part;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint4 hi, lo;
        restored_parts(__ldg(reinterpret_cast<const uint2*>(qk[i].codes + tok * d) + chunk), __ldg(qk[i].scales + tok), hi, lo);
        const bool is_hi = copy == 0 || (kLogits && copy == 2 - i), is_lo = kLogits ? copy == 1 + i : copy == 1 && i == 1;
        reinterpret_cast<uint4*>(qk[i].x + tok * 32)[part] = is_hi ? hi : is_lo ? lo : make_uint4(0u, 0u, 0u, 0u);
    }
}

bool sm100_fwd_supported(const Problem& p);
cudaError_t sm100_fwd(const Problem& p, cudaStream_t stream);
// Frames with a side that is no multiple of 8, at the precision of the any-shape kernel (rib_fwd_frame_sm100.cu).
bool sm100_frame_supported(const Problem& p);
cudaError_t sm100_fwd_frame(const Problem& p, cudaStream_t stream);
bool sm100_bwd_supported(const Problem& p);
size_t sm100_bwd_workspace_bytes(long long pairs, int n, int tables, int r);
cudaError_t sm100_bwd(const Problem& p, cudaStream_t stream);
int sm100_bwd_launches(const Problem& p);     // kernels it enqueues
bool sm100_bwd_takes_narrow(const Problem& p);    // Problem::narrow may be set
bool sm100_bwd_takes_saved(const Problem& p);     // Problem::saved may be set
// Windows of 8 x 8 tokens (rib_window8_sm100.cu); the backward launches 2 kernels.
bool sm100_window8(const Problem& p);
cudaError_t sm100_window8_fwd(const Problem& p, cudaStream_t stream);
cudaError_t sm100_window8_bwd(const Problem& p, cudaStream_t stream);
// Windows of 16 x 16 tokens (rib_window16_sm100.cu); the backward launches 3 kernels.
bool sm100_window16(const Problem& p);
bool sm100_window16_prefers(const Problem& p);        // ... the forward kernel
cudaError_t sm100_window16_fwd(const Problem& p, cudaStream_t stream);
cudaError_t sm100_window16_bwd(const Problem& p, cudaStream_t stream);
// Even head widths and ranks up to 32 whose rows TMA cannot address (60-byte rows of d = 30, 36-byte rows of r = 18):
// the tensors are copied into zero-padded scratch (stream-ordered allocation), the tcgen05 kernels run on the copies,
// and the results are copied back.  `launches` receives the number of kernels enqueued.
// The forward pass takes frames of any size, the backward pass sides that are multiples of 8.
bool sm100_repack_fwd_supported(const Problem& p);
bool sm100_repack_bwd_supported(const Problem& p);
int repacked_width(int w);                    // the next multiple of 8
cudaError_t sm100_fwd_repacked(const Problem& p, cudaStream_t stream, int* launches);
cudaError_t sm100_bwd_repacked(const Problem& p, cudaStream_t stream, int* launches);

// Channel counts the gate kernels do not take (even D up to 192): zero-padded copies in the library's scratch pool.
int cla_padded_channels(int D);               // 64, 128 or 192; 0 = not paddable
cudaError_t cla_gate_padded(const __nv_bfloat16* x, const float* w_dw, const float* b_dw, const float* w_pw, const float* b_pw, int B, int H,
                            int W, int D, __nv_bfloat16* gate, int* status, cudaStream_t stream, int* launches);
cudaError_t cla_gate_bwd_padded(const __nv_bfloat16* x, const float* w_dw, const float* b_dw, const float* w_pw, const float* b_pw,
                                const __nv_bfloat16* dgate, int B, int H, int W, int D, __nv_bfloat16* dx, float* dw_dw, float* db_dw,
                                float* dw_pw, float* db_pw, void* workspace, bool tensor_cores, int* status, cudaStream_t stream, int* launches);
bool cla_gate_supported(int H, int W, int D);
cudaError_t cla_gate(const __nv_bfloat16* x, const float* w_dw, const float* b_dw, const float* w_pw, const float* b_pw, int B, int H,
                     int W, int D, __nv_bfloat16* gate, int* status, cudaStream_t stream);

// Backward of the CLA gate (Eq. 8) and the product of Eq. 9 with its chain rule (dout_gated == nullptr: forward product).
bool cla_gate_bwd_supported(int D);
size_t cla_gate_bwd_workspace_bytes(long long pixels, int D);
cudaError_t cla_gate_bwd(const __nv_bfloat16* x, const float* w_dw, const float* b_dw, const float* w_pw, const float* b_pw,
                         const __nv_bfloat16* dgate, int B, int H, int W, int D, __nv_bfloat16* dx, float* dw_dw, float* db_dw,
                         float* dw_pw, float* db_pw, void* workspace, bool tensor_cores, int* status, cudaStream_t stream);
cudaError_t cla_product(const __nv_bfloat16* out, const __nv_bfloat16* gate, const __nv_bfloat16* dout_gated, long long count,
                        __nv_bfloat16* res0, __nv_bfloat16* res1, cudaStream_t stream);

bool generator_supported(int window, int L, int dh, int r);
cudaError_t generator_fwd(const float* w_h, const float* b_h, const float* w_pq, const float* w_pk, int window, int L, int dh, int r,
                          __nv_bfloat16* pq, __nv_bfloat16* pk, cudaStream_t stream);
cudaError_t generator_bwd(const float* w_h, const float* b_h, const float* w_pq, const float* w_pk, const float* dpq, const float* dpk,
                          int window, int L, int dh, int r, float* dw_h, float* db_h, float* dw_pq, float* dw_pk, cudaStream_t stream);

// Norms of queries and keys for each head and the rotation by position (rib_rope.cu).
struct RopeRows { const __nv_bfloat16 *x, *g; __nv_bfloat16* y; long long x_stride, y_stride; const float* w; float* dw; };      // y: result, or gradient of x; strides of tokens; w null: no norm
struct RopeProblem { RopeRows t[2]; const float* table; long long tokens; int H, W, heads, kv_heads, d, rot, interleaved, per_head; float eps; };      // q, k (kv_heads = 0: no k)
cudaError_t rope_table(const float* frequencies, int H, int W, int pairs, long long y0, long long x0, float magnitude, float* table, cudaStream_t stream);
cudaError_t qk_norm_rope_fwd(const RopeProblem& p, cudaStream_t stream);
size_t qk_norm_rope_bwd_workspace(const RopeProblem& p);
cudaError_t qk_norm_rope_bwd(const RopeProblem& p, float* workspace, int* launches, cudaStream_t stream);

// Hits and misses of the host-side tensor-map cache (rib_fwd_sm100.cu).
void tensor_map_cache_counts(long long* hits, long long* misses);

// Measurement / self-test kernels (rib_probe.cu).
cudaError_t exp_probe(float* sink, int blocks, int iters, cudaStream_t stream);
long long exp_probe_count(int blocks, int iters);
cudaError_t wait_probe(int* status, unsigned long long limit_ns, cudaStream_t stream);

// Per-kernel device timing (off unless rib_profile_begin was called): records a CUDA event on
// `stream` before (phase 0) and after (phase 1) the launch of kernel `kernel_id` (RIB_KERNEL_*).
void profile_mark(int kernel_id, int phase, cudaStream_t stream);
struct ProfileScope {
    int id; cudaStream_t stream;
    ProfileScope(int kernel_id, cudaStream_t s) : id(kernel_id), stream(s) { profile_mark(id, 0, stream); }
    ~ProfileScope() { profile_mark(id, 1, stream); }
};

// Launch of a kernel that may start while the kernel before it on the stream still runs (it waits for that one's end by itself).
template <typename Kernel, typename... Args>
inline cudaError_t launch_overtaking(Kernel kernel, dim3 grid, int threads, size_t smem, cudaStream_t stream, const Args&... args)
{
    cudaLaunchAttribute overtake;
    overtake.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overtake.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = dim3((unsigned)threads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    config.attrs = &overtake;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, args...);
}

// Window partition with cyclic shift: token i = y*M + x of window (wy, wx) -> image pixel.
__host__ __device__ inline void token_pixel(int H, int W, int M, int s, int wy, int wx, int i,
                                            int& Y, int& X)
{
    const int y = i / M, x = i - y * M;
    Y = wy * M + y + s; if (Y >= H) Y -= H;
    X = wx * M + x + s; if (X >= W) X -= W;
}

// Shifted windows with a mask: in the last window row (column) the positions from M - s on come from the other side of
// the map.  Part of a window position: bit 1 = wrapped rows, bit 0 = wrapped columns; two tokens of a window attend to each
// other when their parts are equal.
__host__ __device__ inline int window_part(int M, int s, bool last_wy, bool last_wx, int y, int x)
{
    return ((last_wy && y >= M - s) ? 2 : 0) | ((last_wx && x >= M - s) ? 1 : 0);
}

}  // namespace rib
