// Attention of a map's tokens to a sequence of states of another length: what the forward and the backward kernels share.
//
//     S = q k^T / sqrt(d) over the keys j < length,   out = SoftMax(S) v,   lse = log sum exp S
//
// q [B][H][W][heads][d]; k, v [contexts][L][kv_heads][d], contexts = B, or 1 when the maps of the batch share one sequence: the batch is then one map of B H W
// tokens, which is the same memory.  heads / kv_heads = G query heads share a head of keys and values; the rows of a (context, kv head) group are its
// tokens times its G heads, token by token, and that is one TMA box {d, G heads, 128 / G tokens} per tile of up to 128 rows.
// Every kernel may start under the one before it on the stream, waits for its end before it reads what that may have written, and reads that by plain loads: the read-only path is for what nothing writes while
// a kernel is there.  The one exception is dQ over long sequences (rib_cross_bwd_sm100.cu), which runs beside the kernel before it, reads nothing of it, and relies on that one's wait.
#pragma once
#include "rib_sm100_common.cuh"

namespace rib {

struct CrossProblem {
    const __nv_bfloat16 *q, *k, *v;       // rows of `width` channels
    const __nv_bfloat16 *out, *dout;      // backward; rows of d channels (out, but in the short form) and `width` channels
    const float* lse_in;                  // backward
    const int* lengths;                   // [contexts], or null: L
    __nv_bfloat16 *out_w, *dq, *dk, *dv;  // rows of d channels
    float* lse_w;                         // may be null
    int B, heads, kv_heads, d, L, contexts;
    int width;                            // channels of a row in what is read by TMA: d, or d rounded up to a multiple of 8 on padded copies
    long long pixels, tokens;             // H W; tokens per context (pixels, or B pixels when the context is shared)
    int* status;
    bool exact_softmax;                   // forward: the exact form for every item
    void* workspace;
};

// sizes of the launches, from the shape alone
struct CrossPlan {
    int G, rows_per_tile, tokens_per_tile, tiles, pairs, groups;       // groups: contexts x kv_heads; pairs: of tiles
    long long rows;                                                    // of a group: tokens x G
    int splits, blocks_per_split;                                      // forward: runs of blocks of 128 keys that are computed apart and joined
    int dq_tiles, dq_splits, dq_blocks_per_split;                      // dQ: tiles of two row tiles, and such runs of blocks of 64
    int key_tiles, row_splits, row_tiles_per_split;                    // dK and dV: tiles of 128 keys, runs of tiles of 64 rows
    int row_tiles, kv_rows_per_tile, kv_tokens_per_tile;
    bool short_bwd;                                                    // backward in one kernel; dK and dV: a CTA has all keys, and row_tiles_per_split is even
    bool few_rows;                                                     // forward on the plain pipes; splits are then runs of a context's own keys
};

constexpr int kCrossSms = 148;            // the same number everywhere, so that a call's shape decides the launch
constexpr int kCrossBlock = 64;           // keys of a block
// Rows of a group (tokens x heads that share a head of keys) up to which the forward pass takes the plain pipes.  Plain pipes / tensor cores, us with the join: 64 contexts of 64 to 4096 states, 6 heads
// of keys of 32, 1 row 31 / 80, 2 rows 35 / 81; 16 contexts of 256 to 4096, 2 heads of 64, 1 row 12 / 17, 2 rows 12 / 18, 4 rows 18.5 / 17.5, 8 rows 33 / 17.
// (Figures of whole calls here and in the kernels' files, where nothing else is said: us of a call among others, each behind a write of 256 MB, which is still on its way to memory while the call reads.)
constexpr int kCrossFewRows = 2;
// Weights are held down by a power of two, 2^-cross_bits(their number), where they are added up with values: every sum is then one of a weighted mean and stays in range if the values do.
inline int cross_bits(long long n) { int b = 0; while ((1ll << b) < n) ++b; return b; }
// States up to which the forward pass takes a row's scores at once (rib_cross_short_sm100.cu has both sides); 128 columns of tensor memory for each of four tiles are all there is.
constexpr int kCrossShort = 128;

CrossPlan cross_plan(const CrossProblem& p);
bool cross_padded(const CrossProblem& p);                                       // rows that TMA cannot address: copies filled up with zero channels
size_t cross_fwd_workspace(const CrossProblem& p);
size_t cross_bwd_workspace(const CrossProblem& p);
cudaError_t cross_fwd(CrossProblem p, cudaStream_t stream, int* launches);
cudaError_t cross_bwd(CrossProblem p, cudaStream_t stream, int* launches);
// Forward over up to kCrossShort keys (rib_cross_short_sm100.cu).
cudaError_t cross_fwd_short(const CrossProblem& p, const CrossPlan& plan, cudaStream_t stream);
// Backward where cross_plan says short_bwd, without the sum of the splits (rib_cross_short_bwd_sm100.cu).
cudaError_t cross_bwd_short(const CrossProblem& p, const CrossPlan& plan, float* part_dk, float* part_dv, cudaStream_t stream);
// Forward of few rows (rib_cross_rows.cu), without the join of the splits, whose outputs are rows of `stride` floats.
cudaError_t cross_fwd_rows(const CrossProblem& p, const CrossPlan& plan, float* part_out, float* part_lse, int stride, cudaStream_t stream);

// Fills up rows of d channels with zeros to rows of `width`, up to five tensors in one launch (rib_cross_fwd_sm100.cu).
struct CrossPad { const __nv_bfloat16* src[5]; __nv_bfloat16* dst[5]; long long rows[5]; int tensors, d, width; };
cudaError_t cross_pad(const CrossPad& args, cudaStream_t stream);

namespace sm100 {

inline size_t cross_align(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// bf16 [contexts][tokens][heads][width], box = `tokens_in_box` tokens of `heads_in_box` heads, DP channels wide (zeros beyond the width)
inline bool cross_rows_map(CUtensorMap* map, const void* ptr, long long contexts, long long tokens, int heads, int width, int dp, int heads_in_box, int tokens_in_box)
{
    const MapKey key{ptr, contexts, tokens, 6, heads, width, dp, heads_in_box, tokens_in_box};
    return cached_map(map, key, [&](CUtensorMap* m) {
        const cuuint64_t row = (cuuint64_t)width * 2;
        const cuuint64_t dims[4] = {(cuuint64_t)width, (cuuint64_t)heads, (cuuint64_t)tokens, (cuuint64_t)contexts};
        const cuuint64_t strides[3] = {row, row * heads, row * heads * (cuuint64_t)tokens};
        const cuuint32_t box[4] = {(cuuint32_t)dp, (cuuint32_t)heads_in_box, (cuuint32_t)tokens_in_box, 1};
        const cuuint32_t estr[4] = {1, 1, 1, 1};
        return encode_fn()(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           dp == 16 ? CU_TENSOR_MAP_SWIZZLE_32B : dp == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    });
}

// Tiles of rows of DP = 32 or 64 channels in shared memory: 64-byte rows under SWIZZLE_64B, 128-byte rows under SWIZZLE_128B; eight rows are
// an atom.  The same descriptor serves a K-major operand (a K16 step is 32 bytes on) and an MN-major one whose contraction runs over the rows (16 rows on).
template <int DP> struct CrossTile {
    static constexpr uint32_t kRow = DP * 2;
    static constexpr uint64_t kDesc = smem_desc_const(16, 8 * kRow, DP == 32 ? kSwizzle64B : kSwizzle128B);
    static constexpr uint32_t kStepK = 2, kStepRows = kRow;            // in units of 16 bytes: 32 bytes; 16 rows
};

// scores of one lowest finite reference: a row whose keys all give minus infinity (infinite inputs) has weights 0 and 0 / 0 as its result
constexpr float kCrossLowest = -1.8e38f;

// `count` (a multiple of 8) fp32 values as bf16 to dst, of a row of d channels beginning at channel c0; `vector`: rows are whole 16-byte words
template <int count>
__device__ __forceinline__ void cross_store_row(__nv_bfloat16* row, int c0, int d, const float (&x)[count], bool vector)
{
    if (vector) {
#pragma unroll
        for (int g = 0; g < count / 8; ++g)
            if (c0 + 8 * g < d)
                *reinterpret_cast<uint4*>(row + c0 + 8 * g) = make_uint4(pack_bf16x2(x[8 * g], x[8 * g + 1]), pack_bf16x2(x[8 * g + 2], x[8 * g + 3]),
                                                                         pack_bf16x2(x[8 * g + 4], x[8 * g + 5]), pack_bf16x2(x[8 * g + 6], x[8 * g + 7]));
    } else {
#pragma unroll
        for (int e = 0; e < count; ++e)
            if (c0 + e < d) row[c0 + e] = __float2bfloat16_rn(x[e]);
    }
}

// Rows of a tile that no token fills are zero for good, since the boxes end before them; a tile of shared memory that a role
// writes by hand is handed over to the asynchronous copies and products by the fence.
__device__ __forceinline__ void cross_zero_rows(uint8_t* tile, uint32_t row_bytes, int first, int last, int thread, int threads)
{
    uint4* at = reinterpret_cast<uint4*>(tile + (size_t)first * row_bytes);
    const int words = (last - first) * (int)(row_bytes / 16);
    for (int i = thread; i < words; i += threads) at[i] = make_uint4(0u, 0u, 0u, 0u);
}

}  // namespace sm100
}  // namespace rib
