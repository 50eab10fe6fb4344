// C ABI of the RIB window-attention library: argument validation, kernel selection, status word.
// The contract of every entry point is stated in include/rib_window_attn.h.
#include "../../include/rib_window_attn.h"
#include "rib_common.cuh"

#include <atomic>
#include <mutex>
#include <vector>

namespace {

__device__ int g_status_word = 0;   // written by bounded device-side waits that ran out

std::atomic<int> g_forced_path{RIB_PATH_NONE};
thread_local int t_last_path = RIB_PATH_NONE;
std::atomic<long long> g_kernel_launches{0};

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_shape(int B, int H, int W, int heads, int d, int r, int window, int shift, bool partial_windows = false)
{
    if (B <= 0 || H <= 0 || W <= 0 || heads <= 0 || d <= 0 || r < 0 || window <= 0) return RIB_ERR_SHAPE;
    if (!partial_windows && (H % window || W % window)) return RIB_ERR_SHAPE;
    if (shift < 0 || shift >= window) return RIB_ERR_SHAPE;
    if (d > 64 || r > 64) return RIB_ERR_UNSUPPORTED;      // any width up to 64: the any-shape kernels read element by element
    // places of windows laid over the map, shifted and not yet wrapped, are ints
    const long long rows = ((long long)H + window - 1) / window, columns = ((long long)W + window - 1) / window;
    if ((rows + 1) * window > 0x7fffffffLL || (columns + 1) * window > 0x7fffffffLL) return RIB_ERR_UNSUPPORTED;
    if (rows * columns > 0x7fffffffLL || rows * columns * B > 0x7fffffffLL) return RIB_ERR_SHAPE;          // (each factor below 2^31: no product passes 64 bits)
    const long long pairs = rows * columns * B * heads;
    if (pairs > 0x7fffffffLL || (long long)window * window > (1 << 20)) return RIB_ERR_SHAPE;
    // launch limits of the kernels: the any-shape kernels put n / 16 row groups on grid.y, the tcgen05 kernels count
    // pairs * key blocks in an int
    const long long n = (long long)window * window;
    if (n > 65535LL * 16 || pairs * ((n + 127) / 128) > 0x7fffffffLL) return RIB_ERR_UNSUPPORTED;
    return RIB_OK;
}

// Device address of the status word on the current device; looked up once per device.
constexpr int kMaxStatusDevices = 64;
std::mutex g_status_mutex;
int* g_status_ptr[kMaxStatusDevices] = {};

int device_status_ptr(int** out)
{
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxStatusDevices) return RIB_ERR_CUDA;
    std::lock_guard<std::mutex> lock(g_status_mutex);
    if (!g_status_ptr[dev]) {
        void* ptr = nullptr;
        if (cudaGetSymbolAddress(&ptr, g_status_word) != cudaSuccess || !ptr) return RIB_ERR_CUDA;
        g_status_ptr[dev] = static_cast<int*>(ptr);
    }
    *out = g_status_ptr[dev];
    return RIB_OK;
}

void fill_shape(rib::Problem& p, int B, int H, int W, int heads, int d, int r, int window, int shift)
{
    p.B = B; p.H = H; p.W = W; p.heads = heads; p.d = d; p.r = r; p.M = window; p.s = shift;
    p.nWy = (int)(((long long)H + window - 1) / window); p.nWx = (int)(((long long)W + window - 1) / window);   // exact in the plain calls (H, W multiples of window)
    p.Hp = p.nWy * window; p.Wp = p.nWx * window;
    p.n = window * window;
    p.pairs = B * p.nWy * p.nWx * heads;
}

// A learned bias by buckets, which takes the place of the rank-r tables (r = 0).
struct BiasArgs { const void* table; int dtype; long long head_stride; const int* buckets; int num_buckets; };

int check_bias(const BiasArgs& b)
{
    if (!b.table || !b.buckets) return RIB_ERR_NULL;
    if (b.num_buckets <= 0 || b.head_stride < 0 || (b.head_stride && b.head_stride < b.num_buckets)) return RIB_ERR_SHAPE;
    if (b.dtype != RIB_DTYPE_F32 && b.dtype != RIB_DTYPE_BF16) return RIB_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(b.table) & (b.dtype == RIB_DTYPE_F32 ? 3u : 1u)) return RIB_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(b.buckets) & 3u) return RIB_ERR_ALIGN;
    return RIB_OK;
}

void fill_bias(rib::Problem& p, const BiasArgs& b)
{
    p.bias = b.table; p.bias_bf16 = b.dtype == RIB_DTYPE_BF16; p.bias_head_stride = b.head_stride;
    p.buckets = b.buckets; p.num_buckets = b.num_buckets;
}

int fwd_impl(const void* q, const void* k, const void* v, const void* pq, const void* pk, long long pos_head_stride, const void* gate,
             int B, int H, int W, int heads, int d, int r, int window, int shift, void* out, float* lse, void* stream,
             bool validate_only = false, bool masked = false, const BiasArgs* bias = nullptr);

int check_pos_stride(long long stride, int window, int r)
{
    if (stride == 0) return RIB_OK;
    if (stride < (long long)window * window * r || (stride & 7)) return RIB_ERR_SHAPE;
    return RIB_OK;
}

size_t rowdot_bytes(int B, int H, int W, int heads)
{
    const size_t bytes = sizeof(float) * (size_t)B * H * W * heads;
    return (bytes + 255) & ~(size_t)255;
}

// ---- per-kernel device timing (rib_profile_begin / rib_profile_end) ------------------------------
struct ProfileState {
    std::mutex mutex;
    bool on = false, pending = false;     // pending: a start event without its stop event yet
    int capacity = 0, count = 0;          // launches
    std::vector<cudaEvent_t> events;      // 2 per launch
    std::vector<int> ids;
};
ProfileState g_profile;
std::atomic<bool> g_profile_on{false};

// ---- built-in scratch of rib_window_attn_bwd_noalloc -------------------------------------------
// Lives in the library image: every device that loads the library holds these bytes until exit.
// In host code the name below is only a handle for cudaGetSymbolAddress, never a device pointer.
static __device__ __align__(256) unsigned char g_noalloc_scratch[RIB_NOALLOC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
std::mutex g_noalloc_mutex;
void* g_noalloc_ptr[kMaxDevices] = {};

// Device address of the built-in scratch on the current device; looked up once per device.
int noalloc_scratch_ptr(void** out)
{
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return RIB_ERR_CUDA;
    std::lock_guard<std::mutex> lock(g_noalloc_mutex);
    if (!g_noalloc_ptr[dev]) {
        void* ptr = nullptr;
        if (cudaGetSymbolAddress(&ptr, g_noalloc_scratch) != cudaSuccess || !ptr) return RIB_ERR_CUDA;
        g_noalloc_ptr[dev] = ptr;
    }
    *out = g_noalloc_ptr[dev];
    return RIB_OK;
}

}  // namespace

namespace rib {

void profile_mark(int kernel_id, int phase, cudaStream_t stream)
{
    if (!g_profile_on.load(std::memory_order_relaxed)) return;
    std::lock_guard<std::mutex> lock(g_profile.mutex);
    if (!g_profile.on) return;
    if (phase == 0) {
        if (g_profile.count >= g_profile.capacity) return;
        g_profile.ids[g_profile.count] = kernel_id;
        cudaEventRecord(g_profile.events[2 * g_profile.count], stream);
        g_profile.pending = true;
    } else if (g_profile.pending) {
        cudaEventRecord(g_profile.events[2 * g_profile.count + 1], stream);
        ++g_profile.count;
        g_profile.pending = false;
    }
}

}  // namespace rib

extern "C" {

int rib_profile_begin(int max_launches)
{
    if (max_launches <= 0 || max_launches > (1 << 20)) return RIB_ERR_SHAPE;
    std::lock_guard<std::mutex> lock(g_profile.mutex);
    if (g_profile.on) return RIB_ERR_UNSUPPORTED;
    g_profile.events.assign(2 * (size_t)max_launches, nullptr);
    g_profile.ids.assign((size_t)max_launches, 0);
    for (auto& e : g_profile.events)
        if (cudaEventCreate(&e) != cudaSuccess) {
            for (auto& d : g_profile.events) if (d) cudaEventDestroy(d);
            g_profile.events.clear();
            return RIB_ERR_CUDA;
        }
    g_profile.capacity = max_launches;
    g_profile.count = 0;
    g_profile.pending = false;
    g_profile.on = true;
    g_profile_on.store(true);
    return RIB_OK;
}

int rib_profile_end(int* kernel_ids, float* ms, int capacity)
{
    std::lock_guard<std::mutex> lock(g_profile.mutex);
    if (!g_profile.on) return RIB_ERR_UNSUPPORTED;
    g_profile_on.store(false);
    g_profile.on = false;
    int written = 0, rc = RIB_OK;
    for (int i = 0; i < g_profile.count; ++i) {
        float t = 0.f;
        if (cudaEventSynchronize(g_profile.events[2 * i + 1]) != cudaSuccess ||
            cudaEventElapsedTime(&t, g_profile.events[2 * i], g_profile.events[2 * i + 1]) != cudaSuccess) { rc = RIB_ERR_CUDA; break; }
        if (kernel_ids && ms && written < capacity) { kernel_ids[written] = g_profile.ids[i]; ms[written] = t; ++written; }
    }
    for (auto& e : g_profile.events) cudaEventDestroy(e);
    g_profile.events.clear();
    g_profile.ids.clear();
    g_profile.capacity = g_profile.count = 0;
    return rc == RIB_OK ? written : rc;
}

int rib_window_attn_fwd(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                        int B, int H, int W, int heads, int d, int r, int window, int shift,
                        void* out, float* lse, void* stream)
{
    return rib_window_attn_fwd_headwise(q, k, v, pq, pk, 0, B, H, W, heads, d, r, window, shift, out, lse, stream);
}

int rib_window_attn_fwd_headwise(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                                 long long pos_head_stride,
                                 int B, int H, int W, int heads, int d, int r, int window, int shift,
                                 void* out, float* lse, void* stream)
{
    if (H > 0 && W > 0 && window > 0 && (H % window || W % window)) return RIB_ERR_SHAPE;
    return rib_window_attn_fwd_padded(q, k, v, pq, pk, pos_head_stride, B, H, W, heads, d, r, window, shift, out, lse, stream);
}

int rib_window_attn_fwd_padded(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                               long long pos_head_stride,
                               int B, int H, int W, int heads, int d, int r, int window, int shift,
                               void* out, float* lse, void* stream)
{
    return fwd_impl(q, k, v, pq, pk, pos_head_stride, nullptr, B, H, W, heads, d, r, window, shift, out, lse, stream);
}

int rib_window_attn_fwd_gated(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                              long long pos_head_stride, const void* gate,
                              int B, int H, int W, int heads, int d, int r, int window, int shift,
                              void* out, float* lse, void* stream)
{
    if (!gate) return RIB_ERR_NULL;
    if (H > 0 && W > 0 && window > 0 && (H % window || W % window)) return RIB_ERR_SHAPE;
    if (!aligned16(gate)) return RIB_ERR_ALIGN;
    return fwd_impl(q, k, v, pq, pk, pos_head_stride, gate, B, H, W, heads, d, r, window, shift, out, lse, stream);
}

int rib_window_cycle_fwd(const void* const* q, const void* const* k, const void* const* v, const void* const* pq, const void* const* pk,
                         const int* windows, const int* shifts, int layers,
                         int B, int H, int W, int heads, int d, int r, void* const* out, float* const* lse, void* stream)
{
    if (!q || !k || !v || !pq || !pk || !windows || !out) return RIB_ERR_NULL;
    if (layers <= 0 || layers > 64) return RIB_ERR_SHAPE;
    // every layer is checked before the first one is launched
    for (int pass = 0; pass < 2; ++pass)
        for (int l = 0; l < layers; ++l) {
            const int rc = fwd_impl(q[l], k[l], v[l], pq[l], pk[l], 0, nullptr, B, H, W, heads, d, r, windows[l], shifts ? shifts[l] : 0,
                                    out[l], lse ? lse[l] : nullptr, stream, pass == 0);
            if (rc != RIB_OK) return rc;
        }
    return RIB_OK;
}

int rib_cla_gate(const void* x, const float* w_dw, const float* b_dw, const float* w_pw, const float* b_pw,
                 int B, int H, int W, int D, void* gate, void* stream)
{
    if (!x || !w_dw || !b_dw || !w_pw || !b_pw || !gate) return RIB_ERR_NULL;
    if (B <= 0 || H <= 0 || W <= 0 || D <= 0) return RIB_ERR_SHAPE;
    // other even channel counts up to 192 (6 heads of 30 or 16 channels) run on zero-padded copies
    const bool native = rib::cla_gate_supported(H, W, D);
    if (!native && !(rib::cla_padded_channels(D) && rib::cla_gate_supported(H, W, rib::cla_padded_channels(D)))) return RIB_ERR_UNSUPPORTED;
    const void* ptrs[] = {x, w_dw, b_dw, w_pw, b_pw, gate};
    for (const void* ptr : ptrs)
        if (!aligned16(ptr)) return RIB_ERR_ALIGN;
    int* status = nullptr;
    if (int rc = device_status_ptr(&status)) return rc;
    int launches = 1;
    const cudaError_t e = native ? rib::cla_gate(static_cast<const __nv_bfloat16*>(x), w_dw, b_dw, w_pw, b_pw, B, H, W, D,
                                                 static_cast<__nv_bfloat16*>(gate), status, static_cast<cudaStream_t>(stream))
                                 : rib::cla_gate_padded(static_cast<const __nv_bfloat16*>(x), w_dw, b_dw, w_pw, b_pw, B, H, W, D,
                                                        static_cast<__nv_bfloat16*>(gate), status, static_cast<cudaStream_t>(stream), &launches);
    if (e != cudaSuccess) return RIB_ERR_CUDA;
    g_kernel_launches += launches;
    return RIB_OK;
}

int rib_cla_product(const void* out, const void* gate, long long count, void* out_gated, void* stream)
{
    if (!out || !gate || !out_gated) return RIB_ERR_NULL;
    if (count < 0 || count % 8) return RIB_ERR_SHAPE;
    if (!aligned16(out) || !aligned16(gate) || !aligned16(out_gated)) return RIB_ERR_ALIGN;
    if (count == 0) return RIB_OK;
    const cudaError_t e = rib::cla_product(static_cast<const __nv_bfloat16*>(out), static_cast<const __nv_bfloat16*>(gate), nullptr,
                                           count, static_cast<__nv_bfloat16*>(out_gated), nullptr, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return RIB_ERR_CUDA;
    g_kernel_launches += 1;
    return RIB_OK;
}

int rib_cla_product_bwd(const void* out, const void* gate, const void* dout_gated, long long count, void* dout, void* dgate,
                        void* stream)
{
    if (!out || !gate || !dout_gated || !dout || !dgate) return RIB_ERR_NULL;
    if (count < 0 || count % 8) return RIB_ERR_SHAPE;
    const void* ptrs[] = {out, gate, dout_gated, dout, dgate};
    for (const void* ptr : ptrs)
        if (!aligned16(ptr)) return RIB_ERR_ALIGN;
    if (count == 0) return RIB_OK;
    const cudaError_t e = rib::cla_product(static_cast<const __nv_bfloat16*>(out), static_cast<const __nv_bfloat16*>(gate),
                                           static_cast<const __nv_bfloat16*>(dout_gated), count, static_cast<__nv_bfloat16*>(dout),
                                           static_cast<__nv_bfloat16*>(dgate), static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return RIB_ERR_CUDA;
    g_kernel_launches += 1;
    return RIB_OK;
}

size_t rib_cla_gate_bwd_workspace(int B, int H, int W, int D)
{
    if (B <= 0 || H <= 0 || W <= 0 || D <= 0) return 0;
    if (!rib::cla_gate_bwd_supported(D) && rib::cla_padded_channels(D)) D = rib::cla_padded_channels(D);     // runs on padded copies
    return rib::cla_gate_bwd_workspace_bytes((long long)B * H * W, D);
}

int rib_cla_gate_bwd(const void* x, const float* w_dw, const float* b_dw, const float* w_pw, const float* b_pw,
                     const void* dgate, int B, int H, int W, int D,
                     void* dx, float* dw_dw, float* db_dw, float* dw_pw, float* db_pw,
                     void* workspace, size_t workspace_bytes, void* stream)
{
    if (!x || !w_dw || !b_dw || !w_pw || !b_pw || !dgate || !dx || !dw_dw || !db_dw || !dw_pw || !db_pw) return RIB_ERR_NULL;
    if (B <= 0 || H <= 0 || W <= 0 || D <= 0) return RIB_ERR_SHAPE;
    const bool native = rib::cla_gate_bwd_supported(D);
    if (!native && !rib::cla_padded_channels(D)) return RIB_ERR_UNSUPPORTED;
    const void* ptrs[] = {x, w_dw, b_dw, w_pw, b_pw, dgate, dx, dw_dw, db_dw, dw_pw, db_pw, workspace};
    for (const void* ptr : ptrs)
        if (!aligned16(ptr)) return RIB_ERR_ALIGN;
    if (!workspace || workspace_bytes < rib_cla_gate_bwd_workspace(B, H, W, D)) return RIB_ERR_WORKSPACE;
    int* status = nullptr;
    if (int rc = device_status_ptr(&status)) return rc;
    const bool fast = g_forced_path.load() != RIB_PATH_GENERIC;
    int launches = fast ? 3 : 4;           // zeroing of the weight gradients, (transpose,) point-wise part, depth-wise part
    const cudaError_t e =
        native ? rib::cla_gate_bwd(static_cast<const __nv_bfloat16*>(x), w_dw, b_dw, w_pw, b_pw, static_cast<const __nv_bfloat16*>(dgate), B, H,
                                   W, D, static_cast<__nv_bfloat16*>(dx), dw_dw, db_dw, dw_pw, db_pw, workspace, fast, status,
                                   static_cast<cudaStream_t>(stream))
               : rib::cla_gate_bwd_padded(static_cast<const __nv_bfloat16*>(x), w_dw, b_dw, w_pw, b_pw, static_cast<const __nv_bfloat16*>(dgate),
                                          B, H, W, D, static_cast<__nv_bfloat16*>(dx), dw_dw, db_dw, dw_pw, db_pw, workspace, fast, status,
                                          static_cast<cudaStream_t>(stream), &launches);
    if (e != cudaSuccess) return RIB_ERR_CUDA;
    t_last_path = fast ? RIB_PATH_SM100 : RIB_PATH_GENERIC;
    g_kernel_launches += launches;
    return RIB_OK;
}

}  // extern "C"

namespace {

int fwd_impl(const void* q, const void* k, const void* v, const void* pq, const void* pk, long long pos_head_stride, const void* gate,
             int B, int H, int W, int heads, int d, int r, int window, int shift, void* out, float* lse, void* stream, bool validate_only,
             bool masked, const BiasArgs* bias)
{
    if (!q || !k || !v || !out || (r > 0 && (!pq || !pk))) return RIB_ERR_NULL;
    if (int rc = check_shape(B, H, W, heads, d, r, window, shift, true)) return rc;
    if (int rc = check_pos_stride(pos_head_stride, window, r)) return rc;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(pq) ||
        !aligned16(pk) || !aligned16(lse))
        return RIB_ERR_ALIGN;
    if (validate_only) return RIB_OK;
    rib::Problem p{};
    fill_shape(p, B, H, W, heads, d, r, window, shift);
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k = static_cast<const __nv_bfloat16*>(k);
    p.v = static_cast<const __nv_bfloat16*>(v);
    p.pq = static_cast<const __nv_bfloat16*>(pq);
    p.pk = static_cast<const __nv_bfloat16*>(pk);
    p.out_w = static_cast<__nv_bfloat16*>(out);
    p.lse_w = lse;
    p.pos_head_stride = pos_head_stride;
    p.gate = static_cast<const __nv_bfloat16*>(gate);
    p.masked = masked;
    if (bias) fill_bias(p, *bias);
    if (int rc = device_status_ptr(&p.status)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int forced = g_forced_path.load();
    const bool frame = !bias && rib::sm100_frame_supported(p);
    bool fast = forced != RIB_PATH_GENERIC && (bias ? rib::sm100_bias_fwd_supported(p) : frame || rib::sm100_fwd_supported(p));
    p.exact_softmax = forced == RIB_PATH_SM100_EXACT;
    int launches = 1;
    cudaError_t e;
    if (fast) {
        e = bias ? rib::sm100_bias_fwd(p, st) : frame ? rib::sm100_fwd_frame(p, st) : rib::sm100_fwd(p, st);
    } else if (forced != RIB_PATH_GENERIC && !bias && rib::sm100_repack_fwd_supported(p)) {
        // rows TMA cannot address (d = 30, r = 18, ...): the tensor-core kernels on zero-padded copies
        e = rib::sm100_fwd_repacked(p, st, &launches);
        fast = e == cudaSuccess;
        if (e == cudaErrorMemoryAllocation) {       // no scratch to be had: the any-shape kernel needs none
            (void)cudaGetLastError();
            launches = 1;
            e = rib::generic_fwd(p, st);
        }
    } else if (forced != RIB_PATH_GENERIC && rib::bias_small_supported(p)) {
        e = rib::bias_small_fwd(p, st);
    } else {
        e = rib::generic_fwd(p, st);
    }
    if (e != cudaSuccess) return RIB_ERR_CUDA;
    t_last_path = fast ? RIB_PATH_SM100 : RIB_PATH_GENERIC;
    g_kernel_launches += launches;
    return RIB_OK;
}

}  // namespace

extern "C" {

size_t rib_window_attn_bwd_workspace(int B, int H, int W, int heads, int d, int r, int window)
{
    return rib_window_attn_bwd_headwise_workspace(0, B, H, W, heads, d, r, window);
}

size_t rib_window_attn_bwd_headwise_workspace(long long pos_head_stride, int B, int H, int W, int heads, int d, int r,
                                              int window)
{
    if (check_shape(B, H, W, heads, d, r, window, 0) != RIB_OK) return 0;
    if (check_pos_stride(pos_head_stride, window, r) != RIB_OK) return 0;
    size_t need = rowdot_bytes(B, H, W, heads);
    rib::Problem p{};
    fill_shape(p, B, H, W, heads, d, r, window, 0);
    if (rib::sm100_bwd_supported(p) || rib::sm100_repack_bwd_supported(p)) {   // whatever the shift: one size per shape
        const size_t fast = rib::sm100_bwd_workspace_bytes(p.pairs, p.n, pos_head_stride ? heads : 1, rib::repacked_width(r));
        if (fast > need) need = fast;
    }
    return need;
}

int rib_window_attn_bwd(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                        const void* out, const float* lse, const void* dout,
                        int B, int H, int W, int heads, int d, int r, int window, int shift,
                        void* dq, void* dk, void* dv, float* dpq, float* dpk,
                        void* workspace, size_t workspace_bytes, void* stream)
{
    return rib_window_attn_bwd_headwise(q, k, v, pq, pk, 0, out, lse, dout, B, H, W, heads, d, r, window, shift, dq, dk, dv,
                                        dpq, dpk, workspace, workspace_bytes, stream);
}

int rib_window_attn_bwd_headwise(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                                 long long pos_head_stride,
                                 const void* out, const float* lse, const void* dout,
                                 int B, int H, int W, int heads, int d, int r, int window, int shift,
                                 void* dq, void* dk, void* dv, float* dpq, float* dpk,
                                 void* workspace, size_t workspace_bytes, void* stream)
{
    if (H > 0 && W > 0 && window > 0 && (H % window || W % window)) return RIB_ERR_SHAPE;
    return rib_window_attn_bwd_padded(q, k, v, pq, pk, pos_head_stride, out, lse, dout, B, H, W, heads, d, r, window, shift, dq, dk,
                                      dv, dpq, dpk, workspace, workspace_bytes, stream);
}

size_t rib_window_attn_bwd_padded_workspace(long long pos_head_stride, int B, int H, int W, int heads, int d, int r, int window)
{
    if (H > 0 && W > 0 && window > 0 && H % window == 0 && W % window == 0)
        return rib_window_attn_bwd_headwise_workspace(pos_head_stride, B, H, W, heads, d, r, window);
    if (check_shape(B, H, W, heads, d, r, window, 0, true) != RIB_OK) return 0;
    if (check_pos_stride(pos_head_stride, window, r) != RIB_OK) return 0;
    size_t need = rowdot_bytes(B, H, W, heads);
    rib::Problem p{};
    fill_shape(p, B, H, W, heads, d, r, window, 0);
    if (rib::sm100_bwd_supported(p) || rib::sm100_repack_bwd_supported(p)) {        // sized by the windows of the extended map
        const size_t fast = rib::sm100_bwd_workspace_bytes(p.pairs, p.n, pos_head_stride ? heads : 1, rib::repacked_width(r));
        if (fast > need) need = fast;
    }
    return need;
}

}  // extern "C"

namespace {

struct BwdBias : BiasArgs { void* gradient; };

// A backward call from checkpoints: the four tensors come back as bf16 at the start of the workspace, what is behind them is the backward
// pass's own.
struct Restored {
    rib::CheckpointRows t[4];
    long long rows;
    int d;
    void* rest;
    size_t rest_bytes;
};

int restore(const Restored& r, void* stream, bool wide = false)
{
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if ((wide ? rib::checkpoint_restore_wide(r.t, r.rows, r.d, st) : rib::checkpoint_restore(r.t, 4, r.rows, r.d, st)) != cudaSuccess) return RIB_ERR_CUDA;
    g_kernel_launches += 1;
    return RIB_OK;
}

// Scratch of a backward pass with a bias: what the attention kernels need, then the sums of the table's gradient.
size_t bucketed_attention_bytes(int B, int H, int W, int heads, int window)
{
    rib::Problem p{};
    fill_shape(p, B, H, W, heads, 8, 0, window, 0);
    const size_t any = rowdot_bytes(B, H, W, heads), fast = window % 8 == 0 ? rib::sm100_bias_bwd_workspace_bytes(p.pairs, p.n) : 0;
    return any > fast ? any : fast;
}

size_t bucketed_workspace(long long bias_head_stride, int num_buckets, int B, int H, int W, int heads, int d, int window)
{
    if (check_shape(B, H, W, heads, d, 0, window, 0, true) != RIB_OK) return 0;
    if (num_buckets <= 0 || bias_head_stride < 0 || (bias_head_stride && bias_head_stride < num_buckets)) return 0;
    return bucketed_attention_bytes(B, H, W, heads, window) + rib::bias_grad_layout(heads, bias_head_stride ? heads : 1, window, num_buckets, nullptr).bytes;
}

}  // namespace

extern "C" {

static int bwd_impl(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                    long long pos_head_stride,
                    const void* out, const float* lse, const void* dout,
                    int B, int H, int W, int heads, int d, int r, int window, int shift,
                    void* dq, void* dk, void* dv, float* dpq, float* dpk,
                    void* workspace, size_t workspace_bytes, void* stream, bool masked, bool validate_only = false,
                    const BwdBias* bias = nullptr, const Restored* saved = nullptr)
{
    if (!q || !k || !v || !out || !lse || !dout || !dq || !dk || !dv) return RIB_ERR_NULL;
    if (r > 0 && (!pq || !pk || !dpq || !dpk)) return RIB_ERR_NULL;
    if (int rc = check_shape(B, H, W, heads, d, r, window, shift, true)) return rc;
    if (int rc = check_pos_stride(pos_head_stride, window, r)) return rc;
    const void* ptrs[] = {q, k, v, pq, pk, out, lse, dout, dq, dk, dv, dpq, dpk};
    for (const void* ptr : ptrs)
        if (!aligned16(ptr)) return RIB_ERR_ALIGN;
    const size_t need = bias ? bucketed_workspace(bias->head_stride, bias->num_buckets, B, H, W, heads, d, window)
                             : rib_window_attn_bwd_padded_workspace(pos_head_stride, B, H, W, heads, d, r, window);
    if (!workspace || workspace_bytes < need) return RIB_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return RIB_ERR_ALIGN;
    if (validate_only) return RIB_OK;
    rib::Problem p{};
    fill_shape(p, B, H, W, heads, d, r, window, shift);
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k = static_cast<const __nv_bfloat16*>(k);
    p.v = static_cast<const __nv_bfloat16*>(v);
    p.pq = static_cast<const __nv_bfloat16*>(pq);
    p.pk = static_cast<const __nv_bfloat16*>(pk);
    p.out = static_cast<const __nv_bfloat16*>(out);
    p.dout = static_cast<const __nv_bfloat16*>(dout);
    p.lse_in = lse;
    p.dq = static_cast<__nv_bfloat16*>(dq);
    p.dk = static_cast<__nv_bfloat16*>(dk);
    p.dv = static_cast<__nv_bfloat16*>(dv);
    p.dpq = dpq;
    p.dpk = dpk;
    p.rowdot = static_cast<float*>(workspace);
    p.workspace = workspace;
    p.workspace_bytes = workspace_bytes;
    p.pos_head_stride = pos_head_stride;
    p.masked = masked;
    if (int rc = device_status_ptr(&p.status)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (bias) {
        fill_bias(p, *bias);
        p.dbias = bias->gradient;
        const rib::BiasGrad g = rib::bias_grad_layout(heads, rib::bias_tables(p), window, bias->num_buckets,
                                                      static_cast<unsigned char*>(workspace) + bucketed_attention_bytes(B, H, W, heads, window));
        const bool fast = g_forced_path.load() != RIB_PATH_GENERIC && rib::sm100_bias_bwd_supported(p);
        if (saved && fast && rib::restored_width(d) != d) p.qk_width = rib::restored_width(d);
        if (saved && fast) p.saved = saved->t;
        else if (saved)
            if (int rc = restore(*saved, stream)) return rc;
        cudaError_t e;
        int launches = fast ? 4 : 5;
        if (fast) {
            e = rib::sm100_bias_bwd(p, g, st);
        } else {
            e = rib::bias_grad_clear(g, st);
            const bool small = g_forced_path.load() != RIB_PATH_GENERIC && rib::bias_small_supported(p);
            if (small) launches = 3;
            if (e == cudaSuccess) e = small ? rib::bias_small_bwd(p, g.offsets, st) : rib::generic_bwd(p, st, g.offsets);
            if (e == cudaSuccess) e = rib::bias_grad_scatter(p, g, st);
            if (e == cudaSuccess) e = rib::bias_grad_convert(p, g, st);
        }
        if (e != cudaSuccess) return RIB_ERR_CUDA;
        t_last_path = fast ? RIB_PATH_SM100 : RIB_PATH_GENERIC;
        g_kernel_launches += launches;
        return RIB_OK;
    }
    const bool allowed = g_forced_path.load() != RIB_PATH_GENERIC;
    bool fast = allowed && rib::sm100_bwd_supported(p);
    if (saved && fast && rib::restored_width(d) != d) p.qk_width = rib::restored_width(d);
    if (saved && fast && rib::sm100_bwd_takes_saved(p)) p.saved = saved->t;
    else if (saved)
        if (int rc = restore(*saved, stream, p.qk_width != 0)) return rc;
    int launches = fast ? rib::sm100_bwd_launches(p) : 3;          // any-shape kernels: rowdot, dq, dk/dv
    cudaError_t e;
    if (fast) {
        e = rib::sm100_bwd(p, st);
    } else if (allowed && rib::sm100_repack_bwd_supported(p)) {
        e = rib::sm100_bwd_repacked(p, st, &launches);
        fast = e == cudaSuccess;
        if (e == cudaErrorMemoryAllocation) {
            (void)cudaGetLastError();
            launches = 3;
            e = rib::generic_bwd(p, st);
        }
    } else {
        e = rib::generic_bwd(p, st);
    }
    if (e != cudaSuccess) return RIB_ERR_CUDA;
    t_last_path = fast ? RIB_PATH_SM100 : RIB_PATH_GENERIC;
    g_kernel_launches += launches;
    return RIB_OK;
}

int rib_window_attn_bwd_padded(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                               long long pos_head_stride,
                               const void* out, const float* lse, const void* dout,
                               int B, int H, int W, int heads, int d, int r, int window, int shift,
                               void* dq, void* dk, void* dv, float* dpq, float* dpk,
                               void* workspace, size_t workspace_bytes, void* stream)
{
    return bwd_impl(q, k, v, pq, pk, pos_head_stride, out, lse, dout, B, H, W, heads, d, r, window, shift, dq, dk, dv, dpq, dpk,
                    workspace, workspace_bytes, stream, false);
}

size_t rib_window_cycle_bwd_workspace(const int* windows, int layers, int B, int H, int W, int heads, int d, int r)
{
    if (!windows || layers <= 0 || layers > 64) return 0;
    size_t need = 0;
    for (int l = 0; l < layers; ++l) {
        const size_t one = rib_window_attn_bwd_padded_workspace(0, B, H, W, heads, d, r, windows[l]);
        if (one == 0) return 0;
        if (one > need) need = one;
    }
    return need;
}

int rib_window_cycle_bwd(const void* const* q, const void* const* k, const void* const* v, const void* const* pq, const void* const* pk,
                         const void* const* out, const float* const* lse, const void* const* dout,
                         const int* windows, const int* shifts, int layers,
                         int B, int H, int W, int heads, int d, int r,
                         void* const* dq, void* const* dk, void* const* dv, float* const* dpq, float* const* dpk,
                         void* workspace, size_t workspace_bytes, void* stream)
{
    if (!q || !k || !v || !pq || !pk || !out || !lse || !dout || !windows || !dq || !dk || !dv || !dpq || !dpk) return RIB_ERR_NULL;
    if (layers <= 0 || layers > 64) return RIB_ERR_SHAPE;
    // every layer is checked before the first one is launched; the layers run one after the other on the stream and share the workspace
    for (int pass = 0; pass < 2; ++pass)
        for (int l = 0; l < layers; ++l) {
            const int rc = bwd_impl(q[l], k[l], v[l], pq[l], pk[l], 0, out[l], lse[l], dout[l], B, H, W, heads, d, r, windows[l],
                                    shifts ? shifts[l] : 0, dq[l], dk[l], dv[l], dpq[l], dpk[l], workspace, workspace_bytes, stream, false,
                                    pass == 0);
            if (rc != RIB_OK) return rc;
        }
    return RIB_OK;
}

int rib_window_attn_fwd_masked(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                               long long pos_head_stride,
                               int B, int H, int W, int heads, int d, int r, int window, int shift,
                               void* out, float* lse, void* stream)
{
    if (H > 0 && W > 0 && window > 0 && (H % window || W % window)) return RIB_ERR_SHAPE;
    return fwd_impl(q, k, v, pq, pk, pos_head_stride, nullptr, B, H, W, heads, d, r, window, shift, out, lse, stream, false, true);
}

int rib_window_attn_bwd_masked(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                               long long pos_head_stride,
                               const void* out, const float* lse, const void* dout,
                               int B, int H, int W, int heads, int d, int r, int window, int shift,
                               void* dq, void* dk, void* dv, float* dpq, float* dpk,
                               void* workspace, size_t workspace_bytes, void* stream)
{
    if (H > 0 && W > 0 && window > 0 && (H % window || W % window)) return RIB_ERR_SHAPE;
    return bwd_impl(q, k, v, pq, pk, pos_head_stride, out, lse, dout, B, H, W, heads, d, r, window, shift, dq, dk, dv, dpq, dpk,
                    workspace, workspace_bytes, stream, true);
}

int rib_window_attn_fwd_bucketed(const void* q, const void* k, const void* v, const void* bias, int bias_dtype, long long bias_head_stride,
                                 const int* buckets, int num_buckets,
                                 int B, int H, int W, int heads, int d, int window, int shift, int masked,
                                 void* out, float* lse, void* stream)
{
    if (masked && H > 0 && W > 0 && window > 0 && (H % window || W % window)) return RIB_ERR_SHAPE;
    const BiasArgs b{bias, bias_dtype, bias_head_stride, buckets, num_buckets};
    if (int rc = check_bias(b)) return rc;
    return fwd_impl(q, k, v, nullptr, nullptr, 0, nullptr, B, H, W, heads, d, 0, window, shift, out, lse, stream, false, masked != 0, &b);
}

size_t rib_window_attn_bwd_bucketed_workspace(long long bias_head_stride, int num_buckets, int B, int H, int W, int heads, int d, int window)
{
    return bucketed_workspace(bias_head_stride, num_buckets, B, H, W, heads, d, window);
}

}  // extern "C"

namespace {

// The bias of a backward call, checked.
int bwd_bias(const void* bias, int dtype, long long head_stride, const int* buckets, int num_buckets, void* dbias, BwdBias* b)
{
    *b = BwdBias{{bias, dtype, head_stride, buckets, num_buckets}, dbias};
    if (!dbias) return RIB_ERR_NULL;
    if (int rc = check_bias(*b)) return rc;
    return reinterpret_cast<uintptr_t>(dbias) & (dtype == RIB_DTYPE_F32 ? 3u : 1u) ? RIB_ERR_ALIGN : RIB_OK;
}

int check_checkpoint(const void* codes, const float* scales, long long rows, int d)
{
    if (!codes || !scales) return RIB_ERR_NULL;
    if (rows < 0 || d <= 0) return RIB_ERR_SHAPE;
    if (d > 64 || rows > (1ll << 31)) return RIB_ERR_UNSUPPORTED;
    if (!aligned16(codes) || !aligned16(scales)) return RIB_ERR_ALIGN;
    return RIB_OK;
}

size_t image_bytes(int B, int H, int W, int heads, int d) { return (2 * (size_t)B * H * W * heads * d + 255) & ~(size_t)255; }
// q and k (which may be restored to wider rows), v and out
size_t restored_bytes(int B, int H, int W, int heads, int d)
{
    return 2 * (image_bytes(B, H, W, heads, rib::restored_width(d)) + image_bytes(B, H, W, heads, d));
}

int plan_restore(const rib_checkpoint* saved, int B, int H, int W, int heads, int d, void* workspace, size_t workspace_bytes, Restored* r)
{
    if (!saved) return RIB_ERR_NULL;
    if (B <= 0 || H <= 0 || W <= 0 || heads <= 0) return RIB_ERR_SHAPE;
    const __int128 rows = (__int128)B * H * W * heads;
    if (rows > (1ll << 31)) return RIB_ERR_UNSUPPORTED;
    r->rows = (long long)rows;
    r->d = d;
    for (int i = 0; i < 4; ++i)
        if (int rc = check_checkpoint(saved[i].codes, saved[i].scales, r->rows, d)) return rc;
    const size_t all = restored_bytes(B, H, W, heads, d);
    if (!workspace || workspace_bytes < all) return RIB_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return RIB_ERR_ALIGN;
    unsigned char* at = static_cast<unsigned char*>(workspace);
    for (int i = 0; i < 4; at += image_bytes(B, H, W, heads, i < 2 ? rib::restored_width(d) : d), ++i)
        r->t[i] = {static_cast<const int8_t*>(saved[i].codes), saved[i].scales, reinterpret_cast<__nv_bfloat16*>(at)};
    r->rest = at;
    r->rest_bytes = workspace_bytes - all;
    return RIB_OK;
}

}  // namespace

extern "C" {

int rib_window_attn_bwd_bucketed(const void* q, const void* k, const void* v, const void* bias, int bias_dtype, long long bias_head_stride,
                                 const int* buckets, int num_buckets, const void* out, const float* lse, const void* dout,
                                 int B, int H, int W, int heads, int d, int window, int shift, int masked,
                                 void* dq, void* dk, void* dv, void* dbias, void* workspace, size_t workspace_bytes, void* stream)
{
    if (masked && H > 0 && W > 0 && window > 0 && (H % window || W % window)) return RIB_ERR_SHAPE;
    BwdBias b;
    if (int rc = bwd_bias(bias, bias_dtype, bias_head_stride, buckets, num_buckets, dbias, &b)) return rc;
    return bwd_impl(q, k, v, nullptr, nullptr, 0, out, lse, dout, B, H, W, heads, d, 0, window, shift, dq, dk, dv, nullptr, nullptr,
                    workspace, workspace_bytes, stream, masked != 0, false, &b);
}

int rib_checkpoint_store(const void* x, long long rows, int d, void* codes, float* scales, void* stream)
{
    if (!x) return RIB_ERR_NULL;
    if (int rc = check_checkpoint(codes, scales, rows, d)) return rc;
    if (!aligned16(x)) return RIB_ERR_ALIGN;
    if (rows == 0) return RIB_OK;
    if (rib::checkpoint_store(static_cast<const __nv_bfloat16*>(x), rows, d, static_cast<int8_t*>(codes), scales, static_cast<cudaStream_t>(stream)) != cudaSuccess)
        return RIB_ERR_CUDA;
    g_kernel_launches += 1;
    return RIB_OK;
}

int rib_checkpoint_restore(const void* codes, const float* scales, long long rows, int d, void* x, void* stream)
{
    if (!x) return RIB_ERR_NULL;
    if (int rc = check_checkpoint(codes, scales, rows, d)) return rc;
    if (!aligned16(x)) return RIB_ERR_ALIGN;
    if (rows == 0) return RIB_OK;
    const rib::CheckpointRows t{static_cast<const int8_t*>(codes), scales, static_cast<__nv_bfloat16*>(x)};
    if (rib::checkpoint_restore(&t, 1, rows, d, static_cast<cudaStream_t>(stream)) != cudaSuccess) return RIB_ERR_CUDA;
    g_kernel_launches += 1;
    return RIB_OK;
}

size_t rib_window_attn_bwd_checkpointed_workspace(long long pos_head_stride, int B, int H, int W, int heads, int d, int r, int window)
{
    const size_t need = rib_window_attn_bwd_padded_workspace(pos_head_stride, B, H, W, heads, d, r, window);
    return need ? need + restored_bytes(B, H, W, heads, d) : 0;
}

int rib_window_attn_bwd_checkpointed(const rib_checkpoint* saved, const void* pq, const void* pk, long long pos_head_stride, const float* lse,
                                     const void* dout, int B, int H, int W, int heads, int d, int r, int window, int shift, int masked,
                                     void* dq, void* dk, void* dv, float* dpq, float* dpk, void* workspace, size_t workspace_bytes, void* stream)
{
    if (masked && H > 0 && W > 0 && window > 0 && (H % window || W % window)) return RIB_ERR_SHAPE;
    Restored s;
    if (int rc = plan_restore(saved, B, H, W, heads, d, workspace, workspace_bytes, &s)) return rc;
    return bwd_impl(s.t[0].x, s.t[1].x, s.t[2].x, pq, pk, pos_head_stride, s.t[3].x, lse, dout, B, H, W, heads, d, r, window, shift, dq, dk, dv,
                    dpq, dpk, s.rest, s.rest_bytes, stream, masked != 0, false, nullptr, &s);
}

size_t rib_window_attn_bwd_bucketed_checkpointed_workspace(long long bias_head_stride, int num_buckets, int B, int H, int W, int heads, int d, int window)
{
    const size_t need = bucketed_workspace(bias_head_stride, num_buckets, B, H, W, heads, d, window);
    return need ? need + restored_bytes(B, H, W, heads, d) : 0;
}

int rib_window_attn_bwd_bucketed_checkpointed(const rib_checkpoint* saved, const void* bias, int bias_dtype, long long bias_head_stride,
                                              const int* buckets, int num_buckets, const float* lse, const void* dout,
                                              int B, int H, int W, int heads, int d, int window, int shift, int masked,
                                              void* dq, void* dk, void* dv, void* dbias, void* workspace, size_t workspace_bytes, void* stream)
{
    if (masked && H > 0 && W > 0 && window > 0 && (H % window || W % window)) return RIB_ERR_SHAPE;
    BwdBias b;
    if (int rc = bwd_bias(bias, bias_dtype, bias_head_stride, buckets, num_buckets, dbias, &b)) return rc;
    Restored s;
    if (int rc = plan_restore(saved, B, H, W, heads, d, workspace, workspace_bytes, &s)) return rc;
    return bwd_impl(s.t[0].x, s.t[1].x, s.t[2].x, nullptr, nullptr, 0, s.t[3].x, lse, dout, B, H, W, heads, d, 0, window, shift, dq, dk, dv,
                    nullptr, nullptr, s.rest, s.rest_bytes, stream, masked != 0, false, &b, &s);
}

int rib_window_attn_bwd_noalloc(const void* q, const void* k, const void* v, const void* pq, const void* pk,
                                const void* out, const float* lse, const void* dout,
                                int B, int H, int W, int heads, int d, int r, int window, int shift,
                                void* dq, void* dk, void* dv, float* dpq, float* dpk, void* stream)
{
    if (int rc = check_shape(B, H, W, heads, d, r, window, shift)) return rc;
    if (rib_window_attn_bwd_workspace(B, H, W, heads, d, r, window) > (size_t)RIB_NOALLOC_SCRATCH_BYTES)
        return RIB_ERR_TOO_LARGE;
    void* scratch = nullptr;
    if (int rc = noalloc_scratch_ptr(&scratch)) return rc;
    return rib_window_attn_bwd(q, k, v, pq, pk, out, lse, dout, B, H, W, heads, d, r, window, shift, dq, dk, dv,
                               dpq, dpk, scratch, (size_t)RIB_NOALLOC_SCRATCH_BYTES, stream);
}

int rib_generate_features(const float* w_h, const float* b_h, const float* w_pq, const float* w_pk,
                          int window, int L, int dh, int r, void* pq, void* pk, void* stream)
{
    if (!w_h || !b_h || !w_pq || !w_pk || !pq || !pk) return RIB_ERR_NULL;
    if (window <= 0 || L < 0 || dh <= 0 || r <= 0) return RIB_ERR_SHAPE;
    if (!rib::generator_supported(window, L, dh, r)) return RIB_ERR_UNSUPPORTED;
    const void* ptrs[] = {w_h, b_h, w_pq, w_pk, pq, pk};
    for (const void* ptr : ptrs)
        if (!aligned16(ptr)) return RIB_ERR_ALIGN;
    const cudaError_t e = rib::generator_fwd(w_h, b_h, w_pq, w_pk, window, L, dh, r, static_cast<__nv_bfloat16*>(pq),
                                             static_cast<__nv_bfloat16*>(pk), static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return RIB_ERR_CUDA;
    g_kernel_launches += 1;
    return RIB_OK;
}

int rib_generate_features_bwd(const float* w_h, const float* b_h, const float* w_pq, const float* w_pk,
                              const float* dpq, const float* dpk, int window, int L, int dh, int r,
                              float* dw_h, float* db_h, float* dw_pq, float* dw_pk, void* stream)
{
    if (!w_h || !b_h || !w_pq || !w_pk || !dpq || !dpk || !dw_h || !db_h || !dw_pq || !dw_pk) return RIB_ERR_NULL;
    if (window <= 0 || L < 0 || dh <= 0 || r <= 0) return RIB_ERR_SHAPE;
    if (!rib::generator_supported(window, L, dh, r)) return RIB_ERR_UNSUPPORTED;
    const void* ptrs[] = {w_h, b_h, w_pq, w_pk, dpq, dpk, dw_h, db_h, dw_pq, dw_pk};
    for (const void* ptr : ptrs)
        if (!aligned16(ptr)) return RIB_ERR_ALIGN;
    const cudaError_t e = rib::generator_bwd(w_h, b_h, w_pq, w_pk, dpq, dpk, window, L, dh, r, dw_h, db_h, dw_pq, dw_pk,
                                             static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return RIB_ERR_CUDA;
    g_kernel_launches += 2;          // clearing of the gradients, main kernel
    return RIB_OK;
}

long long rib_exp_probe(float* sink, int blocks, int iters, void* stream)
{
    if (!sink) return RIB_ERR_NULL;
    if (blocks <= 0 || iters <= 0 || blocks > (1 << 20) || iters > (1 << 24)) return RIB_ERR_SHAPE;
    if (rib::exp_probe(sink, blocks, iters, static_cast<cudaStream_t>(stream)) != cudaSuccess) return RIB_ERR_CUDA;
    g_kernel_launches += 1;
    return rib::exp_probe_count(blocks, iters);
}

int rib_wait_probe(unsigned long long limit_ns, void* stream)
{
    if (limit_ns == 0 || limit_ns > 100000000ull) return RIB_ERR_SHAPE;      // at most 0.1 s
    int* status = nullptr;
    if (int rc = device_status_ptr(&status)) return rc;
    if (rib::wait_probe(status, limit_ns, static_cast<cudaStream_t>(stream)) != cudaSuccess) return RIB_ERR_CUDA;
    g_kernel_launches += 1;
    return RIB_OK;
}

int rib_query_status(void* stream)
{
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int word = 0;
    if (cudaMemcpyFromSymbolAsync(&word, g_status_word, sizeof(int), 0, cudaMemcpyDeviceToHost, st) != cudaSuccess)
        return RIB_ERR_CUDA;
    if (cudaStreamSynchronize(st) != cudaSuccess) return RIB_ERR_CUDA;
    if (word != 0) {
        const int zero = 0;
        if (cudaMemcpyToSymbolAsync(g_status_word, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, st) != cudaSuccess ||
            cudaStreamSynchronize(st) != cudaSuccess)
            return RIB_ERR_CUDA;
        return RIB_ERR_DEVICE_WAIT;
    }
    return RIB_OK;
}

const char* rib_status_string(int status)
{
    switch (status) {
        case RIB_OK: return "RIB_OK";
        case RIB_ERR_NULL: return "RIB_ERR_NULL: a required pointer is NULL";
        case RIB_ERR_SHAPE: return "RIB_ERR_SHAPE: bad sizes, H/W not a multiple of window, or shift out of range";
        case RIB_ERR_UNSUPPORTED: return "RIB_ERR_UNSUPPORTED: d or r outside the supported range";
        case RIB_ERR_ALIGN: return "RIB_ERR_ALIGN: a pointer is not sufficiently aligned";
        case RIB_ERR_WORKSPACE: return "RIB_ERR_WORKSPACE: workspace missing or too small";
        case RIB_ERR_CUDA: return "RIB_ERR_CUDA: a CUDA call failed";
        case RIB_ERR_DEVICE_WAIT: return "RIB_ERR_DEVICE_WAIT: a bounded device-side wait ran out";
        case RIB_ERR_TOO_LARGE: return "RIB_ERR_TOO_LARGE: the shape needs more scratch than the built-in array holds";
        default: return "unknown RIB status";
    }
}

int rib_set_path(int path)
{
    if (path != RIB_PATH_NONE && path != RIB_PATH_GENERIC && path != RIB_PATH_SM100_EXACT) return g_forced_path.load();
    return g_forced_path.exchange(path);
}

int rib_last_path(void) { return t_last_path; }

long long rib_kernel_launches(void) { return g_kernel_launches.load(); }

void rib_tensor_map_cache_counts(long long* hits, long long* misses)
{
    long long h = 0, m = 0;
    rib::tensor_map_cache_counts(&h, &m);
    if (hits) *hits = h;
    if (misses) *misses = m;
}

}  // extern "C"
