// Public C ABI of libvitcop: argument validation, workspace carving and dispatch to the launchers.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <mutex>
#include <vector>

#include "attention.cuh"
#include "gram.cuh"
#include "internal.cuh"
#include "kv_cache.cuh"
#include "rotary.cuh"

namespace vitcop {

static thread_local int g_last_cuda_error = 0;

int record_cuda(cudaError_t e) {
    if (e == cudaSuccess) return VITCOP_OK;
    g_last_cuda_error = static_cast<int>(e);
    return VITCOP_ERR_CUDA;
}

// ---- diagnostic kernel timing ------------------------------------------------------------------------
namespace {
struct TimedLaunch {
    const char* name;
    cudaEvent_t start, stop;
    bool complete;
};
std::atomic<bool> g_timing_on{false};
std::mutex g_timing_mutex;
std::vector<TimedLaunch> g_timed;
}  // namespace

bool kernel_timing_on() { return g_timing_on.load(std::memory_order_relaxed); }

KernelTimeScope::KernelTimeScope(const char* name, cudaStream_t stream) : slot_(-1), stream_(stream) {
    if (!kernel_timing_on()) return;
    TimedLaunch t{name, nullptr, nullptr, false};
    if (cudaEventCreate(&t.start) != cudaSuccess) return;
    if (cudaEventCreate(&t.stop) != cudaSuccess) { cudaEventDestroy(t.start); return; }
    cudaEventRecord(t.start, stream);
    std::lock_guard<std::mutex> lock(g_timing_mutex);
    slot_ = (int)g_timed.size();
    g_timed.push_back(t);
}

KernelTimeScope::~KernelTimeScope() {
    if (slot_ < 0) return;
    std::lock_guard<std::mutex> lock(g_timing_mutex);
    if (slot_ < (int)g_timed.size()) {
        cudaEventRecord(g_timed[slot_].stop, stream_);
        g_timed[slot_].complete = true;
    }
}

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
inline bool aligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }

inline bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
    if (!a || !b || na == 0 || nb == 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

// Workspace of the fused step: status | score [B,Nv] | keep_idx [B,Nv] | n_keep [B]
struct StepWs {
    size_t off_score, off_keep, off_nkeep, total;
    StepWs(int B, int Nv) {
        size_t o = kStatusBytes;
        off_score = o; o += align_up((size_t)B * Nv * sizeof(float), 256);
        off_keep = o;  o += align_up((size_t)B * Nv * sizeof(int32_t), 256);
        off_nkeep = o; o += align_up((size_t)B * sizeof(int32_t), 256);
        total = o;
    }
};

// (Calls whose first kernel can do it clear the word there: a memset in front of a small kernel costs more than a microsecond.)
int reset_status(void* ws, cudaStream_t s) { return record_cuda(cudaMemsetAsync(ws, 0, kStatusBytes, s)); }

int check_span(int N, int vis_start, const int32_t* vis_len, int vis_len_uniform, int Nv_cap) {
    if (vis_start < 0 || vis_start > N) return VITCOP_ERR_INVALID_ARG;
    if (!vis_len) {
        if (vis_len_uniform < 0 || vis_start + (int64_t)vis_len_uniform > N) return VITCOP_ERR_INVALID_ARG;
        if (Nv_cap >= 0 && vis_len_uniform > Nv_cap) return VITCOP_ERR_INVALID_ARG;
    } else if (Nv_cap >= 0 && vis_start + (int64_t)Nv_cap > N) {
        // device-side lengths are clamped to the capacity, which itself must fit the sequence
        return VITCOP_ERR_INVALID_ARG;
    }
    return VITCOP_OK;
}

}  // namespace
}  // namespace vitcop

using namespace vitcop;

// ---- built-in scratch of vitcop_prune_step_static ------------------------------------------------------
// Lives in every GPU that loads the library, from load to exit.  In host code the array's name is only a
// stand-in for the symbol, not a device address: the address each device gives it is looked up once per
// device with cudaGetSymbolAddress and that pointer is what the kernels receive.
constexpr size_t kStaticScratchBytes = VITCOP_STATIC_SCRATCH_BYTES;
static __device__ __align__(256) unsigned char g_static_scratch[kStaticScratchBytes];

namespace {
std::mutex g_scratch_mutex;
void* g_scratch_addr[kMaxDevices] = {};

// Device address of g_static_scratch on the current device (looked up on the first call per device).
int static_scratch_address(void** out) {
    int dev = -1;
    int rc = record_cuda(cudaGetDevice(&dev));
    if (rc != VITCOP_OK) return rc;
    if (dev < 0 || dev >= kMaxDevices) return VITCOP_ERR_UNSUPPORTED;
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_addr[dev]) {
        void* p = nullptr;
        rc = record_cuda(cudaGetSymbolAddress(&p, g_static_scratch));
        if (rc != VITCOP_OK) return rc;
        if (!p) return VITCOP_ERR_CUDA;
        g_scratch_addr[dev] = p;
    }
    *out = g_scratch_addr[dev];
    return VITCOP_OK;
}
}  // namespace

extern "C" {

const char* vitcop_status_string(int status) {
    switch (status) {
        case VITCOP_OK: return "ok";
        case VITCOP_ERR_INVALID_ARG: return "invalid argument";
        case VITCOP_ERR_UNSUPPORTED: return "unsupported shape or alignment";
        case VITCOP_ERR_WORKSPACE: return "workspace missing or too small";
        case VITCOP_ERR_BUDGET: return "budget smaller than the number of clusters";
        case VITCOP_ERR_CUDA: return "CUDA runtime error";
        case VITCOP_ERR_TIMEOUT: return "bounded device wait expired";
        default: return "unknown status";
    }
}

int vitcop_last_cuda_error(void) { return g_last_cuda_error; }

int vitcop_set_wait_limit(unsigned long long limit_ns, int expire_roles) {
    gram_set_wait_debug(limit_ns, expire_roles);
    return VITCOP_OK;
}

int vitcop_kernel_timing_begin(void) {
    std::lock_guard<std::mutex> lock(g_timing_mutex);
    for (auto& t : g_timed) { cudaEventDestroy(t.start); cudaEventDestroy(t.stop); }
    g_timed.clear();
    g_timing_on.store(true);
    return VITCOP_OK;
}

int vitcop_kernel_timing_end(vitcop_kernel_time* out, int capacity, int* count) {
    if (!count || capacity < 0 || (capacity > 0 && !out)) return VITCOP_ERR_INVALID_ARG;
    g_timing_on.store(false);
    std::lock_guard<std::mutex> lock(g_timing_mutex);
    int n = 0, rc = VITCOP_OK;
    for (auto& t : g_timed) {
        float ms = 0.f;
        if (t.complete && rc == VITCOP_OK) {
            rc = record_cuda(cudaEventSynchronize(t.stop));
            if (rc == VITCOP_OK) rc = record_cuda(cudaEventElapsedTime(&ms, t.start, t.stop));
            if (rc == VITCOP_OK) {
                int k = 0;
                while (k < n && std::strncmp(out[k].name, t.name, sizeof(out[k].name) - 1) != 0) ++k;
                if (k == n && n < capacity) {
                    std::memset(&out[n], 0, sizeof(out[n]));
                    std::strncpy(out[n].name, t.name, sizeof(out[n].name) - 1);
                    ++n;
                }
                if (k < n) { out[k].launches += 1; out[k].total_ms += ms; }
            }
        }
        cudaEventDestroy(t.start);
        cudaEventDestroy(t.stop);
    }
    g_timed.clear();
    *count = n;
    return rc;
}

// More query rows than the attention over the cache counts (their product may pass 64 bits).
static bool too_many_queries(int B, int Hq, int Tq) {
    const int64_t rows = (int64_t)Hq * Tq;
    return rows > 0 && B > 0x7fffffff / rows;
}

int vitcop_workspace_bytes(int op, int B, int H, int N, int d, int Nv, int D, int Dh, size_t* bytes) {
    (void)Dh;
    if (!bytes || B < 0 || Nv < 0 || D < 0) return VITCOP_ERR_INVALID_ARG;
    switch (op) {
        case VITCOP_OP_FILTER: *bytes = filter_workspace_bytes(B, Nv, D); return VITCOP_OK;
        case VITCOP_OP_SIMILARITY: *bytes = similarity_workspace_bytes(B, Nv, D); return VITCOP_OK;
        case VITCOP_OP_KNORM: *bytes = 0; return VITCOP_OK;
        case VITCOP_OP_COMPACT: *bytes = 0; return VITCOP_OK;
        case VITCOP_OP_SELECT: *bytes = kStatusBytes; return VITCOP_OK;
        case VITCOP_OP_PRUNE_STEP: *bytes = StepWs(B, Nv).total; return VITCOP_OK;
        case VITCOP_OP_COLLAB_STEP:
            *bytes = align_up(filter_workspace_bytes(B, Nv, D), 256) + StepWs(B, Nv).total;
            return VITCOP_OK;
        case VITCOP_OP_MERGE:
            if (N < 0) return VITCOP_ERR_INVALID_ARG;
            *bytes = merge_workspace_bytes(B, Nv, N);
            return VITCOP_OK;
        case VITCOP_OP_KPROJ:
            if (H < 0 || N < 0 || d < 0) return VITCOP_ERR_INVALID_ARG;
            *bytes = kproj_workspace_bytes(B, N, H, d);
            return VITCOP_OK;
        case VITCOP_OP_SALIENCY:
            if (H < 0 || N < 0) return VITCOP_ERR_INVALID_ARG;
            *bytes = saliency_workspace_bytes(B, H, N);
            return VITCOP_OK;
        case VITCOP_OP_CACHE_ATTENTION:
            if (H < 0 || N < 0 || d < 0) return VITCOP_ERR_INVALID_ARG;
            if (too_many_queries(B, D, Nv)) return VITCOP_ERR_UNSUPPORTED;
            *bytes = cache_attention_workspace_bytes(B, H, N, d, Nv, D);
            return VITCOP_OK;
        case VITCOP_OP_ATTENTION:
            if (H < 0 || N < 0 || d < 0) return VITCOP_ERR_INVALID_ARG;
            if (too_many_queries(B, D, Nv)) return VITCOP_ERR_UNSUPPORTED;
            *bytes = attention_workspace_bytes(B, H, N, d, Nv, D);
            return VITCOP_OK;
        default: return VITCOP_ERR_INVALID_ARG;
    }
}

int vitcop_poll_status(const void* workspace, void* stream, int* device_status) {
    if (!workspace || !device_status) return VITCOP_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int v = 0;
    int rc = record_cuda(cudaMemcpyAsync(&v, workspace, sizeof(int), cudaMemcpyDeviceToHost, s));
    if (rc != VITCOP_OK) return rc;
    rc = record_cuda(cudaStreamSynchronize(s));
    if (rc != VITCOP_OK) return rc;
    if ((v & ~(kStatusInReports - 1)) == kStatusInReports) {
        uint8_t reports[kMaxReports];
        const int n = std::min(v & (kStatusInReports - 1), kMaxReports);
        rc = record_cuda(cudaMemcpyAsync(reports, static_cast<const char*>(workspace) + kReportsAt, n, cudaMemcpyDeviceToHost, s));
        if (rc != VITCOP_OK) return rc;
        rc = record_cuda(cudaStreamSynchronize(s));
        if (rc != VITCOP_OK) return rc;
        v = std::any_of(reports, reports + n, [](uint8_t r) { return r != 0; }) ? VITCOP_ERR_TIMEOUT : VITCOP_OK;
    }
    *device_status = v;
    return VITCOP_OK;
}

int vitcop_knorm_score(const void* K, int B, int H, int N, int d, int64_t stride_b, int64_t stride_h,
                       int64_t stride_n, int vis_start, const int32_t* vis_len, int vis_len_uniform, float* score,
                       int Nv_cap, void* stream) {
    if (!K || !score || B < 0 || H < 0 || N < 0 || d < 0 || Nv_cap < 0) return VITCOP_ERR_INVALID_ARG;
    if (stride_b < 0 || stride_h < 0 || stride_n < 0) return VITCOP_ERR_INVALID_ARG;
    int rc = check_span(N, vis_start, vis_len, vis_len_uniform, Nv_cap);
    if (rc != VITCOP_OK) return rc;
    if (d % 8 || stride_b % 8 || stride_h % 8 || stride_n % 8 || !aligned16(K)) return VITCOP_ERR_UNSUPPORTED;
    if (B > 65535) return VITCOP_ERR_UNSUPPORTED;
    return launch_knorm(K, B, H, d, stride_b, stride_h, stride_n, vis_start, vis_len, vis_len_uniform, score, Nv_cap,
                        static_cast<cudaStream_t>(stream));
}

int vitcop_select(const float* score, const int32_t* label, int B, const int32_t* vis_len, int vis_len_uniform,
                  int Nv_cap, const vitcop_select_params* p, int32_t* keep_idx, int keep_stride, int32_t* n_keep,
                  uint8_t* keep_mask, void* workspace, size_t workspace_bytes, void* stream) {
    if (!score || !p || !keep_idx || !n_keep || B < 0 || Nv_cap < 0 || keep_stride < 0) return VITCOP_ERR_INVALID_ARG;
    if (p->mode != 0 && p->mode != 1) return VITCOP_ERR_INVALID_ARG;
    if (p->budget < 0) return VITCOP_ERR_INVALID_ARG;
    if (p->mode == 1 && !label) return VITCOP_ERR_INVALID_ARG;
    if (!vis_len && (vis_len_uniform < 0 || vis_len_uniform > Nv_cap)) return VITCOP_ERR_INVALID_ARG;
    if (keep_stride < (p->budget < Nv_cap ? p->budget : Nv_cap)) return VITCOP_ERR_INVALID_ARG;
    if (Nv_cap > VITCOP_MAX_VISUAL_TOKENS) return VITCOP_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < kStatusBytes) return VITCOP_ERR_WORKSPACE;
    if (!aligned256(workspace)) return VITCOP_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // (quota mode: any of the CTAs may set the word, so none of them can clear it)
    int* const status = static_cast<int*>(workspace);
    const bool in_kernel = p->mode == 0 && B > 0;
    if (!in_kernel) {
        const int rc = reset_status(workspace, s);
        if (rc != VITCOP_OK) return rc;
    }
    return launch_select(score, label, B, vis_len, vis_len_uniform, Nv_cap, p->mode, p->largest ? 1 : 0, p->budget,
                         keep_idx, keep_stride, n_keep, keep_mask, status, s, in_kernel, in_kernel ? status : nullptr);
}

static int check_compact_args(const void* hidden, const void* K, const void* V, int B, int H, int N, int d, int Dh,
                              int vis_start, const int32_t* vis_len, int vis_len_uniform, void* hidden_out,
                              void* K_out, void* V_out, int Ncap) {
    if (B < 0 || H < 0 || N < 0 || d < 0 || Dh < 0 || Ncap < 0) return VITCOP_ERR_INVALID_ARG;
    if ((hidden == nullptr) != (hidden_out == nullptr)) return VITCOP_ERR_INVALID_ARG;
    if ((K == nullptr) != (K_out == nullptr)) return VITCOP_ERR_INVALID_ARG;
    if ((V == nullptr) != (V_out == nullptr)) return VITCOP_ERR_INVALID_ARG;
    int rc = check_span(N, vis_start, vis_len, vis_len_uniform, -1);
    if (rc != VITCOP_OK) return rc;
    if (d % 8 || Dh % 8) return VITCOP_ERR_UNSUPPORTED;
    if (!aligned16(hidden) || !aligned16(K) || !aligned16(V) || !aligned16(hidden_out) || !aligned16(K_out) ||
        !aligned16(V_out))
        return VITCOP_ERR_UNSUPPORTED;
    if (B > 65535) return VITCOP_ERR_UNSUPPORTED;
    const size_t hin = (size_t)B * N * Dh * 2, hout = (size_t)B * Ncap * Dh * 2;
    const size_t kin = (size_t)B * H * N * d * 2, kout = (size_t)B * H * Ncap * d * 2;
    const void* ins[3] = {hidden, K, V};
    const size_t insz[3] = {hin, kin, kin};
    const void* outs[3] = {hidden_out, K_out, V_out};
    const size_t outsz[3] = {hout, kout, kout};
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < 3; ++j)
            if (overlaps(ins[i], insz[i], outs[j], outsz[j])) return VITCOP_ERR_INVALID_ARG;
    return VITCOP_OK;
}

int vitcop_compact_kv(const void* hidden, const void* K, const void* V, int B, int H, int N, int d, int Dh,
                      const int32_t* seq_len, int vis_start, const int32_t* vis_len, int vis_len_uniform,
                      const int32_t* keep_idx, int keep_stride, const int32_t* n_keep, void* hidden_out, void* K_out,
                      void* V_out, int Ncap, int32_t* kept_pos, int32_t* out_len, void* stream) {
    if (!keep_idx || !n_keep || !out_len || keep_stride < 0) return VITCOP_ERR_INVALID_ARG;
    int rc = check_compact_args(hidden, K, V, B, H, N, d, Dh, vis_start, vis_len, vis_len_uniform, hidden_out, K_out,
                                V_out, Ncap);
    if (rc != VITCOP_OK) return rc;
    return launch_compact(hidden, K, V, B, H, N, d, Dh, seq_len, vis_start, vis_len, vis_len_uniform, keep_idx,
                          keep_stride, n_keep, hidden_out, K_out, V_out, Ncap, kept_pos, out_len,
                          static_cast<cudaStream_t>(stream), /*early=*/false);
}

int vitcop_prune_step(const void* hidden, const void* K, const void* V, int B, int H, int N, int d, int Dh,
                      const int32_t* seq_len, int vis_start, const int32_t* vis_len, int vis_len_uniform, int Nv_cap,
                      const int32_t* label, int budget, void* hidden_out, void* K_out, void* V_out, int Ncap,
                      int32_t* kept_pos, int32_t* out_len, float* score_out, int32_t* keep_idx_out,
                      int32_t* n_keep_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (!K || !out_len || budget < 0 || Nv_cap < 0) return VITCOP_ERR_INVALID_ARG;
    int rc = check_compact_args(hidden, K, V, B, H, N, d, Dh, vis_start, vis_len, vis_len_uniform, hidden_out, K_out,
                                V_out, Ncap);
    if (rc != VITCOP_OK) return rc;
    rc = check_span(N, vis_start, vis_len, vis_len_uniform, Nv_cap);
    if (rc != VITCOP_OK) return rc;
    if (Nv_cap > VITCOP_MAX_VISUAL_TOKENS) return VITCOP_ERR_UNSUPPORTED;
    const StepWs lay(B, Nv_cap);
    if (!workspace || workspace_bytes < lay.total || !aligned256(workspace)) return VITCOP_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    float* score = score_out ? score_out : reinterpret_cast<float*>(ws + lay.off_score);
    int32_t* keep = keep_idx_out ? keep_idx_out : reinterpret_cast<int32_t*>(ws + lay.off_keep);
    int32_t* nkeep = n_keep_out ? n_keep_out : reinterpret_cast<int32_t*>(ws + lay.off_nkeep);
    bool have_knorm = false;
    rc = launch_knorm(K, B, H, d, (int64_t)H * N * d, (int64_t)N * d, d, vis_start, vis_len, vis_len_uniform, score,
                      Nv_cap, s, false, &have_knorm, reinterpret_cast<int*>(ws));
    if (rc != VITCOP_OK) return rc;
    if (!have_knorm) {
        rc = reset_status(workspace, s);
        if (rc != VITCOP_OK) return rc;
    }
    // The selection releases its dependents before it waits for its predecessor, and the compaction copies the rows
    // in front of the span before its own wait: that is safe only behind a kernel of this call that has itself
    // waited for everything queued before the call.  With an empty span there is no such kernel, so the selection
    // is then launched in plain stream order.
    if (have_knorm && !label && compact_selects(hidden != nullptr, V != nullptr, B, H, d, Dh, Nv_cap, Ncap)) {
        const SmallestJob smallest = {score, budget, keep, nkeep};
        return launch_compact(hidden, K, V, B, H, N, d, Dh, seq_len, vis_start, vis_len, vis_len_uniform, nullptr, Nv_cap,
                              nullptr, hidden_out, K_out, V_out, Ncap, kept_pos, out_len, s, true, &smallest);
    }
    rc = launch_select(score, label, B, vis_len, vis_len_uniform, Nv_cap, label ? 1 : 0, 0, budget, keep, Nv_cap,
                       nkeep, nullptr, reinterpret_cast<int*>(ws), s, have_knorm);
    if (rc != VITCOP_OK) return rc;
    return launch_compact(hidden, K, V, B, H, N, d, Dh, seq_len, vis_start, vis_len, vis_len_uniform, keep, Nv_cap,
                          nkeep, hidden_out, K_out, V_out, Ncap, kept_pos, out_len, s, true);
}

int vitcop_collaborative_step(const void* feat, const float* pos, int D, const vitcop_filter_params* fp,
                              const void* hidden, const void* K, const void* V, int B, int H, int N, int d, int Dh,
                              int vis_start, int Nv, int budget, void* hidden_out, void* K_out, void* V_out, int Ncap,
                              int32_t* kept_pos, int32_t* out_len, int32_t* label_out, int32_t* n_clusters_out,
                              float* rho_out, float* delta2_out, int32_t* parent_out, float* score_out,
                              int32_t* keep_idx_out, int32_t* n_keep_out, void* workspace, size_t workspace_bytes,
                              void* stream) {
    if (!feat || !fp || !K || !out_len || !label_out || !n_clusters_out || budget < 0 || Nv < 0 || D < 0)
        return VITCOP_ERR_INVALID_ARG;
    if (fp->metric != 0 && fp->metric != 1) return VITCOP_ERR_INVALID_ARG;
    if (!(fp->d_c > 0.f)) return VITCOP_ERR_INVALID_ARG;
    int rc = check_compact_args(hidden, K, V, B, H, N, d, Dh, vis_start, nullptr, Nv, hidden_out, K_out, V_out, Ncap);
    if (rc != VITCOP_OK) return rc;
    rc = check_span(N, vis_start, nullptr, Nv, Nv);
    if (rc != VITCOP_OK) return rc;
    if (D % 64 || !aligned16(feat) || !aligned8(pos) || Nv > VITCOP_MAX_VISUAL_TOKENS || B > 65535)
        return VITCOP_ERR_UNSUPPORTED;
    const StepWs lay(B, Nv);
    size_t filter_bytes = align_up(filter_workspace_bytes(B, Nv, D), 256);
    if (!workspace || workspace_bytes < lay.total || !aligned256(workspace)) return VITCOP_ERR_WORKSPACE;
    if (workspace_bytes - lay.total < filter_bytes) filter_bytes = (workspace_bytes - lay.total) / 256 * 256;
    if (filter_bytes < filter_workspace_least_bytes(B, Nv)) return VITCOP_ERR_WORKSPACE;
    int nc = fp->n_centers;
    if (nc <= 0) {
        const double v = std::ceil((double)Nv * fp->alpha);
        nc = v < 0 ? 0 : (v > Nv ? Nv : (int)v);
    }
    if (nc > Nv) nc = Nv;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    char* ws2 = ws + filter_bytes;
    float* score = score_out ? score_out : reinterpret_cast<float*>(ws2 + lay.off_score);
    int32_t* keep = keep_idx_out ? keep_idx_out : reinterpret_cast<int32_t*>(ws2 + lay.off_keep);
    int32_t* nkeep = n_keep_out ? n_keep_out : reinterpret_cast<int32_t*>(ws2 + lay.off_nkeep);
    if (B == 0 || Nv == 0) {
        rc = reset_status(workspace, s);
        if (rc != VITCOP_OK || B == 0) return rc;
    }
    QuotaJob quota = {score, budget, keep, nkeep, false};
    if (Nv > 0) {
        const KnormJob job = {K, B, H, N, d, vis_start, Nv, score};
        rc = launch_filter(feat, pos, B, Nv, D, *fp, nc, label_out, n_clusters_out, rho_out, delta2_out, parent_out,
                           workspace, filter_bytes, s, &job, &quota);
        if (rc != VITCOP_OK) return rc;
    }
    if (!quota.taken) {
        // (plain stream order when the filter was skipped: see vitcop_prune_step)
        rc = launch_select(score, label_out, B, nullptr, Nv, Nv, 1, 0, budget, keep, Nv, nkeep, nullptr,
                           reinterpret_cast<int*>(ws), s, Nv > 0);
        if (rc != VITCOP_OK) return rc;
    }
    return launch_compact(hidden, K, V, B, H, N, d, Dh, nullptr, vis_start, nullptr, Nv, keep, Nv, nkeep, hidden_out,
                          K_out, V_out, Ncap, kept_pos, out_len, s, true);
}

int vitcop_merge_clusters(const void* hidden, int B, int N, int Dh, int vis_start, const int32_t* vis_len,
                          int vis_len_uniform, int Nv_cap, const int32_t* label, const uint8_t* keep_mask, void* merged,
                          float* merged_f32, int32_t* merged_label, int32_t* merged_count, int32_t* n_merged, int Mcap,
                          void* workspace, size_t workspace_bytes, void* stream) {
    if (!hidden || !label || !keep_mask || !merged_label || !merged_count || !n_merged) return VITCOP_ERR_INVALID_ARG;
    if (B < 0 || N < 0 || Dh < 0 || Nv_cap < 0 || Mcap < 0) return VITCOP_ERR_INVALID_ARG;
    int rc = check_span(N, vis_start, vis_len, vis_len_uniform, Nv_cap);
    if (rc != VITCOP_OK) return rc;
    if (Dh % 8 || !aligned16(hidden) || !aligned16(merged) || !aligned16(merged_f32)) return VITCOP_ERR_UNSUPPORTED;
    if (Nv_cap > VITCOP_MAX_VISUAL_TOKENS || B > 65535) return VITCOP_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < merge_workspace_bytes(B, Nv_cap, Mcap) || !aligned256(workspace))
        return VITCOP_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (B == 0) return reset_status(workspace, s);
    return launch_merge(hidden, B, N, Dh, vis_start, vis_len, vis_len_uniform, Nv_cap, label, keep_mask, merged,
                        merged_f32, merged_label, merged_count, n_merged, Mcap, workspace, s);
}

int vitcop_cls_saliency(const void* q_cls, const void* K, int B, int H, int M, int d, float scale, float* saliency,
                        float* cls_self, void* workspace, size_t workspace_bytes, void* stream) {
    if (!q_cls || !K || (!saliency && M > 1) || B < 0 || H < 0 || M < 0 || d < 0) return VITCOP_ERR_INVALID_ARG;
    if (d % 8 || !aligned16(q_cls) || !aligned16(K) || B > 65535 || H > 4096 || d > 4096) return VITCOP_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < saliency_workspace_bytes(B, H, M) || !aligned256(workspace))
        return VITCOP_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (B == 0 || H == 0 || M == 0) return reset_status(workspace, s);
    return launch_cls_saliency(q_cls, K, B, H, M, d, scale, saliency, cls_self, workspace, s);
}

int vitcop_kproj_knorm(const void* hidden, const void* W_k, int B, int N, int Dh, int H, int d, const float* rope_cos,
                       const float* rope_sin, const int32_t* position_ids, int n_pos, void* K_out, int vis_start, int Nv,
                       float* score, void* workspace, size_t workspace_bytes, void* stream) {
    if (!hidden || !W_k || !K_out || B < 0 || N < 0 || Dh < 0 || H < 0 || d < 0 || Nv < 0 || vis_start < 0)
        return VITCOP_ERR_INVALID_ARG;
    if ((rope_cos == nullptr) != (rope_sin == nullptr)) return VITCOP_ERR_INVALID_ARG;
    if (rope_cos && n_pos <= 0) return VITCOP_ERR_INVALID_ARG;
    if (score && vis_start + (int64_t)Nv > N) return VITCOP_ERR_INVALID_ARG;
    if (Dh % 64 || d % 32 || !aligned16(hidden) || !aligned16(W_k) || !aligned16(K_out)) return VITCOP_ERR_UNSUPPORTED;
    if (rope_cos && ((d != 64 && d != 128 && d != 256) || !aligned16(rope_cos) || !aligned16(rope_sin)))
        return VITCOP_ERR_UNSUPPORTED;
    if ((int64_t)B * N > 0x7fffffff || (int64_t)H * d > 0x7fffffff || B > 65535) return VITCOP_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < kproj_workspace_bytes(B, N, H, d) || !aligned256(workspace))
        return VITCOP_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (B == 0 || N == 0 || H == 0 || d == 0 || Dh == 0) return reset_status(workspace, s);
    return launch_kproj_knorm(hidden, W_k, B, N, Dh, H, d, rope_cos, rope_sin, position_ids, n_pos, K_out, vis_start,
                              score ? Nv : 0, score, workspace, s);
}

// Bytes that a tensor [B, H, N, d] of 2-byte elements with these strides (elements, not negative) reaches over.
static size_t extent(int B, int H, int N, int d, int64_t sb, int64_t sh, int64_t sn) {
    if (B <= 0 || H <= 0 || N <= 0 || d <= 0) return 0;
    return ((size_t)(B - 1) * (size_t)sb + (size_t)(H - 1) * (size_t)sh + (size_t)(N - 1) * (size_t)sn + (size_t)d) * 2;
}

// Whether rows of such a tensor share elements: in the order of their strides, each dimension has to step over what those before it reach.
static bool rows_share(int B, int H, int N, int d, int64_t sb, int64_t sh, int64_t sn) {
    struct Dim {
        int64_t n, stride;
    } dims[3] = {{B, sb}, {H, sh}, {N, sn}};
    std::sort(dims, dims + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
    int64_t reach = d;
    for (const Dim& dim : dims) {
        if (dim.n <= 1) continue;
        if (dim.stride < reach) return true;
        int64_t span;
        if (__builtin_mul_overflow(dim.n - 1, dim.stride, &span) || __builtin_add_overflow(reach, span, &reach)) return true;
    }
    return false;
}

static int check_cache(int B, int H, int Ncap, int d, const void* cache) {
    if (!cache && cache_bytes(B, H, Ncap, d) > 0) return VITCOP_ERR_INVALID_ARG;
    if ((d != 64 && d != 128 && d != 256) || Ncap % kCacheBlock || !aligned16(cache)) return VITCOP_ERR_UNSUPPORTED;
    return VITCOP_OK;
}

int vitcop_cache_write(const void* K, const void* V, int B, int H, int N, int d, int64_t k_stride_b, int64_t k_stride_h,
                       int64_t k_stride_n, int64_t v_stride_b, int64_t v_stride_h, int64_t v_stride_n, const int32_t* seq_len,
                       int vis_start, const int32_t* vis_len, int vis_len_uniform, const int32_t* keep_idx, int keep_stride,
                       const int32_t* n_keep, const int32_t* cache_len, void* cache, int Ncap, int32_t* new_len, void* stream) {
    if (B < 0 || H < 0 || N < 0 || d <= 0 || Ncap < 0) return VITCOP_ERR_INVALID_ARG;
    if ((!K && !V && extent(B, H, N, d, 0, 0, 0) > 0) || (!new_len && B > 0)) return VITCOP_ERR_INVALID_ARG;
    const int64_t strides[6] = {k_stride_b, k_stride_h, k_stride_n, v_stride_b, v_stride_h, v_stride_n};
    for (int i = 0; i < 6; ++i)
        if (strides[i] < 0) return VITCOP_ERR_INVALID_ARG;
    if (keep_idx) {
        if (!n_keep || keep_stride <= 0) return VITCOP_ERR_INVALID_ARG;
        const int rc = check_span(N, vis_start, vis_len, vis_len_uniform, -1);
        if (rc != VITCOP_OK) return rc;
    }
    const int rc = check_cache(B, H, Ncap, d, cache);
    if (rc != VITCOP_OK) return rc;
    for (int i = 0; i < 6; ++i)
        if (strides[i] % 8 && (i < 3 ? K : V)) return VITCOP_ERR_UNSUPPORTED;
    if (!aligned16(K) || !aligned16(V) || B > 65535) return VITCOP_ERR_UNSUPPORTED;
    const size_t kbytes = K ? extent(B, H, N, d, k_stride_b, k_stride_h, k_stride_n) : 0;
    const size_t vbytes = V ? extent(B, H, N, d, v_stride_b, v_stride_h, v_stride_n) : 0;
    const size_t cbytes = cache_bytes(B, H, Ncap, d), lens = (size_t)B * sizeof(int32_t);
    const size_t list = keep_idx ? (size_t)B * keep_stride * sizeof(int32_t) : 0;
    if (overlaps(K, kbytes, cache, cbytes) || overlaps(V, vbytes, cache, cbytes)) return VITCOP_ERR_INVALID_ARG;
    const void* ins[] = {K, V, cache_len, seq_len, keep_idx ? vis_len : nullptr, keep_idx, keep_idx ? n_keep : nullptr, cache};
    const size_t insz[] = {kbytes, vbytes, lens, lens, lens, list, lens, cbytes};
    for (int i = 0; i < 8; ++i)
        if (overlaps(ins[i], insz[i], new_len, lens)) return VITCOP_ERR_INVALID_ARG;
    for (int i = 2; i < 7; ++i)
        if (overlaps(ins[i], insz[i], cache, cbytes)) return VITCOP_ERR_INVALID_ARG;
    const auto bf16 = [](const void* p) { return static_cast<const __nv_bfloat16*>(p); };
    const CacheSource src = {bf16(K), bf16(V), k_stride_b, k_stride_h, k_stride_n, v_stride_b, v_stride_h, v_stride_n};
    const CacheRows rows = {seq_len, vis_start, vis_len, vis_len_uniform, keep_idx, keep_stride, n_keep};
    return launch_cache_write(src, rows, B, H, N, d, cache_len, cache, Ncap, new_len, static_cast<cudaStream_t>(stream));
}

int vitcop_cache_read(const void* cache, int B, int H, int Ncap, int d, const int32_t* cache_len, const int32_t* row_begin,
                      int row_begin_uniform, void* K_out, void* V_out, int N_out, void* stream) {
    if (B < 0 || H < 0 || Ncap < 0 || d <= 0 || N_out < 0) return VITCOP_ERR_INVALID_ARG;
    if (!K_out && !V_out && extent(B, H, N_out, d, 0, 0, 0) > 0) return VITCOP_ERR_INVALID_ARG;
    if (!row_begin && row_begin_uniform < 0) return VITCOP_ERR_INVALID_ARG;
    const int rc = check_cache(B, H, Ncap, d, cache);
    if (rc != VITCOP_OK) return rc;
    if (!aligned16(K_out) || !aligned16(V_out) || B > 65535) return VITCOP_ERR_UNSUPPORTED;
    const size_t cbytes = cache_bytes(B, H, Ncap, d), obytes = (size_t)B * H * N_out * d * 2, lens = (size_t)B * sizeof(int32_t);
    void* outs[] = {K_out, V_out};
    for (void* out : outs)
        if (overlaps(cache, cbytes, out, obytes) || overlaps(cache_len, lens, out, obytes) || overlaps(row_begin, lens, out, obytes))
            return VITCOP_ERR_INVALID_ARG;
    if (overlaps(K_out, obytes, V_out, obytes)) return VITCOP_ERR_INVALID_ARG;
    return launch_cache_read(cache, B, H, Ncap, d, cache_len, row_begin, row_begin_uniform, K_out, V_out, N_out,
                             static_cast<cudaStream_t>(stream));
}

int vitcop_cache_attention(const void* q, const void* cache, int B, int Hq, int H, int Tq, int d, int Ncap, int64_t q_stride_b,
                           int64_t q_stride_h, int64_t q_stride_t, const int32_t* cache_len, float scale, int causal, void* out,
                           int64_t out_stride_b, int64_t out_stride_h, int64_t out_stride_t, float* lse, void* workspace,
                           size_t workspace_bytes, void* stream) {
    if (B < 0 || Hq < 0 || H < 0 || Tq < 0 || d <= 0 || Ncap < 0) return VITCOP_ERR_INVALID_ARG;
    if ((!q || !out) && extent(B, Hq, Tq, d, 0, 0, 0) > 0) return VITCOP_ERR_INVALID_ARG;
    if (!(std::fabs(scale) <= 0x1p127f)) return VITCOP_ERR_INVALID_ARG;    // (NaN, infinite, or so in powers of two)
    if (H > 0 ? Hq % H != 0 : Hq != 0) return VITCOP_ERR_INVALID_ARG;
    const int64_t strides[6] = {q_stride_b, q_stride_h, q_stride_t, out_stride_b, out_stride_h, out_stride_t};
    for (int i = 0; i < 6; ++i)
        if (strides[i] < 0) return VITCOP_ERR_INVALID_ARG;
    const int rc = check_cache(B, H, Ncap, d, cache);
    if (rc != VITCOP_OK) return rc;
    for (int i = 0; i < 6; ++i)
        if (strides[i] % 8) return VITCOP_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(out) || B > 65535) return VITCOP_ERR_UNSUPPORTED;
    // (rows of the output that share elements have no value)
    if (extent(B, Hq, Tq, d, 0, 0, 0) > 0 && rows_share(B, Hq, Tq, d, out_stride_b, out_stride_h, out_stride_t)) return VITCOP_ERR_INVALID_ARG;
    if (too_many_queries(B, Hq, Tq)) return VITCOP_ERR_UNSUPPORTED;
    const size_t need = cache_attention_workspace_bytes(B, H, Ncap, d, Tq, Hq);
    const size_t obytes = extent(B, Hq, Tq, d, out_stride_b, out_stride_h, out_stride_t);
    const size_t rows = (size_t)B * Hq * Tq * sizeof(float), lens = (size_t)B * sizeof(int32_t);
    const void* ins[] = {q, cache, cache_len};
    const size_t insz[] = {extent(B, Hq, Tq, d, q_stride_b, q_stride_h, q_stride_t), cache_bytes(B, H, Ncap, d), lens};
    for (int i = 0; i < 3; ++i)
        if (overlaps(ins[i], insz[i], out, obytes) || overlaps(ins[i], insz[i], lse, rows) || overlaps(ins[i], insz[i], workspace, need))
            return VITCOP_ERR_INVALID_ARG;
    if (overlaps(out, obytes, lse, rows) || overlaps(out, obytes, workspace, need) || overlaps(lse, rows, workspace, need))
        return VITCOP_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < need || !aligned256(workspace)) return VITCOP_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (B == 0 || Hq == 0 || Tq == 0) return reset_status(workspace, s);
    const CacheQueries io = {static_cast<const __nv_bfloat16*>(q), static_cast<__nv_bfloat16*>(out), q_stride_b, q_stride_h, q_stride_t,
                             out_stride_b, out_stride_h, out_stride_t};
    return launch_cache_attention(io, cache, B, Hq, H, Tq, d, Ncap, cache_len, scale, causal != 0, lse, workspace, s);
}

// Whether two such tensors may share elements.  Not where they lie apart, nor where one lies in the gaps of the other: tokens (or samples) step alike, and
// what a token (a sample) reaches over has places of its own inside that step.
struct Rows4 {
    const void* data;
    int H;
    int64_t sb, sh, sn;
    size_t bytes;                                          // reached over
};
static bool rows_meet(const Rows4& x, const Rows4& y, int B, int N, int d) {
    if (!overlaps(x.data, x.bytes, y.data, y.bytes)) return false;
    const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(y.data) - reinterpret_cast<uintptr_t>(x.data)) / 2;
    const auto in_gaps = [&](int64_t step, int64_t reach_x, int64_t reach_y) {
        const int64_t at = (apart % step + step) % step;
        return at >= reach_x && at + reach_y <= step;
    };
    const int64_t token_x = (x.H - 1) * x.sh + d, token_y = (y.H - 1) * y.sh + d;
    if (N > 1 && x.sn == y.sn && x.sn > 0 && (B <= 1 || (x.sb % x.sn == 0 && y.sb % y.sn == 0)) && in_gaps(x.sn, token_x, token_y)) return false;
    return !(B > 1 && x.sb == y.sb && x.sb > 0 && in_gaps(x.sb, token_x + (N - 1) * x.sn, token_y + (N - 1) * y.sn));
}

int vitcop_rotary_axes(const void* q, const void* k, int B, int Hq, int Hk, int N, int d, int64_t q_stride_b, int64_t q_stride_h,
                       int64_t q_stride_t, int64_t k_stride_b, int64_t k_stride_h, int64_t k_stride_t, const int32_t* position, int axes,
                       int n_pos, const int32_t* token, const int32_t* seq_len, const double* inv_freq, const int32_t* axis, int n_freq,
                       int inverse, void* q_out, int64_t qo_stride_b, int64_t qo_stride_h, int64_t qo_stride_t, void* k_out,
                       int64_t ko_stride_b, int64_t ko_stride_h, int64_t ko_stride_t, void* stream) {
    if (B < 0 || Hq < 0 || Hk < 0 || N < 0 || d <= 0 || axes < 1 || n_pos < 0 || n_freq < 0) return VITCOP_ERR_INVALID_ARG;
    // (tensors of no elements have no address)
    const bool any = B > 0 && N > 0 && (int64_t)Hq + Hk > 0;
    if ((!q && !k && any) || (q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr)) return VITCOP_ERR_INVALID_ARG;
    const int64_t strides[12] = {q_stride_b, q_stride_h, q_stride_t, qo_stride_b, qo_stride_h, qo_stride_t,
                                 k_stride_b, k_stride_h, k_stride_t, ko_stride_b, ko_stride_h, ko_stride_t};
    for (int i = 0; i < 12; ++i)
        if (strides[i] < 0) return VITCOP_ERR_INVALID_ARG;
    if (n_freq > 0 && (!inv_freq || !axis)) return VITCOP_ERR_INVALID_ARG;
    if (B > 0 && N > 0 && (n_pos == 0 || (n_freq > 0 && !position) || (!token && n_pos < N))) return VITCOP_ERR_INVALID_ARG;
    if (d % 8 || d > 4096 || n_freq % 8 || 2 * (int64_t)n_freq > d || n_freq > kMostFrequencies || Hq > 32767 || Hk > 32767) return VITCOP_ERR_UNSUPPORTED;
    for (int i = 0; i < 12; ++i)
        if (strides[i] % 8 && (i < 6 ? q : k)) return VITCOP_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !aligned8(inv_freq) || B > 65535) return VITCOP_ERR_UNSUPPORTED;
    if (!q) Hq = 0;
    if (!k) Hk = 0;
    if (N > 0 && (int64_t)B * N > 0x7fff0000 / std::max<int64_t>(1, (int64_t)Hq + Hk)) return VITCOP_ERR_UNSUPPORTED;
    if (B == 0 || N == 0 || Hq + Hk == 0) return VITCOP_OK;
    const Rows4 rows[4] = {{q, Hq, q_stride_b, q_stride_h, q_stride_t, extent(B, Hq, N, d, q_stride_b, q_stride_h, q_stride_t)},
                           {k, Hk, k_stride_b, k_stride_h, k_stride_t, extent(B, Hk, N, d, k_stride_b, k_stride_h, k_stride_t)},
                           {q_out, Hq, qo_stride_b, qo_stride_h, qo_stride_t, extent(B, Hq, N, d, qo_stride_b, qo_stride_h, qo_stride_t)},
                           {k_out, Hk, ko_stride_b, ko_stride_h, ko_stride_t, extent(B, Hk, N, d, ko_stride_b, ko_stride_h, ko_stride_t)}};
    const size_t n = sizeof(int32_t), lens = (size_t)B * n;
    const void* small[] = {position, token, seq_len, inv_freq, axis};
    const size_t bytes[] = {(size_t)axes * B * n_pos * n, token ? lens * N : 0, lens, (size_t)n_freq * sizeof(double), (size_t)n_freq * n};
    for (int o = 2; o < 4; ++o) {
        const Rows4& out = rows[o];
        if (out.bytes == 0) continue;
        if (rows_share(B, out.H, N, d, out.sb, out.sh, out.sn)) return VITCOP_ERR_INVALID_ARG;
        for (int i = 0; i < 5; ++i)
            if (overlaps(small[i], bytes[i], out.data, out.bytes)) return VITCOP_ERR_INVALID_ARG;
        for (int i = 0; i < 4; ++i) {
            const Rows4& x = rows[i];
            const bool in_place = i == o - 2 && x.data == out.data && x.sb == out.sb && x.sh == out.sh && x.sn == out.sn;
            if (i != o && x.bytes > 0 && !in_place && rows_meet(x, out, B, N, d)) return VITCOP_ERR_INVALID_ARG;
        }
    }
    RotaryArgs a = {};
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.k = static_cast<const __nv_bfloat16*>(k);
    a.q_out = static_cast<__nv_bfloat16*>(q_out);
    a.k_out = static_cast<__nv_bfloat16*>(k_out);
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = strides[i];
        a.qo[i] = strides[3 + i];
        a.ks[i] = strides[6 + i];
        a.ko[i] = strides[9 + i];
    }
    a.position = position;
    a.token = token;
    a.seq_len = seq_len;
    a.axis = axis;
    a.inv_freq = inv_freq;
    a.B = B;
    a.Hq = Hq;
    a.Hk = Hk;
    a.N = N;
    a.d = d;
    a.axes = axes;
    a.n_pos = n_pos;
    a.F = n_freq;
    a.inverse = inverse != 0;
    return launch_rotary_axes(a, static_cast<cudaStream_t>(stream));
}

// What the two calls of the attention over bf16 rows have in common.
struct AttentionCall {
    const void *q, *K, *V;
    int B, Hq, H, Tq, d, N;
    int64_t at[12];                                        // strides of q, K, V, out
    const int32_t *cache_len, *query_len;
    const int64_t* tree;
    int window, n_sink;
    float scale;
    void* out;
    float* lse;
    void* workspace;
    size_t workspace_bytes;
};
static int run_attention(const AttentionCall& c, bool is_tree, void* stream) {
    if (c.B < 0 || c.Hq < 0 || c.H < 0 || c.Tq < 0 || c.d <= 0 || c.N < 0 || c.window < 0 || c.n_sink < 0) return VITCOP_ERR_INVALID_ARG;
    const size_t queries = extent(c.B, c.Hq, c.Tq, c.d, 0, 0, 0);
    if ((!c.q || !c.out || (is_tree && !c.tree)) && queries > 0) return VITCOP_ERR_INVALID_ARG;
    if ((!c.K || !c.V) && queries > 0 && c.N > 0) return VITCOP_ERR_INVALID_ARG;
    if (!(std::fabs(c.scale) <= 0x1p127f)) return VITCOP_ERR_INVALID_ARG;  // (NaN, infinite, or so in powers of two)
    if (c.H > 0 ? c.Hq % c.H != 0 : c.Hq != 0) return VITCOP_ERR_INVALID_ARG;
    for (int64_t s : c.at)
        if (s < 0) return VITCOP_ERR_INVALID_ARG;
    if ((c.d != 64 && c.d != 128 && c.d != 256) || c.B > 65535 || c.N > 0x7fff0000 || (is_tree && c.Tq > 64)) return VITCOP_ERR_UNSUPPORTED;
    for (int64_t s : c.at)
        if (s % 8) return VITCOP_ERR_UNSUPPORTED;
    if (!aligned16(c.q) || !aligned16(c.K) || !aligned16(c.V) || !aligned16(c.out) || !aligned8(c.tree)) return VITCOP_ERR_UNSUPPORTED;
    // (rows of the output that share elements have no value)
    if (queries > 0 && rows_share(c.B, c.Hq, c.Tq, c.d, c.at[9], c.at[10], c.at[11])) return VITCOP_ERR_INVALID_ARG;
    if (too_many_queries(c.B, c.Hq, c.Tq)) return VITCOP_ERR_UNSUPPORTED;
    const size_t need = attention_workspace_bytes(c.B, c.H, c.N, c.d, c.Tq, c.Hq), lens = (size_t)c.B * sizeof(int32_t);
    const size_t obytes = extent(c.B, c.Hq, c.Tq, c.d, c.at[9], c.at[10], c.at[11]), rows = (size_t)c.B * c.Hq * c.Tq * sizeof(float);
    const void* ins[] = {c.q, c.K, c.V, c.cache_len, c.query_len, c.tree};
    const size_t insz[] = {extent(c.B, c.Hq, c.Tq, c.d, c.at[0], c.at[1], c.at[2]), extent(c.B, c.H, c.N, c.d, c.at[3], c.at[4], c.at[5]),
                           extent(c.B, c.H, c.N, c.d, c.at[6], c.at[7], c.at[8]), lens, lens, (size_t)c.B * c.Tq * sizeof(int64_t)};
    for (int i = 0; i < 6; ++i)
        if (overlaps(ins[i], insz[i], c.out, obytes) || overlaps(ins[i], insz[i], c.lse, rows) || overlaps(ins[i], insz[i], c.workspace, need))
            return VITCOP_ERR_INVALID_ARG;
    if (overlaps(c.out, obytes, c.lse, rows) || overlaps(c.out, obytes, c.workspace, need) || overlaps(c.lse, rows, c.workspace, need))
        return VITCOP_ERR_INVALID_ARG;
    if (!c.workspace || c.workspace_bytes < need || !aligned256(c.workspace)) return VITCOP_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (queries == 0) return reset_status(c.workspace, s);
    const auto bf16 = [](const void* p) { return static_cast<const __nv_bfloat16*>(p); };
    const SeqRows io = {bf16(c.q), bf16(c.K), bf16(c.V), static_cast<__nv_bfloat16*>(c.out), {c.at[0], c.at[1], c.at[2]},
                        {c.at[3], c.at[4], c.at[5]}, {c.at[6], c.at[7], c.at[8]}, {c.at[9], c.at[10], c.at[11]}};
    return launch_attention(io, c.B, c.Hq, c.H, c.Tq, c.d, c.N, c.cache_len, c.query_len, is_tree ? c.tree : nullptr, c.window, c.n_sink, c.scale,
                            c.lse, c.workspace, s);
}

int vitcop_window_attention(const void* q, const void* K, const void* V, int B, int Hq, int H, int Tq, int d, int N, int64_t q_stride_b,
                            int64_t q_stride_h, int64_t q_stride_t, int64_t k_stride_b, int64_t k_stride_h, int64_t k_stride_n,
                            int64_t v_stride_b, int64_t v_stride_h, int64_t v_stride_n, const int32_t* cache_len, const int32_t* query_len,
                            int window, int n_sink, float scale, void* out, int64_t out_stride_b, int64_t out_stride_h, int64_t out_stride_t,
                            float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    return run_attention({q, K, V, B, Hq, H, Tq, d, N,
                          {q_stride_b, q_stride_h, q_stride_t, k_stride_b, k_stride_h, k_stride_n, v_stride_b, v_stride_h, v_stride_n, out_stride_b,
                           out_stride_h, out_stride_t},
                          cache_len, query_len, nullptr, window, n_sink, scale, out, lse, workspace, workspace_bytes}, false, stream);
}

int vitcop_tree_attention(const void* q, const void* K, const void* V, int B, int Hq, int H, int Tq, int d, int N, int64_t q_stride_b,
                          int64_t q_stride_h, int64_t q_stride_t, int64_t k_stride_b, int64_t k_stride_h, int64_t k_stride_n,
                          int64_t v_stride_b, int64_t v_stride_h, int64_t v_stride_n, const int32_t* cache_len, const int32_t* query_len,
                          const int64_t* tree, float scale, void* out, int64_t out_stride_b, int64_t out_stride_h, int64_t out_stride_t, float* lse,
                          void* workspace, size_t workspace_bytes, void* stream) {
    return run_attention({q, K, V, B, Hq, H, Tq, d, N,
                          {q_stride_b, q_stride_h, q_stride_t, k_stride_b, k_stride_h, k_stride_n, v_stride_b, v_stride_h, v_stride_n, out_stride_b,
                           out_stride_h, out_stride_t},
                          cache_len, query_len, tree, 0, 0, scale, out, lse, workspace, workspace_bytes}, true, stream);
}

int vitcop_prune_step_static(const void* hidden, const void* K, const void* V, int B, int H, int N, int d, int Dh,
                             const int32_t* seq_len, int vis_start, const int32_t* vis_len, int vis_len_uniform,
                             int Nv_cap, const int32_t* label, int budget, void* hidden_out, void* K_out, void* V_out,
                             int Ncap, int32_t* kept_pos, int32_t* out_len, float* score_out, int32_t* keep_idx_out,
                             int32_t* n_keep_out, void* stream) {
    if (B < 0 || Nv_cap < 0) return VITCOP_ERR_INVALID_ARG;
    if (StepWs(B, Nv_cap).total > kStaticScratchBytes) return VITCOP_ERR_UNSUPPORTED;
    void* scratch = nullptr;
    const int rc = static_scratch_address(&scratch);
    if (rc != VITCOP_OK) return rc;
    return vitcop_prune_step(hidden, K, V, B, H, N, d, Dh, seq_len, vis_start, vis_len, vis_len_uniform, Nv_cap, label,
                             budget, hidden_out, K_out, V_out, Ncap, kept_pos, out_len, score_out, keep_idx_out,
                             n_keep_out, scratch, kStaticScratchBytes, stream);
}

int vitcop_redundancy_filter(const void* feat, const float* pos, int B, int n, int D, const vitcop_filter_params* p,
                             int32_t* label, int32_t* n_clusters, float* rho, float* delta2, int32_t* parent,
                             void* workspace, size_t workspace_bytes, void* stream) {
    if (!feat || !p || !label || !n_clusters || B < 0 || n < 0 || D < 0) return VITCOP_ERR_INVALID_ARG;
    if (p->metric != 0 && p->metric != 1) return VITCOP_ERR_INVALID_ARG;
    if (!(p->d_c > 0.f)) return VITCOP_ERR_INVALID_ARG;
    if (D % 64 || !aligned16(feat) || !aligned8(pos) || n > VITCOP_MAX_VISUAL_TOKENS || B > 65535)
        return VITCOP_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < filter_workspace_least_bytes(B, n) || !aligned256(workspace))
        return VITCOP_ERR_WORKSPACE;
    int nc = p->n_centers;
    if (nc <= 0) {
        const double v = std::ceil((double)n * p->alpha);
        nc = v < 0 ? 0 : (v > n ? n : (int)v);
    }
    if (nc > n) nc = n;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (B == 0 || n == 0) return reset_status(workspace, s);
    return launch_filter(feat, pos, B, n, D, *p, nc, label, n_clusters, rho, delta2, parent, workspace, workspace_bytes, s);
}

int vitcop_similarity_rows(const void* feat, int B, int n, int D, int metric, int row_begin, int row_end, float* out,
                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!feat || !out || B < 0 || n < 0 || D < 0) return VITCOP_ERR_INVALID_ARG;
    if (metric != 0 && metric != 1) return VITCOP_ERR_INVALID_ARG;
    if (row_begin < 0 || row_end < row_begin || row_end > n) return VITCOP_ERR_INVALID_ARG;
    if (D % 64 || !aligned16(feat) || n > VITCOP_MAX_VISUAL_TOKENS || B > 65535)
        return VITCOP_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < similarity_workspace_bytes(B, n, D) || !aligned256(workspace))
        return VITCOP_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int rc = reset_status(workspace, s);
    if (rc != VITCOP_OK) return rc;
    if (B == 0 || n == 0 || row_end == row_begin) return VITCOP_OK;
    return launch_similarity_rows(feat, B, n, D, metric, row_begin, row_end, out, workspace, s);
}

}  // extern "C"
