// C ABI of the operators for language models: argument checks, their workspace, dispatch.
#include "../../include/heinsen.h"
#include "operators.hpp"

#include <cmath>
#include <map>
#include <mutex>
#include <utility>
#include <vector>

namespace hs {
namespace {

// One grow-only buffer per (device, stream), held like the scan's scratch: replaced by a larger one after the work queued on
// it has drained, kept until heinsen_release_scratch where a captured call holds its address.
struct Workspace {
    void *memory = nullptr;
    size_t size = 0;
    bool in_graph = false;
    std::vector<void *> retired;
};

std::mutex g_mutex;
std::map<std::pair<int, hipStream_t>, Workspace> g_workspaces;

// The buffer's address in `out`.  Called with g_mutex held; the caller keeps it until its kernels are enqueued.
int workspace(hipStream_t stream, size_t want, void *&out)
{
    out = nullptr;
    if (want == 0) return HEINSEN_OK;
    int dev = 0;
    if (!note_hip(hipGetDevice(&dev))) return HEINSEN_ERR_HIP;
    const bool capturing = is_capturing(stream);
    const auto key = std::make_pair(dev, stream);
    if (capturing) {
        const auto it = g_workspaces.find(key);
        if (it == g_workspaces.end() || it->second.size < want) return HEINSEN_ERR_UNSUPPORTED;
        it->second.in_graph = true;
        out = it->second.memory;
        return HEINSEN_OK;
    }
    Workspace &w = g_workspaces[key];
    if (w.size < want) {
        if (w.memory && !note_hip(hipStreamSynchronize(stream))) return HEINSEN_ERR_HIP;
        if (w.memory) {
            if (w.in_graph) w.retired.push_back(w.memory);
            else (void)hipFree(w.memory);
        }
        w.memory = nullptr;
        w.size = 0;
        w.in_graph = false;
        const size_t size = align_up(want + want / 8, (size_t)1 << 21);
        void *p = nullptr;
        if (!note_hip(hipMalloc(&p, size))) return HEINSEN_ERR_ALLOC;
        w.memory = p;
        w.size = size;
    }
    out = w.memory;
    return HEINSEN_OK;
}

bool aligned(std::initializer_list<const void *> pointers, size_t to)
{
    for (const void *p : pointers)
        if (reinterpret_cast<uintptr_t>(p) % to != 0) return false;
    return true;
}

int make_attention(const void *q, const void *k, const void *v, const void *log_a, const void *s0, const void *starts, int64_t B, int64_t n,
                   int64_t H, int64_t Hk, int64_t K, int64_t V, int64_t q_stride, int64_t k_stride, int64_t v_stride, float scale,
                   uint32_t flags, void *stream, AttentionCall &c)
{
    if (!q || !k || !v) return HEINSEN_ERR_INVALID_ARG;
    if (B < 1 || n < 1 || H < 1 || Hk < 1 || K < 1 || V < 1 || H % Hk != 0) return HEINSEN_ERR_INVALID_ARG;
    if (flags & ~(uint32_t)(HEINSEN_IN_BF16 | HEINSEN_DECAY_PER_HEAD)) return HEINSEN_ERR_INVALID_ARG;
    if (!std::isfinite(scale)) return HEINSEN_ERR_INVALID_ARG;
    const bool bf16 = flags & HEINSEN_IN_BF16;
    if (!aligned({q, k, v, log_a}, bf16 ? 2 : 4) || !aligned({s0}, 4) || !aligned({starts}, 8)) return HEINSEN_ERR_INVALID_ARG;
    // indexes of workgroups and chunks are 32-bit, offsets 64-bit
    const int64_t many = (int64_t)1 << 24;
    if (K > 128 || V > 128 || H > many || B > many / H || n > ((int64_t)1 << 31) || B * n > ((int64_t)1 << 36)) return HEINSEN_ERR_UNSUPPORTED;
    const int64_t qk = Hk * K, values = H * V, most = (int64_t)1 << 23; // 64 tokens within 32 bits of bytes
    if (q_stride == 0) q_stride = qk;
    if (k_stride == 0) k_stride = qk;
    if (v_stride == 0) v_stride = values;
    if (q_stride < qk || k_stride < qk || v_stride < values) return HEINSEN_ERR_INVALID_ARG;
    if (q_stride > most || k_stride > most || v_stride > most) return HEINSEN_ERR_UNSUPPORTED;
    c.q = q, c.k = k, c.v = v, c.log_a = log_a;
    c.s0 = static_cast<const float *>(s0);
    c.starts = static_cast<const int64_t *>(starts);
    c.n = n, c.q_stride = q_stride, c.k_stride = k_stride, c.v_stride = v_stride;
    c.B = (int)B, c.H = (int)H, c.share = (int)(H / Hk), c.K = (int)K, c.V = (int)V;
    c.bf16 = bf16;
    c.per_head = flags & HEINSEN_DECAY_PER_HEAD;
    c.scale = scale;
    c.stream = static_cast<hipStream_t>(stream);
    return HEINSEN_OK;
}

int make_norm(const void *u, const void *gate, const void *residual, const void *scale, const void *w_post, const void *w_pre, int64_t rows,
              int64_t D, int64_t u_stride, int64_t gate_stride, float eps, uint32_t flags, void *stream, NormCall &c)
{
    if (!u || rows < 1 || D < 1) return HEINSEN_ERR_INVALID_ARG;
    if (flags & ~(uint32_t)(HEINSEN_IN_BF16 | HEINSEN_GATE_SIGMOID)) return HEINSEN_ERR_INVALID_ARG;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return HEINSEN_ERR_INVALID_ARG;
    const bool bf16 = flags & HEINSEN_IN_BF16;
    if (!aligned({u, gate, residual}, bf16 ? 2 : 4) || !aligned({scale, w_post, w_pre}, 4)) return HEINSEN_ERR_INVALID_ARG;
    if (u_stride == 0) u_stride = D;
    if (gate_stride == 0) gate_stride = D;
    if (u_stride < D || gate_stride < D) return HEINSEN_ERR_INVALID_ARG;
    const int64_t most = (int64_t)1 << 24;
    if (D > HEINSEN_NORM_MAX_D || rows > ((int64_t)1 << 40) || u_stride > most || gate_stride > most) return HEINSEN_ERR_UNSUPPORTED;
    c.u = u, c.gate = gate, c.residual = residual;
    c.scale = static_cast<const float *>(scale), c.w_post = static_cast<const float *>(w_post), c.w_pre = static_cast<const float *>(w_pre);
    c.rows = rows, c.u_stride = u_stride, c.gate_stride = gate_stride, c.D = (int)D, c.eps = eps;
    c.bf16 = bf16;
    c.sigmoid = flags & HEINSEN_GATE_SIGMOID;
    c.stream = static_cast<hipStream_t>(stream);
    return HEINSEN_OK;
}

// Workspace, then the call's kernels.
template <typename Call> int run(const Call &c, size_t want, hipError_t (*launch)(const Call &, void *))
{
    std::lock_guard<std::mutex> lock(g_mutex);
    void *scratch = nullptr;
    const int st = workspace(c.stream, want, scratch);
    if (st != HEINSEN_OK) return st;
    return note_hip(launch(c, scratch)) ? HEINSEN_OK : HEINSEN_ERR_HIP;
}

hipError_t norm_forward_launch(const NormCall &c, void *) { return norm_launch(c); }

} // namespace

int compute_units()
{
    constexpr int kMaxDevices = 64;
    static int units[kMaxDevices] = {}; // written under g_mutex
    int dev = 0, count = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return 256;
    if (units[dev] == 0) units[dev] = hipDeviceGetAttribute(&count, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && count > 0 ? count : 256;
    return units[dev];
}

int release_workspaces()
{
    std::lock_guard<std::mutex> lock(g_mutex);
    int status = HEINSEN_OK;
    for (auto &kv : g_workspaces) {
        if (hipSetDevice(kv.first.first) != hipSuccess) {
            status = HEINSEN_ERR_HIP;
            continue;
        }
        (void)hipDeviceSynchronize();
        if (kv.second.memory) (void)hipFree(kv.second.memory);
        for (void *old : kv.second.retired) (void)hipFree(old);
    }
    g_workspaces.clear();
    return status;
}

} // namespace hs

extern "C" {

int heinsen_linear_attention(const void *q, const void *k, const void *v, const void *log_a, const void *s0, void *out, void *sn,
                             const void *starts, int64_t B, int64_t n, int64_t H, int64_t Hk, int64_t K, int64_t V, int64_t q_stride,
                             int64_t k_stride, int64_t v_stride, float scale, uint32_t flags, void *stream)
{
    hs::AttentionCall c = {};
    const int st = hs::make_attention(q, k, v, log_a, s0, starts, B, n, H, Hk, K, V, q_stride, k_stride, v_stride, scale, flags, stream, c);
    if (st != HEINSEN_OK) return st;
    if (!out || !hs::aligned({out}, c.bf16 ? 2 : 4) || !hs::aligned({sn}, 4)) return HEINSEN_ERR_INVALID_ARG;
    c.out = out;
    c.sn = static_cast<float *>(sn);
    return hs::run(c, hs::attention_scratch(c), hs::attention_launch);
}

int heinsen_linear_attention_backward(const void *q, const void *k, const void *v, const void *log_a, const void *s0, const void *grad_out,
                                      const void *grad_sn, void *grad_q, void *grad_k, void *grad_v, void *grad_log_a, void *grad_s0,
                                      const void *starts, int64_t B, int64_t n, int64_t H, int64_t Hk, int64_t K, int64_t V,
                                      int64_t q_stride, int64_t k_stride, int64_t v_stride, float scale, uint32_t flags, void *stream)
{
    hs::AttentionCall c = {};
    const int st = hs::make_attention(q, k, v, log_a, s0, starts, B, n, H, Hk, K, V, q_stride, k_stride, v_stride, scale, flags, stream, c);
    if (st != HEINSEN_OK) return st;
    if (!grad_out || !grad_q || !grad_k || !grad_v || (grad_log_a && !log_a)) return HEINSEN_ERR_INVALID_ARG;
    if (!hs::aligned({grad_out, grad_q, grad_k, grad_v, grad_log_a}, c.bf16 ? 2 : 4) || !hs::aligned({grad_sn, grad_s0}, 4))
        return HEINSEN_ERR_INVALID_ARG;
    if (c.share > 1 && H * K > ((int64_t)1 << 23)) return HEINSEN_ERR_UNSUPPORTED; // rows of the heads' own gradients, as above
    c.grad_out = grad_out;
    c.grad_sn = static_cast<const float *>(grad_sn);
    c.grad_q = grad_q, c.grad_k = grad_k, c.grad_v = grad_v, c.grad_log_a = grad_log_a;
    c.grad_s0 = static_cast<float *>(grad_s0);
    return hs::run(c, hs::attention_backward_scratch(c), hs::attention_backward_launch);
}

int heinsen_block_norm(const void *u, const void *gate, const void *residual, const void *scale, const void *w_post, const void *w_pre,
                       void *h, void *y, int64_t rows, int64_t D, int64_t u_stride, int64_t gate_stride, float eps, uint32_t flags,
                       void *stream)
{
    hs::NormCall c = {};
    const int st = hs::make_norm(u, gate, residual, scale, w_post, w_pre, rows, D, u_stride, gate_stride, eps, flags, stream, c);
    if (st != HEINSEN_OK) return st;
    if ((!h && !y) || (y && !w_pre) || !hs::aligned({h, y}, c.bf16 ? 2 : 4)) return HEINSEN_ERR_INVALID_ARG;
    c.h = h;
    c.y = y;
    return hs::run(c, 0, hs::norm_forward_launch);
}

int heinsen_block_norm_backward(const void *u, const void *gate, const void *residual, const void *scale, const void *w_post,
                                const void *w_pre, const void *grad_h, const void *grad_y, void *grad_u, void *grad_gate,
                                void *grad_residual, void *grad_scale, void *grad_w_post, void *grad_w_pre, int64_t rows, int64_t D,
                                int64_t u_stride, int64_t gate_stride, float eps, uint32_t flags, void *stream)
{
    hs::NormCall c = {};
    const int st = hs::make_norm(u, gate, residual, scale, w_post, w_pre, rows, D, u_stride, gate_stride, eps, flags, stream, c);
    if (st != HEINSEN_OK) return st;
    if ((!grad_h && !grad_y) || (grad_y && !w_pre) || !grad_u) return HEINSEN_ERR_INVALID_ARG;
    if ((grad_gate && !gate) || (grad_residual && !residual) || (grad_scale && !scale) || (grad_w_post && !w_post) || (grad_w_pre && !w_pre))
        return HEINSEN_ERR_INVALID_ARG;
    if (!hs::aligned({grad_h, grad_y, grad_u, grad_gate, grad_residual}, c.bf16 ? 2 : 4) || !hs::aligned({grad_scale, grad_w_post, grad_w_pre}, 4))
        return HEINSEN_ERR_INVALID_ARG;
    c.grad_h = grad_h, c.grad_y = grad_y;
    c.grad_u = grad_u, c.grad_gate = grad_gate, c.grad_residual = grad_residual;
    c.grad_scale = static_cast<float *>(grad_scale);
    c.grad_w_post = static_cast<float *>(grad_w_post);
    c.grad_w_pre = static_cast<float *>(grad_w_pre);
    return hs::run(c, hs::norm_backward_scratch(c), hs::norm_backward_launch);
}

} // extern "C"
