// What the operators for language models share on the host side (not part of the public ABI).
#pragma once
#include "heinsen_internal.hpp"

namespace hs {

// Validated description of one linear attention call.
struct AttentionCall {
    const void *q, *k, *v, *log_a; // float32 or bfloat16
    const float *s0;               // [B, H, K, V] or null (zeros)
    const int64_t *starts;         // device [B + 1], or null: B sequences of n tokens
    int64_t n;                     // tokens of a sequence; with starts, of the longest one
    int64_t q_stride, k_stride, v_stride; // elements from one token to the next
    int B, H, share, K, V;         // share: heads of v and of the state to one head of q and k
    bool bf16, per_head;
    float scale;
    hipStream_t stream;
    // forward
    void *out;
    float *sn;                     // or null
    // gradients
    const void *grad_out;          // or null (zeros)
    const float *grad_sn;          // or null (zeros)
    void *grad_q, *grad_k, *grad_v, *grad_log_a; // grad_log_a may be null
    float *grad_s0;                // or null
};

// Sequences of few heads are cut into segments of a whole number of 64 tokens that run side by side.
struct Segments {
    int64_t tokens;
    int count;
};
Segments attention_segments(const AttentionCall &c, bool back);
size_t segment_scratch(const AttentionCall &c, const Segments &s);
hipError_t attention_segment_states(const AttentionCall &c, const Segments &s, void *states, void *gradients);
hipError_t attention_chunk_states(const AttentionCall &c, const Segments &s, float *segment_state, void *states, uint32_t *fine, int chunks);
constexpr int kFewTokens = 4; // sequences of up to so many go token by token
int attention_chunk_tokens(bool bf16); // of the stored chunk states

size_t attention_scratch(const AttentionCall &c);                    // bytes
hipError_t attention_launch(const AttentionCall &c, void *scratch);
size_t attention_backward_scratch(const AttentionCall &c);
hipError_t attention_backward_launch(const AttentionCall &c, void *scratch);

struct NormCall {
    const void *u, *gate, *residual;            // gate and residual may be null
    const float *scale, *w_post, *w_pre;        // each may be null
    void *h, *y;                                // forward; each may be null
    const void *grad_h, *grad_y;                // backward; each may be null
    void *grad_u, *grad_gate, *grad_residual;   // grad_gate and grad_residual may be null
    float *grad_scale, *grad_w_post, *grad_w_pre;
    int64_t rows, u_stride, gate_stride;
    int D;
    float eps;
    bool bf16, sigmoid;
    hipStream_t stream;
};

hipError_t norm_launch(const NormCall &c);
size_t norm_backward_scratch(const NormCall &c);
hipError_t norm_backward_launch(const NormCall &c, void *scratch);

int compute_units(); // of the current device

// of heinsen_api.hip: notes a failed HIP call for heinsen_last_hip_error; whether `stream` is being captured
bool note_hip(hipError_t e);
bool is_capturing(hipStream_t stream);
// of operators_api.hip: frees what heinsen_release_scratch frees beside the scan's buffers; the devices are idle
int release_workspaces();

} // namespace hs
