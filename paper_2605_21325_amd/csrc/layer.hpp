// Host-side launchers of the layer's other operators (chunk attention, single-token step, norm), each in a translation unit of its own.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "dispatch.hpp"

namespace triinv {

// Workgroups 0 to n - 1 as blockIdx.y gridDim.x + blockIdx.x, and some more behind them: a dimension of a grid has fewer than 2^32 threads.
inline dim3 long_grid(int64_t n)
{
    constexpr int64_t MOST = 1 << 21;  // of up to 1024 threads
    return n <= MOST ? dim3((unsigned)n) : dim3((unsigned)MOST, (unsigned)((n + MOST - 1) / MOST));
}

// Chunk attention: arguments checked by the entry points.
struct AttnCall {
    const void *Q, *K, *U, *W;
    const float *g, *state;
    void* O;
    float* final_state;
    char* workspace;
    const int64_t *cu_seqlens, *cu_chunks;  // device, or null: n_seq sequences of Tlen tokens
    int64_t Tlen;
    int n_seq;
    int64_t n_chunk;  // of all sequences
    int H, H_k, d_k, d_v, C, n_seg;
    float scale;
    hipStream_t stream;
};
int launch_chunk_attn_f16(const AttnCall& a);
int launch_chunk_attn_bf16(const AttnCall& a);

struct AttnBwdCall {
    const void *Q, *K, *U, *W, *dO;
    const float *g, *state, *dstate;
    void *dQ, *dK, *dU, *dW;
    float *dg, *dstate0;
    char* workspace;
    const int64_t *cu_seqlens, *cu_chunks;
    int64_t Tlen;
    int n_seq;
    int64_t n_chunk;
    int H, H_k, d_k, d_v, C;
    float scale;
    hipStream_t stream;
};
int launch_chunk_attn_bwd_f16(const AttnBwdCall& a);
int launch_chunk_attn_bwd_bf16(const AttnBwdCall& a);

struct StepCall {
    const void *q, *k, *v;
    const float *g, *beta;
    float* state;
    const int32_t* slots;
    void* o;
    int64_t n_slot;
    int B, H, H_k, d_k, d_v, dtype;
    float scale;
    hipStream_t stream;
};
int launch_step(const StepCall& a);

struct NormCall {
    const void *x, *residual, *weight;
    void *y, *sum;
    float* scales;
    int64_t N;
    int D, group, dtype;  // group < 0: y has x's type, 0: a scale a row, else columns a scale
    float eps;
    hipStream_t stream;
};
int launch_norm(const NormCall& a);

struct NormBwdCall {
    const void *dy, *x, *weight, *dsum;
    void* dx;
    float *dweight, *partial;
    int64_t N;
    int D, dtype, groups;  // workgroups that keep a partial sum each
    float eps;
    hipStream_t stream;
};
int launch_norm_bwd(const NormBwdCall& a);

// Norms of queries and keys for each head with the rotation: tokens' strides in elements.
struct HeadsCall {
    const void *q, *k, *q_weight, *k_weight, *positions;
    const float* inv_freq;
    void *q_out, *k_out;
    int64_t N, q_stride, k_stride, q_out_stride, k_out_stride;
    int H, H_k, d, rot, dtype;  // rot = 0: no rotation
    bool unit, interleaved, pos64;
    float eps;
    hipStream_t stream;
};
int launch_heads(const HeadsCall& a);

struct HeadsBwdCall {
    const void *dq_out, *dk_out, *q, *k, *q_weight, *k_weight, *positions;
    const float* inv_freq;
    void *dq, *dk;
    float *dq_weight, *dk_weight, *partial;  // partial: [groups_q + groups_k][d], or null where neither weight's gradient is asked for
    int64_t N, dq_out_stride, dk_out_stride, q_stride, k_stride, dq_stride, dk_stride;
    int H, H_k, d, rot, dtype, groups_q, groups_k;
    bool unit, interleaved, pos64;
    float eps;
    hipStream_t stream;
};
int heads_bwd_groups(int64_t N, int H, int heads);  // workgroups for H of the heads
int launch_heads_bwd(const HeadsBwdCall& a);

// The gated recurrence: tokens' strides in elements.
struct ScanCall {
    const void *x, *g;  // x null: not needed (gradient without mix)
    const float* state;
    const void *h, *dh;  // of the gradient
    const float* dstate;
    void *out, *dg;  // out: h, or the gradient of x
    float* last;     // the final state, or the gradient of the initial one
    char* workspace;
    const int64_t* cu_seqlens;  // device, or null: n_seq sequences of Tlen tokens
    int64_t Tlen, N, x_stride, g_stride, h_stride, dh_stride, out_stride, dg_stride;
    int n_seq, D, dtype, g_dtype;
    bool logit, mix;
    hipStream_t stream;
};
int64_t scan_workspace(int64_t N, int n_seq, int D);
int launch_scan(const ScanCall& a);
int launch_scan_bwd(const ScanCall& a);

struct ScanStepCall {
    const void *x, *g;
    float* state;
    const int32_t* slots;
    void* h;
    int64_t n_slot, x_stride, g_stride, h_stride;
    int B, D, dtype, g_dtype;
    bool logit, mix;
    hipStream_t stream;
};
int launch_scan_step(const ScanStepCall& a);

}  // namespace triinv
