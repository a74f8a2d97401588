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

}  // namespace triinv
