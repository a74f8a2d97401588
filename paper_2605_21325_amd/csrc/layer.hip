// C-ABI of the layer's other operators (see include/triinv.h): arguments checked on the host, then one of the launchers of layer.hpp.
// No allocation, no synchronisation.
#include "layer.hpp"

namespace {

using namespace triinv;

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb)
{
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a && b && na && nb && a0 < b0 + nb && b0 < a0 + na;
}
int finish(int rc) { return rc == LAUNCHED ? TRIINV_OK : rc == NOT_BUILT ? TRIINV_ERR_UNSUPPORTED : TRIINV_ERR_LAUNCH; }
bool any_dtype(int d) { return d == TRIINV_F32 || d == TRIINV_F16 || d == TRIINV_BF16; }

struct Span {
    const void* p;
    uint64_t bytes;
};
// Whether a result overlaps one of the inputs or another result.
template <size_t NI, size_t NO> bool aliased(const Span (&in)[NI], const Span (&out)[NO])
{
    for (size_t i = 0; i < NO; ++i) {
        for (const Span& x : in)
            if (overlap(x.p, x.bytes, out[i].p, out[i].bytes)) return true;
        for (size_t j = 0; j < i; ++j)
            if (overlap(out[j].p, out[j].bytes, out[i].p, out[i].bytes)) return true;
    }
    return false;
}

// Workgroups of 64 columns.
int64_t attn_groups(int n_seq, int H, int d_v) { return (int64_t)n_seq * H * ((d_v + 63) / 64); }

// Segments of a sequence, so that its heads and groups of 64 columns fill the 256 compute units.  With W a segment's state costs as much as its outputs: it pays where
// there are four of them at least (8192 tokens in chunks of 64, d_k = d_v = 128, in us, segments in brackets: 8 heads 376 [1], 110 [16]; 16 heads 371 [1], 135 [8]; 32
// heads 382 [1], 232 [4], 253 [8]; 48 heads 407 [1], 418 [2], 387 [5]; 64 heads 384 [1], 452 [4]; 96 heads 417 [1], 686 [4]).  Without W the states are half the
// work, and twice the segments: 16 heads 328 [1], 88 [16]; 32 heads 327 [1], 150 [8]; 64 heads 337 [1], 257 [4]; 80 heads 341 [1], 336 [3]; 96 heads 348 [1], 446 [3].
// Four chunks a segment at least, and four segments: with two of them W's states cost what the outputs save.  More than sixteen segments only of eight chunks or more,
// for the join takes them one after the other.  8 heads of 128, chunks of 64, W, one segment / segments of four chunks / of eight: 12 chunks 38 / 41 / 38, 16 50 / 43 / 60, 24 73 /
// 48 / 63, 32 95 / 53 / 65, 64 185 / 73 / 74, of 2 heads 128 363 / 101 / 89, 256 720 / 168 / 123; without W 16 46 / 31 / 46, 32 87 / 34 / 48, 128 333 / 62 / 54, of 2 heads 330 / 40 / 51.
int attn_segments(int n_seq, int64_t n_chunk, int H, int d_v, bool has_w)
{
    const int64_t units = attn_groups(n_seq, H, d_v), by_units = (has_w ? 256 : 512) / units, chunks = n_chunk / n_seq;
    if (by_units < 4 || chunks < 16) return 1;
    const int64_t by_chunks = chunks < 64 ? chunks / 4 : chunks < 128 ? 16 : chunks / 8;
    return (int)(by_units < by_chunks ? by_units : by_chunks);
}
int64_t attn_workspace(int n_seq, int64_t n_chunk, int H, int d_k, int d_v, bool has_w)
{
    const int64_t n_seg = attn_segments(n_seq, n_chunk, H, d_v, has_w);
    if (n_seg == 1) return 0;
    return 4 * n_seq * H * (n_seg * d_k * d_v + (n_seg - 1) * (has_w ? (int64_t)d_k * d_k : 1));  // (a state more: the one before the first token, which final_state may lie upon)
}

// Sizes of the chunk attention, and the part of them that a workspace depends on.
int attn_states_shape(int n_seq, int64_t n_chunk, int H, int d_k, int d_v)
{
    if (n_seq <= 0 || H <= 0 || n_chunk < 0) return TRIINV_ERR_BAD_SHAPE;
    if (d_k <= 0 || d_k % 32 || d_k > 128 || d_v <= 0 || d_v % 8 || d_v > 512) return TRIINV_ERR_BAD_SHAPE;
    if (n_chunk > 0x7fffffffLL / H || (int64_t)n_seq > 0x7fffffffLL / ((int64_t)H * 16)) return TRIINV_ERR_BAD_SHAPE;
    return TRIINV_OK;
}
bool attn_C(int C) { return C == 16 || C == 32 || C == 64 || C == 128; }
int attn_shape(int n_seq, int64_t n_token, int64_t n_chunk, int H, int H_k, int d_k, int d_v, int C)
{
    if (!attn_C(C)) return TRIINV_ERR_BAD_C;
    if (H_k <= 0 || H % H_k || n_token < 0) return TRIINV_ERR_BAD_SHAPE;
    if (const int rc = attn_states_shape(n_seq, n_chunk, H, d_k, d_v)) return rc;
    if ((int64_t)H * (d_k > d_v ? d_k : d_v) * C * 2 >= (1LL << 31)) return TRIINV_ERR_UNSUPPORTED;
    if (attn_groups(n_seq, H, d_v) >= (1LL << 23)) return TRIINV_ERR_UNSUPPORTED;  // (512 threads each: a grid has fewer than 2^32)
    return TRIINV_OK;
}

int attn_common(const void* Q, const void* K, const void* U, const void* W, const float* g, const float* state, void* O, float* final_state,
                void* workspace, int64_t workspace_bytes, const int64_t* cu_seqlens, const int64_t* cu_chunks, int n_seq, int64_t Tlen,
                int64_t n_token, int64_t n_chunk, int H, int H_k, int d_k, int d_v, int C, int dtype, float scale, void* hip_stream)
{
    if (dtype == TRIINV_F32) return TRIINV_ERR_UNSUPPORTED;
    const int64_t need = attn_workspace(n_seq, n_chunk, H, d_k, d_v, W != nullptr);
    if (n_token > 0 && (!Q || !K || !U || !O)) return TRIINV_ERR_NULL;
    if (need > 0 && !workspace) return TRIINV_ERR_NULL;
    if (workspace_bytes < need) return TRIINV_ERR_BAD_SHAPE;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(U, 16) || !aligned(W, 16) || !aligned(O, 16) || !aligned(g, 4) || !aligned(state, 16) ||
        !aligned(final_state, 16) || !aligned(workspace, 16) || !aligned(cu_seqlens, 8) || !aligned(cu_chunks, 8))
        return TRIINV_ERR_ALIGN;
    const uint64_t qk = (uint64_t)n_token * H_k * d_k * 2, v = (uint64_t)n_token * H * d_v * 2, w = (uint64_t)n_token * H * d_k * 2, st = (uint64_t)n_seq * H * d_k * d_v * 4,
                   cu = (uint64_t)(n_seq + 1) * 8;
    const Span in[] = {{Q, qk}, {K, qk}, {U, v}, {W, w}, {g, (uint64_t)n_token * H * 4}, {state == final_state ? nullptr : state, st}, {cu_seqlens, cu}, {cu_chunks, cu}};
    const Span out[] = {{O, v}, {final_state, st}, {need ? workspace : nullptr, (uint64_t)need}};
    if (aliased(in, out)) return TRIINV_ERR_ALIAS;
    if (state && state == final_state && (overlap(state, st, O, v) || overlap(state, st, workspace, need))) return TRIINV_ERR_ALIAS;
    const AttnCall a{Q, K, U, W, g, state, O, final_state, static_cast<char*>(workspace), cu_seqlens, cu_chunks, Tlen, n_seq, n_chunk, H, H_k, d_k, d_v, C,
                     attn_segments(n_seq, n_chunk, H, d_v, W != nullptr), scale, static_cast<hipStream_t>(hip_stream)};
    return finish(dtype == TRIINV_F16 ? launch_chunk_attn_f16(a) : launch_chunk_attn_bf16(a));
}

// States before and gradients behind every 64 tokens or chunk, and the values where they are not U.
int64_t attn_bwd_workspace(int64_t n_token, int64_t n_chunk, int H, int d_k, int d_v, int C, bool has_w)
{
    return 4 * H * (2 * n_chunk * (C > 64 ? 2 : 1) * d_k * d_v + (has_w ? n_token * d_v : 0));
}

int attn_bwd_common(const void* Q, const void* K, const void* U, const void* W, const float* g, const float* state, const void* dO, const float* dstate, void* dQ,
                    void* dK, void* dU, void* dW, float* dg, float* dstate0, void* workspace, int64_t workspace_bytes, const int64_t* cu_seqlens,
                    const int64_t* cu_chunks, int n_seq, int64_t Tlen, int64_t n_token, int64_t n_chunk, int H, int H_k, int d_k, int d_v, int C, int dtype, float scale,
                    void* hip_stream)
{
    if (dtype == TRIINV_F32) return TRIINV_ERR_UNSUPPORTED;
    if ((int64_t)H * d_v * C * 4 >= (1LL << 31)) return TRIINV_ERR_UNSUPPORTED;  // (values are read back in fp32)
    // two walks, then 512 threads (256 each where there are two) a step and key head
    if (attn_groups(n_seq, H, d_v) >= (1LL << 22) || n_chunk * (C > 64 ? 2 : 1) * H_k >= (1LL << 23)) return TRIINV_ERR_UNSUPPORTED;
    const int64_t need = attn_bwd_workspace(n_token, n_chunk, H, d_k, d_v, C, W != nullptr);
    if (n_token > 0 && (!Q || !K || !U || !dO || !dQ || !dK || !dU || !workspace || (W != nullptr) != (dW != nullptr))) return TRIINV_ERR_NULL;
    if (dg && !g) return TRIINV_ERR_NULL;
    if (workspace_bytes < need) return TRIINV_ERR_BAD_SHAPE;
    for (const void* p : {Q, K, U, W, dO, (const void*)state, (const void*)dstate, (const void*)dQ, (const void*)dK, (const void*)dU, (const void*)dW, (const void*)dstate0, (const void*)workspace})
        if (!aligned(p, 16)) return TRIINV_ERR_ALIGN;
    if (!aligned(g, 4) || !aligned(dg, 4) || !aligned(cu_seqlens, 8) || !aligned(cu_chunks, 8)) return TRIINV_ERR_ALIGN;
    const uint64_t qk = (uint64_t)n_token * H_k * d_k * 2, v = (uint64_t)n_token * H * d_v * 2, w = (uint64_t)n_token * H * d_k * 2, st = (uint64_t)n_seq * H * d_k * d_v * 4,
                   gs = (uint64_t)n_token * H * 4, cu = (uint64_t)(n_seq + 1) * 8;
    const Span in[] = {{Q, qk}, {K, qk}, {U, v}, {W, w}, {dO, v}, {g, gs}, {state, st}, {dstate == dstate0 ? nullptr : dstate, st}, {cu_seqlens, cu}, {cu_chunks, cu}};
    const Span out[] = {{dQ, qk}, {dK, qk}, {dU, v}, {dW, w}, {dg, gs}, {dstate0, st}, {workspace, (uint64_t)need}};
    if (aliased(in, out)) return TRIINV_ERR_ALIAS;
    const AttnBwdCall a{Q, K, U, W, dO, g, state, dstate, dQ, dK, dU, dW, dg, dstate0, static_cast<char*>(workspace), cu_seqlens, cu_chunks, Tlen, n_seq, n_chunk, H, H_k,
                        d_k, d_v, C, scale, static_cast<hipStream_t>(hip_stream)};
    return finish(dtype == TRIINV_F16 ? launch_chunk_attn_bwd_f16(a) : launch_chunk_attn_bwd_bf16(a));
}

// Totals of packed sequences against each other.
bool packed_totals_ok(int n_seq, int64_t n_token, int64_t n_chunk, int C)
{
    return n_token >= 0 && n_chunk >= 0 && n_chunk <= n_token && n_chunk * C >= n_token && n_chunk <= (n_token + C - 1) / C + n_seq;
}

}  // namespace

extern "C" {

int gdn_chunk_attn_workspace(int n_seq, int64_t total_chunks, int H, int d_k, int d_v, int has_w, int64_t* bytes)
{
    if (!bytes) return TRIINV_ERR_NULL;
    if (const int rc = attn_states_shape(n_seq, total_chunks, H, d_k, d_v)) return rc;
    *bytes = attn_workspace(n_seq, total_chunks, H, d_k, d_v, has_w != 0);
    return TRIINV_OK;
}

int gdn_chunk_attn(const void* Q, const void* K, const void* U, const void* W, const float* g, const float* state, void* O, float* final_state,
                   void* workspace, int64_t workspace_bytes, int B, int64_t Tlen, int H, int H_k, int d_k, int d_v, int C, int dtype, float scale,
                   void* hip_stream)
{
    if (!any_dtype(dtype)) return TRIINV_ERR_BAD_DTYPE;
    if (B <= 0 || Tlen < 0 || Tlen > 0x7fffffffLL) return TRIINV_ERR_BAD_SHAPE;
    const int64_t n_chunk = C > 0 ? (int64_t)B * ((Tlen + C - 1) / C) : 0;
    const int rc = attn_shape(B, (int64_t)B * Tlen, n_chunk, H, H_k, d_k, d_v, C);
    if (rc) return rc;
    return attn_common(Q, K, U, W, g, state, O, final_state, workspace, workspace_bytes, nullptr, nullptr, B, Tlen, (int64_t)B * Tlen, n_chunk, H, H_k, d_k, d_v,
                       C, dtype, scale, hip_stream);
}

int gdn_chunk_attn_varlen(const void* Q, const void* K, const void* U, const void* W, const float* g, const float* state, void* O, float* final_state,
                          void* workspace, int64_t workspace_bytes, const int64_t* cu_seqlens, const int64_t* cu_chunks, int n_seq, int64_t total_tokens,
                          int64_t total_chunks, int H, int H_k, int d_k, int d_v, int C, int dtype, float scale, void* hip_stream)
{
    if (!any_dtype(dtype)) return TRIINV_ERR_BAD_DTYPE;
    const int rc = attn_shape(n_seq, total_tokens, total_chunks, H, H_k, d_k, d_v, C);
    if (rc) return rc;
    if (!packed_totals_ok(n_seq, total_tokens, total_chunks, C)) return TRIINV_ERR_BAD_SHAPE;
    if (!cu_seqlens || !cu_chunks) return TRIINV_ERR_NULL;
    return attn_common(Q, K, U, W, g, state, O, final_state, workspace, workspace_bytes, cu_seqlens, cu_chunks, n_seq, 0, total_tokens, total_chunks, H, H_k, d_k,
                       d_v, C, dtype, scale, hip_stream);
}

int gdn_chunk_attn_bwd_workspace(int64_t total_tokens, int64_t total_chunks, int H, int d_k, int d_v, int C, int has_w, int64_t* bytes)
{
    if (!bytes) return TRIINV_ERR_NULL;
    if (!attn_C(C)) return TRIINV_ERR_BAD_C;
    if (const int rc = attn_states_shape(1, total_chunks, H, d_k, d_v)) return rc;
    if (total_tokens < 0 || total_tokens > total_chunks * C) return TRIINV_ERR_BAD_SHAPE;
    *bytes = attn_bwd_workspace(total_tokens, total_chunks, H, d_k, d_v, C, has_w != 0);
    return TRIINV_OK;
}

int gdn_chunk_attn_bwd(const void* Q, const void* K, const void* U, const void* W, const float* g, const float* state, const void* dO, const float* dstate, void* dQ,
                       void* dK, void* dU, void* dW, float* dg, float* dstate0, void* workspace, int64_t workspace_bytes, int B, int64_t Tlen, int H, int H_k, int d_k,
                       int d_v, int C, int dtype, float scale, void* hip_stream)
{
    if (!any_dtype(dtype)) return TRIINV_ERR_BAD_DTYPE;
    if (B <= 0 || Tlen < 0 || Tlen > 0x7fffffffLL) return TRIINV_ERR_BAD_SHAPE;
    const int64_t n_chunk = C > 0 ? (int64_t)B * ((Tlen + C - 1) / C) : 0;
    const int rc = attn_shape(B, (int64_t)B * Tlen, n_chunk, H, H_k, d_k, d_v, C);
    if (rc) return rc;
    return attn_bwd_common(Q, K, U, W, g, state, dO, dstate, dQ, dK, dU, dW, dg, dstate0, workspace, workspace_bytes, nullptr, nullptr, B, Tlen, (int64_t)B * Tlen, n_chunk,
                           H, H_k, d_k, d_v, C, dtype, scale, hip_stream);
}

int gdn_chunk_attn_bwd_varlen(const void* Q, const void* K, const void* U, const void* W, const float* g, const float* state, const void* dO, const float* dstate,
                              void* dQ, void* dK, void* dU, void* dW, float* dg, float* dstate0, void* workspace, int64_t workspace_bytes, const int64_t* cu_seqlens,
                              const int64_t* cu_chunks, int n_seq, int64_t total_tokens, int64_t total_chunks, int H, int H_k, int d_k, int d_v, int C, int dtype,
                              float scale, void* hip_stream)
{
    if (!any_dtype(dtype)) return TRIINV_ERR_BAD_DTYPE;
    const int rc = attn_shape(n_seq, total_tokens, total_chunks, H, H_k, d_k, d_v, C);
    if (rc) return rc;
    if (!packed_totals_ok(n_seq, total_tokens, total_chunks, C)) return TRIINV_ERR_BAD_SHAPE;
    if (!cu_seqlens || !cu_chunks) return TRIINV_ERR_NULL;
    return attn_bwd_common(Q, K, U, W, g, state, dO, dstate, dQ, dK, dU, dW, dg, dstate0, workspace, workspace_bytes, cu_seqlens, cu_chunks, n_seq, 0, total_tokens,
                           total_chunks, H, H_k, d_k, d_v, C, dtype, scale, hip_stream);
}

int gdn_step(const void* q, const void* k, const void* v, const float* g, const float* beta, float* state, const int32_t* slots, void* o, int B,
             int64_t n_slot, int H, int H_k, int d_k, int d_v, int dtype, float scale, void* hip_stream)
{
    if (!any_dtype(dtype)) return TRIINV_ERR_BAD_DTYPE;
    if (B < 0 || n_slot < 0 || n_slot > 0x7fffffffLL || H <= 0 || H_k <= 0 || H % H_k || d_k <= 0 || d_k > 256 || d_v <= 0 || d_v % 4 || d_v > 512) return TRIINV_ERR_BAD_SHAPE;
    if (!slots && n_slot < B) return TRIINV_ERR_BAD_SHAPE;
    if ((int64_t)B > 0x7fffffffLL / ((int64_t)H * 16)) return TRIINV_ERR_BAD_SHAPE;
    if (B == 0) return TRIINV_OK;
    if (!q || !k || !v || !o || (n_slot > 0 && !state)) return TRIINV_ERR_NULL;
    if (!aligned(q, 4) || !aligned(k, 4) || !aligned(v, 16) || !aligned(o, 16) || !aligned(state, 16) || !aligned(g, 4) || !aligned(beta, 4) || !aligned(slots, 4))
        return TRIINV_ERR_ALIGN;
    const uint64_t e = dtype == TRIINV_F32 ? 4 : 2, qk = (uint64_t)B * H_k * d_k * e, vo = (uint64_t)B * H * d_v * e, bh = (uint64_t)B * H * 4;
    const Span in[] = {{q, qk}, {k, qk}, {v, vo}, {g, bh}, {beta, bh}, {slots, (uint64_t)B * 4}};
    const Span out[] = {{o, vo}, {state, (uint64_t)n_slot * H * d_k * d_v * 4}};
    if (aliased(in, out)) return TRIINV_ERR_ALIAS;
    return finish(launch_step(StepCall{q, k, v, g, beta, state, slots, o, n_slot, B, H, H_k, d_k, d_v, dtype, scale, static_cast<hipStream_t>(hip_stream)}));
}

int add_rms_norm(const void* x, const void* residual, const void* weight, void* y, float* scales, void* sum, int64_t N, int D, int group, int dtype,
                 float eps, void* hip_stream)
{
    if (!any_dtype(dtype)) return TRIINV_ERR_BAD_DTYPE;
    if (N < 0 || N > 0x7fffffffLL || D <= 0 || D % 8 || D > 16384 || (group != -1 && group != 0 && group != 128) || (group == 128 && D % 128)) return TRIINV_ERR_BAD_SHAPE;
    if (N == 0) return TRIINV_OK;
    if (!x || !weight || !y || (group >= 0 && !scales) || (residual != nullptr) != (sum != nullptr)) return TRIINV_ERR_NULL;
    if (!aligned(x, 16) || !aligned(residual, 16) || !aligned(weight, 16) || !aligned(y, 16) || !aligned(sum, 16) || !aligned(scales, 4)) return TRIINV_ERR_ALIGN;
    const uint64_t e = dtype == TRIINV_F32 ? 4 : 2, n = (uint64_t)N * D;
    const Span in[] = {{x == sum ? nullptr : x, n * e}, {residual == sum ? nullptr : residual, n * e}, {weight, (uint64_t)D * e}};
    const Span out[] = {{y, n * (group < 0 ? e : 1)}, {sum, n * e}, {group >= 0 ? scales : nullptr, (uint64_t)N * (group == 128 ? D / 128 : 1) * 4}};
    if (aliased(in, out)) return TRIINV_ERR_ALIAS;
    return finish(launch_norm(NormCall{x, residual, weight, y, sum, scales, N, D, group, dtype, eps, static_cast<hipStream_t>(hip_stream)}));
}

int add_rms_norm_bwd(const void* dy, const void* s, const void* weight, const void* dsum, void* dx, float* dweight, void* workspace, int64_t workspace_bytes,
                     int64_t N, int D, int dtype, float eps, void* hip_stream)
{
    if (!any_dtype(dtype)) return TRIINV_ERR_BAD_DTYPE;
    if (N < 0 || N > 0x7fffffffLL || D <= 0 || D % 8 || D > 16384) return TRIINV_ERR_BAD_SHAPE;
    const int groups = N < 512 ? (int)N : 512;
    const int64_t need = (int64_t)4 * D * groups;
    if (!dweight || !weight || (N > 0 && (!dy || !s || !dx || !workspace))) return TRIINV_ERR_NULL;
    if (workspace_bytes < need) return TRIINV_ERR_BAD_SHAPE;
    if (!aligned(dy, 16) || !aligned(s, 16) || !aligned(weight, 16) || !aligned(dsum, 16) || !aligned(dx, 16) || !aligned(dweight, 16) || !aligned(workspace, 16))
        return TRIINV_ERR_ALIGN;
    const uint64_t e = dtype == TRIINV_F32 ? 4 : 2, n = (uint64_t)N * D * e;
    const Span in[] = {{dy, n}, {s, n}, {weight, (uint64_t)D * e}, {dsum, n}};
    const Span out[] = {{dx, n}, {dweight, (uint64_t)D * 4}, {workspace, (uint64_t)need}};
    if (aliased(in, out)) return TRIINV_ERR_ALIAS;
    return finish(launch_norm_bwd(NormBwdCall{dy, s, weight, dsum, dx, dweight, static_cast<float*>(workspace), N, D, dtype, groups, eps, static_cast<hipStream_t>(hip_stream)}));
}

}  // extern "C"
