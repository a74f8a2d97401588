// C-ABI of what stands between a projection and the layer's operators (see include/triinv.h): arguments checked on the host, then one of the launchers of layer.hpp.
// No allocation, no synchronisation.
#include "entry.hpp"
#include "layer.hpp"

namespace {

using namespace triinv;

constexpr int64_t MOST_STRIDE = 1LL << 24;  // elements from token to token of a recurrence: a wavefront's rows stay below 2^31 bytes
constexpr int64_t ANY_STRIDE = 1LL << 29;   // elsewhere: N rows stay below 2^62 bytes

uint64_t size_of(int dtype) { return dtype == TRIINV_F32 ? 4 : 2; }
bool strides_ok(std::initializer_list<int64_t> strides, int64_t most)
{
    for (const int64_t s : strides)
        if (s < 0 || s > most) return false;
    return true;
}
// Tokens of a result do not lie upon each other.
bool apart(int64_t n, int64_t stride, int64_t width) { return n <= 1 || stride >= width; }
template <size_t NI, size_t NO> bool aliased(const Rows (&in)[NI], const Rows (&out)[NO])
{
    for (size_t i = 0; i < NO; ++i) {
        for (const Rows& x : in)
            if (overlap(x, out[i])) return true;
        for (size_t j = 0; j < i; ++j)
            if (overlap(out[j], out[i])) return true;
    }
    return false;
}
Rows flat(const void* p, uint64_t bytes) { return {p, 1, bytes, bytes}; }
bool same(const Rows& a, const Rows& b) { return a.p == b.p && (a.stride == b.stride || a.n <= 1); }

int heads_shape(int64_t N, int H, int H_k, int d, int rot, int dtype, uint32_t flags)
{
    if (!any_dtype(dtype)) return TRIINV_ERR_BAD_DTYPE;
    if (N < 0 || N > 0x7fffffffLL || H <= 0 || H_k < 0 || d <= 0 || d > 512 || rot < 0 || rot > d || rot % 2) return TRIINV_ERR_BAD_SHAPE;
    if (flags & ~(TRIINV_HEADS_UNIT | TRIINV_HEADS_INTERLEAVED | TRIINV_HEADS_POS64)) return TRIINV_ERR_BAD_METHOD;
    if ((int64_t)H + H_k > (1 << 20) || N * ((int64_t)H + H_k) > 0x7fffffffLL) return TRIINV_ERR_UNSUPPORTED;
    return TRIINV_OK;
}
int64_t heads_workspace(int64_t N, int H, int H_k, int d) { return ((int64_t)heads_bwd_groups(N, H, H + H_k) + heads_bwd_groups(N, H_k, H + H_k)) * d * 4; }

constexpr uint32_t SCAN_FLAGS = TRIINV_SCAN_LOGIT | TRIINV_SCAN_MIX;
int scan_types(int dtype, int g_dtype, uint32_t flags)
{
    if (!any_dtype(dtype) || (g_dtype != dtype && g_dtype != TRIINV_F32)) return TRIINV_ERR_BAD_DTYPE;
    return flags & ~SCAN_FLAGS ? TRIINV_ERR_BAD_METHOD : TRIINV_OK;
}
int scan_shape(int64_t n_token, int64_t n_seq, int D)
{
    if (n_seq <= 0 || n_seq > 0x7fffffffLL || n_token < 0 || n_token > 0x7fffffffLL || D <= 0 || D > (1 << 20)) return TRIINV_ERR_BAD_SHAPE;
    return n_seq * ((D + 63) / 64) < (1LL << 31) ? TRIINV_OK : TRIINV_ERR_UNSUPPORTED;
}

// Both directions: a.h is null in the forward one.
int scan_common(ScanCall a, int64_t workspace_bytes, bool back)
{
    const int64_t need = scan_workspace(a.N, a.n_seq, a.D);
    if (a.N > 0 && (!a.g || !a.out || (!a.x && (!back || a.mix)) || (back && (!a.h || !a.dh || !a.dg)))) return TRIINV_ERR_NULL;
    if (need > 0 && !a.workspace) return TRIINV_ERR_NULL;
    if (workspace_bytes < need || !strides_ok({a.x_stride, a.g_stride, a.h_stride, a.dh_stride, a.out_stride, a.dg_stride}, MOST_STRIDE)) return TRIINV_ERR_BAD_SHAPE;
    if (!apart(a.N, a.out_stride, a.D) || (back && !apart(a.N, a.dg_stride, a.D))) return TRIINV_ERR_BAD_SHAPE;
    const uint64_t e = size_of(a.dtype), eg = size_of(a.g_dtype), states = (uint64_t)a.n_seq * a.D * 4;
    if (!aligned(a.x, e) || !aligned(a.h, e) || !aligned(a.dh, e) || !aligned(a.out, e) || !aligned(a.g, eg) || !aligned(a.dg, eg) || !aligned(a.state, 4) || !aligned(a.dstate, 4) ||
        !aligned(a.last, 4) || !aligned(a.workspace, 16) || !aligned(a.cu_seqlens, 8))
        return TRIINV_ERR_ALIGN;
    const auto rows = [&](const void* p, int64_t stride, uint64_t size) { return Rows{p, a.N, a.D * size, stride * size}; };
    const bool upon = !back && a.state && a.state == a.last;  // the final state upon the initial one
    const Rows in[] = {rows(a.x, a.x_stride, e), rows(a.g, a.g_stride, eg), rows(a.h, a.h_stride, e), rows(a.dh, a.dh_stride, e), flat(upon ? nullptr : a.state, states), flat(a.dstate, states),
                       flat(a.cu_seqlens, (uint64_t)(a.n_seq + 1) * 8)};
    const Rows out[] = {rows(a.out, a.out_stride, e), rows(a.dg, a.dg_stride, eg), flat(a.last, states), flat(need ? a.workspace : nullptr, (uint64_t)need)};
    if (aliased(in, out)) return TRIINV_ERR_ALIAS;
    return finish(back ? launch_scan_bwd(a) : launch_scan(a));
}

}  // namespace

extern "C" {

int qk_norm_rope(const void* q, const void* k, const void* q_weight, const void* k_weight, const void* positions, const float* inv_freq, void* q_out, void* k_out, int64_t N,
                 int64_t q_stride, int64_t k_stride, int64_t q_out_stride, int64_t k_out_stride, int H, int H_k, int d, int rot, int dtype, uint32_t flags, float eps, void* hip_stream)
{
    if (const int rc = heads_shape(N, H, H_k, d, rot, dtype, flags)) return rc;
    const int64_t wq = (int64_t)H * d, wk = (int64_t)H_k * d;
    if (!strides_ok({q_stride, k_stride, q_out_stride, k_out_stride}, ANY_STRIDE) || !apart(N, q_out_stride, wq) || (H_k > 0 && !apart(N, k_out_stride, wk))) return TRIINV_ERR_BAD_SHAPE;
    if (N == 0) return TRIINV_OK;
    if (!q || !q_out || (H_k > 0 && (!k || !k_out)) || (rot > 0 && (!positions || !inv_freq))) return TRIINV_ERR_NULL;
    const uint64_t e = size_of(dtype), pos = flags & TRIINV_HEADS_POS64 ? 8 : 4;
    if (!aligned(q, e) || !aligned(k, e) || !aligned(q_weight, e) || !aligned(k_weight, e) || !aligned(q_out, e) || !aligned(k_out, e) || !aligned(inv_freq, 4) || !aligned(positions, pos))
        return TRIINV_ERR_ALIGN;
    if (H_k == 0) k = k_out = nullptr;
    const Rows rq{q, N, wq * e, q_stride * e}, rk{k, N, wk * e, k_stride * e};
    const Rows out[] = {{q_out, N, wq * e, q_out_stride * e}, {k_out, N, wk * e, k_out_stride * e}};
    const Rows rest[] = {flat(q_weight, d * e), flat(k_weight, d * e), flat(rot ? positions : nullptr, N * pos), flat(rot ? inv_freq : nullptr, rot * 2)};
    if (aliased(rest, out) || (!same(rq, out[0]) && overlap(rq, out[0])) || (!same(rk, out[1]) && overlap(rk, out[1])) || overlap(rq, out[1]) || overlap(rk, out[0])) return TRIINV_ERR_ALIAS;
    return finish(launch_heads(HeadsCall{q, k, q_weight, k_weight, positions, inv_freq, q_out, k_out, N, q_stride, k_stride, q_out_stride, k_out_stride, H, H_k, d, rot, dtype,
                                         (flags & TRIINV_HEADS_UNIT) != 0, (flags & TRIINV_HEADS_INTERLEAVED) != 0, (flags & TRIINV_HEADS_POS64) != 0, eps,
                                         static_cast<hipStream_t>(hip_stream)}));
}

int qk_norm_rope_bwd_workspace(int64_t N, int H, int H_k, int d, int64_t* bytes)
{
    if (!bytes) return TRIINV_ERR_NULL;
    if (const int rc = heads_shape(N, H, H_k, d, 0, TRIINV_F32, 0)) return rc;
    *bytes = heads_workspace(N, H, H_k, d);
    return TRIINV_OK;
}

int qk_norm_rope_bwd(const void* dq_out, const void* dk_out, const void* q, const void* k, const void* q_weight, const void* k_weight, const void* positions, const float* inv_freq,
                     void* dq, void* dk, float* dq_weight, float* dk_weight, void* workspace, int64_t workspace_bytes, int64_t N, int64_t dq_out_stride, int64_t dk_out_stride,
                     int64_t q_stride, int64_t k_stride, int64_t dq_stride, int64_t dk_stride, int H, int H_k, int d, int rot, int dtype, uint32_t flags, float eps, void* hip_stream)
{
    if (const int rc = heads_shape(N, H, H_k, d, rot, dtype, flags)) return rc;
    const int64_t wq = (int64_t)H * d, wk = (int64_t)H_k * d;
    if (!strides_ok({dq_out_stride, dk_out_stride, q_stride, k_stride, dq_stride, dk_stride}, ANY_STRIDE) || !apart(N, dq_stride, wq) || (H_k > 0 && !apart(N, dk_stride, wk))) return TRIINV_ERR_BAD_SHAPE;
    const bool weights = dq_weight || dk_weight;
    const int64_t need = weights ? heads_workspace(N, H, H_k, d) : 0;
    if (N > 0 && (!dq_out || !q || !dq || (H_k > 0 && (!dk_out || !k || !dk)) || (rot > 0 && (!positions || !inv_freq)) || (need > 0 && !workspace))) return TRIINV_ERR_NULL;
    if ((dq_weight && !q_weight) || (dk_weight && !k_weight)) return TRIINV_ERR_NULL;
    if (workspace_bytes < need) return TRIINV_ERR_BAD_SHAPE;
    const uint64_t e = size_of(dtype), pos = flags & TRIINV_HEADS_POS64 ? 8 : 4;
    for (const void* p : {dq_out, dk_out, q, k, q_weight, k_weight, (const void*)dq, (const void*)dk})
        if (!aligned(p, e)) return TRIINV_ERR_ALIGN;
    if (!aligned(inv_freq, 4) || !aligned(positions, pos) || !aligned(dq_weight, 4) || !aligned(dk_weight, 4) || !aligned(workspace, 16)) return TRIINV_ERR_ALIGN;
    if (H_k == 0) k = dk_out = dk = nullptr;
    const Rows in[] = {{q, N, wq * e, q_stride * e}, {k, N, wk * e, k_stride * e}, flat(q_weight, d * e), flat(k_weight, d * e), flat(rot ? positions : nullptr, N * pos), flat(rot ? inv_freq : nullptr, rot * 2)};
    const Rows out[] = {{dq, N, wq * e, dq_stride * e}, {dk, N, wk * e, dk_stride * e}, flat(dq_weight, d * 4), flat(dk_weight, d * 4), flat(need ? workspace : nullptr, (uint64_t)need)};
    if (aliased(in, out)) return TRIINV_ERR_ALIAS;
    const Rows up[] = {{dq_out, N, wq * e, dq_out_stride * e}, {dk_out, N, wk * e, dk_out_stride * e}};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 5; ++j)
            if (overlap(up[i], out[j]) && !(i == j && same(up[i], out[j]))) return TRIINV_ERR_ALIAS;
    return finish(launch_heads_bwd(HeadsBwdCall{dq_out, dk_out, q, k, q_weight, k_weight, positions, inv_freq, dq, dk, dq_weight, dk_weight, weights ? static_cast<float*>(workspace) : nullptr, N,
                                                dq_out_stride, dk_out_stride, q_stride, k_stride, dq_stride, dk_stride, H, H_k, d, rot, dtype, heads_bwd_groups(N, H, H + H_k), heads_bwd_groups(N, H_k, H + H_k),
                                                (flags & TRIINV_HEADS_UNIT) != 0, (flags & TRIINV_HEADS_INTERLEAVED) != 0, (flags & TRIINV_HEADS_POS64) != 0, eps,
                                                static_cast<hipStream_t>(hip_stream)}));
}

int gated_scan_workspace(int64_t total_tokens, int n_seq, int D, int64_t* bytes)
{
    if (!bytes) return TRIINV_ERR_NULL;
    if (const int rc = scan_shape(total_tokens, n_seq, D)) return rc;
    *bytes = scan_workspace(total_tokens, n_seq, D);
    return TRIINV_OK;
}

int gated_scan(const void* x, const void* g, const float* state, void* h, float* final_state, void* workspace, int64_t workspace_bytes, int B, int64_t Tlen, int D, int64_t x_stride,
               int64_t g_stride, int64_t h_stride, int dtype, int g_dtype, uint32_t flags, void* hip_stream)
{
    if (const int rc = scan_types(dtype, g_dtype, flags)) return rc;
    if (B <= 0 || Tlen < 0 || Tlen > 0x7fffffffLL) return TRIINV_ERR_BAD_SHAPE;
    if (const int rc = scan_shape(B * Tlen, B, D)) return rc;
    return scan_common(ScanCall{x, g, state, nullptr, nullptr, nullptr, h, nullptr, final_state, static_cast<char*>(workspace), nullptr, Tlen, B * Tlen, x_stride, g_stride, 0, 0, h_stride, 0, B, D,
                                dtype, g_dtype, (flags & TRIINV_SCAN_LOGIT) != 0, (flags & TRIINV_SCAN_MIX) != 0, static_cast<hipStream_t>(hip_stream)},
                       workspace_bytes, false);
}

int gated_scan_varlen(const void* x, const void* g, const float* state, void* h, float* final_state, void* workspace, int64_t workspace_bytes, const int64_t* cu_seqlens, int n_seq,
                      int64_t total_tokens, int D, int64_t x_stride, int64_t g_stride, int64_t h_stride, int dtype, int g_dtype, uint32_t flags, void* hip_stream)
{
    if (const int rc = scan_types(dtype, g_dtype, flags)) return rc;
    if (const int rc = scan_shape(total_tokens, n_seq, D)) return rc;
    if (!cu_seqlens) return TRIINV_ERR_NULL;
    return scan_common(ScanCall{x, g, state, nullptr, nullptr, nullptr, h, nullptr, final_state, static_cast<char*>(workspace), cu_seqlens, 0, total_tokens, x_stride, g_stride, 0, 0, h_stride, 0,
                                n_seq, D, dtype, g_dtype, (flags & TRIINV_SCAN_LOGIT) != 0, (flags & TRIINV_SCAN_MIX) != 0, static_cast<hipStream_t>(hip_stream)},
                       workspace_bytes, false);
}

int gated_scan_bwd(const void* x, const void* g, const void* h, const float* state, const void* dh, const float* dstate, void* dx, void* dg, float* dstate0, void* workspace,
                   int64_t workspace_bytes, int B, int64_t Tlen, int D, int64_t x_stride, int64_t g_stride, int64_t h_stride, int64_t dh_stride, int64_t dx_stride, int64_t dg_stride, int dtype,
                   int g_dtype, uint32_t flags, void* hip_stream)
{
    if (const int rc = scan_types(dtype, g_dtype, flags)) return rc;
    if (B <= 0 || Tlen < 0 || Tlen > 0x7fffffffLL) return TRIINV_ERR_BAD_SHAPE;
    if (const int rc = scan_shape(B * Tlen, B, D)) return rc;
    return scan_common(ScanCall{x, g, state, h, dh, dstate, dx, dg, dstate0, static_cast<char*>(workspace), nullptr, Tlen, B * Tlen, x_stride, g_stride, h_stride, dh_stride, dx_stride, dg_stride, B,
                                D, dtype, g_dtype, (flags & TRIINV_SCAN_LOGIT) != 0, (flags & TRIINV_SCAN_MIX) != 0, static_cast<hipStream_t>(hip_stream)},
                       workspace_bytes, true);
}

int gated_scan_bwd_varlen(const void* x, const void* g, const void* h, const float* state, const void* dh, const float* dstate, void* dx, void* dg, float* dstate0, void* workspace,
                          int64_t workspace_bytes, const int64_t* cu_seqlens, int n_seq, int64_t total_tokens, int D, int64_t x_stride, int64_t g_stride, int64_t h_stride, int64_t dh_stride,
                          int64_t dx_stride, int64_t dg_stride, int dtype, int g_dtype, uint32_t flags, void* hip_stream)
{
    if (const int rc = scan_types(dtype, g_dtype, flags)) return rc;
    if (const int rc = scan_shape(total_tokens, n_seq, D)) return rc;
    if (!cu_seqlens) return TRIINV_ERR_NULL;
    return scan_common(ScanCall{x, g, state, h, dh, dstate, dx, dg, dstate0, static_cast<char*>(workspace), cu_seqlens, 0, total_tokens, x_stride, g_stride, h_stride, dh_stride, dx_stride, dg_stride,
                                n_seq, D, dtype, g_dtype, (flags & TRIINV_SCAN_LOGIT) != 0, (flags & TRIINV_SCAN_MIX) != 0, static_cast<hipStream_t>(hip_stream)},
                       workspace_bytes, true);
}

int gated_scan_step(const void* x, const void* g, float* state, const int32_t* slots, void* h, int B, int64_t n_slot, int D, int64_t x_stride, int64_t g_stride, int64_t h_stride, int dtype,
                    int g_dtype, uint32_t flags, void* hip_stream)
{
    if (const int rc = scan_types(dtype, g_dtype, flags)) return rc;
    if (B < 0 || n_slot < 0 || n_slot > 0x7fffffffLL || D <= 0 || D > (1 << 20) || (!slots && n_slot < B)) return TRIINV_ERR_BAD_SHAPE;
    if (!strides_ok({x_stride, g_stride, h_stride}, ANY_STRIDE) || !apart(B, h_stride, D)) return TRIINV_ERR_BAD_SHAPE;
    if ((int64_t)B * ((D + 63) / 64) >= (1LL << 26)) return TRIINV_ERR_UNSUPPORTED;
    if (B == 0) return TRIINV_OK;
    if (!x || !g || !h || (n_slot > 0 && !state)) return TRIINV_ERR_NULL;
    const uint64_t e = size_of(dtype), eg = size_of(g_dtype);
    if (!aligned(x, e) || !aligned(g, eg) || !aligned(h, e) || !aligned(state, 4) || !aligned(slots, 4)) return TRIINV_ERR_ALIGN;
    const Rows in[] = {{x, B, D * e, x_stride * e}, {g, B, D * eg, g_stride * eg}, flat(slots, (uint64_t)B * 4)};
    const Rows out[] = {{h, B, D * e, h_stride * e}, flat(state, (uint64_t)n_slot * D * 4)};
    if (aliased(in, out)) return TRIINV_ERR_ALIAS;
    return finish(launch_scan_step(ScanStepCall{x, g, state, slots, h, n_slot, x_stride, g_stride, h_stride, B, D, dtype, g_dtype, (flags & TRIINV_SCAN_LOGIT) != 0,
                                                (flags & TRIINV_SCAN_MIX) != 0, static_cast<hipStream_t>(hip_stream)}));
}

}  // extern "C"
