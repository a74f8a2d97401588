// Instantiations of the chunk attention's gradient (attn_bwd.hpp) for one operand type, TRIINV_INST_OP.
#include "attn_bwd.hpp"
#include "layer.hpp"

#ifndef TRIINV_INST_OP
#error "compile with -DTRIINV_INST_OP=1|2"
#endif

namespace triinv {

namespace {

constexpr int OP = TRIINV_INST_OP;

template <int MT, int KP, bool DELTA, bool TWO> int go(const AttnBwdCall& c)
{
    const unsigned heads = (unsigned)(c.n_seq * c.H), groups = (unsigned)((c.d_v + ATTN_COLS - 1) / ATTN_COLS);
    const int64_t n_step = c.n_chunk * (c.C > 16 * MT ? 2 : 1), states = n_step * c.H * c.d_k * c.d_v;
    float* const rec = reinterpret_cast<float*>(c.workspace);
    AttnArgs f{};
    f.K = c.K, f.U = c.U, f.W = c.W, f.g = c.g, f.state = c.state, f.rec_state = rec, f.rec_value = rec + 2 * states, f.rec_dg = c.H > c.H_k ? nullptr : c.dg;
    f.map = SeqMap{c.cu_seqlens, c.cu_chunks, c.Tlen, c.n_seq};
    f.H = c.H, f.group = c.H / c.H_k, f.d_k = c.d_k, f.d_v = c.d_v, f.C = c.C, f.n_seg = 1, f.scale = c.scale;
    AttnBwdArgs a{};
    a.Q = c.Q, a.K = c.K, a.U = c.U, a.W = c.W, a.dO = c.dO, a.g = c.g, a.dstate = c.dstate;
    a.dQ = c.dQ, a.dK = c.dK, a.dU = c.dU, a.dW = c.dW, a.dg = c.dg, a.dstate0 = c.dstate0;
    a.rec_state = rec, a.rec_dstate = rec + states, a.rec_value = rec + 2 * states;
    a.map = f.map, a.H = c.H, a.group = f.group, a.d_k = c.d_k, a.d_v = c.d_v, a.C = c.C, a.scale = c.scale;
    const int rc = launch_kernel(false, k_attn_bwd_walks<OP, MT, KP, DELTA, TWO>, dim3(2 * heads * groups), dim3(512), 0, c.stream, a, f);
    if (rc != LAUNCHED || c.n_chunk == 0) return rc;
    // 64 channels a workgroup, two of them on a compute unit; all of them where heads share a key head, whose sums take the LDS of two (4 x 4096 tokens, 16 heads of
    // 128: 268 us, 292 with all of them; 8 key heads 366 and 262).
    const unsigned units = (unsigned)(n_step * c.H_k);
    return f.group > 1 ? launch_kernel(false, k_attn_bwd_chunk<OP, MT, KP, DELTA, TWO, true, 2 * KP>, dim3(units), dim3(128 * KP), 0, c.stream, a)
                       : launch_kernel(false, k_attn_bwd_chunk<OP, MT, KP, DELTA, TWO, false, 4>, dim3(units * (KP / 2)), dim3(256), 0, c.stream, a);
}
template <int MT, bool DELTA, bool TWO> int go_k(const AttnBwdCall& c) { return c.d_k <= 64 ? go<MT, 2, DELTA, TWO>(c) : go<MT, 4, DELTA, TWO>(c); }
template <int MT, bool TWO> int go_delta(const AttnBwdCall& c) { return c.W ? go_k<MT, true, TWO>(c) : go_k<MT, false, false>(c); }

}  // namespace

#if TRIINV_INST_OP == 1
#define LAUNCHER launch_chunk_attn_bwd_f16
#else
#define LAUNCHER launch_chunk_attn_bwd_bf16
#endif
int LAUNCHER(const AttnBwdCall& c) { return c.C <= 32 ? go_delta<2, false>(c) : c.C == 64 ? go_delta<4, false>(c) : go_delta<4, true>(c); }

}  // namespace triinv
