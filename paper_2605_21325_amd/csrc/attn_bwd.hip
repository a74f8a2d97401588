// Instantiations of the chunk attention's gradient (attn_bwd.hpp) for one operand type, TRIINV_INST_OP.
#include "attn_bwd.hpp"
#include "layer.hpp"

#ifndef TRIINV_INST_OP
#error "compile with -DTRIINV_INST_OP=1|2"
#endif

namespace triinv {

namespace {

constexpr int OP = TRIINV_INST_OP;

template <int MT, int KP, bool DELTA> int go(const AttnBwdCall& c)
{
    constexpr int NT = 1, WAVES = 4, COLS = 16 * NT * WAVES;
    const unsigned heads = (unsigned)(c.n_seq * c.H), groups = (unsigned)((c.d_v + COLS - 1) / COLS);
    const int64_t states = c.n_chunk * c.H * c.d_k * c.d_v;
    float* const rec = reinterpret_cast<float*>(c.workspace);
    AttnArgs f{};
    f.K = c.K, f.U = c.U, f.W = c.W, f.g = c.g, f.state = c.state, f.rec_state = rec, f.rec_value = rec + 2 * states;
    f.map = SeqMap{c.cu_seqlens, c.cu_chunks, c.Tlen, c.n_seq};
    f.H = c.H, f.group = c.H / c.H_k, f.d_k = c.d_k, f.d_v = c.d_v, f.C = c.C, f.n_seg = 1, f.scale = c.scale;
    AttnBwdArgs a{};
    a.Q = c.Q, a.K = c.K, a.U = c.U, a.W = c.W, a.dO = c.dO, a.g = c.g, a.dstate = c.dstate;
    a.dQ = c.dQ, a.dK = c.dK, a.dU = c.dU, a.dW = c.dW, a.dg = c.dg, a.dstate0 = c.dstate0;
    a.rec_state = rec, a.rec_dstate = rec + states, a.rec_value = rec + 2 * states;
    a.map = f.map, a.n_chunk = c.n_chunk, a.H = c.H, a.group = f.group, a.d_k = c.d_k, a.d_v = c.d_v, a.C = c.C, a.scale = c.scale;
    if (c.n_chunk > 0) {
        const int rc = launch_kernel(false, k_chunk_attn<OP, MT, KP, NT, WAVES, DELTA, ATTN_RECORD>, dim3(heads * groups), dim3(64 * WAVES), 0, c.stream, f);
        if (rc != LAUNCHED) return rc;
    }
    const int rc = launch_kernel(false, k_attn_bwd_state<OP, MT, KP, NT, WAVES, DELTA>, dim3(heads * groups), dim3(64 * WAVES), 0, c.stream, a);
    if (rc != LAUNCHED || c.n_chunk == 0) return rc;
    // C = 128: eight wavefronts, a tile of channels each, where four with two would hold 192 registers of products
    constexpr int KT = MT == 8 ? 1 : KP / 2, CW = MT == 8 ? 2 * KP : 4;
    return launch_kernel(false, k_attn_bwd_chunk<OP, MT, KT, CW, DELTA>, dim3((unsigned)(c.n_chunk * c.H_k)), dim3(64 * CW), 0, c.stream, a);
}
template <int MT, bool DELTA> int go_k(const AttnBwdCall& c) { return c.d_k <= 64 ? go<MT, 2, DELTA>(c) : go<MT, 4, DELTA>(c); }
template <int MT> int go_delta(const AttnBwdCall& c) { return c.W ? go_k<MT, true>(c) : go_k<MT, false>(c); }

}  // namespace

#if TRIINV_INST_OP == 1
#define LAUNCHER launch_chunk_attn_bwd_f16
#else
#define LAUNCHER launch_chunk_attn_bwd_bf16
#endif
int LAUNCHER(const AttnBwdCall& c) { return c.C <= 32 ? go_delta<2>(c) : c.C == 64 ? go_delta<4>(c) : go_delta<8>(c); }

}  // namespace triinv
