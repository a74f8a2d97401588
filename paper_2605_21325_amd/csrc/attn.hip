// Instantiations of the chunk-attention kernels (attn.hpp) for one operand type, TRIINV_INST_OP.
#include "attn.hpp"
#include "layer.hpp"

#ifndef TRIINV_INST_OP
#error "compile with -DTRIINV_INST_OP=1|2"
#endif

namespace triinv {

namespace {

constexpr int OP = TRIINV_INST_OP;

AttnArgs args_of(const AttnCall& c)
{
    AttnArgs a{};
    a.Q = c.Q, a.K = c.K, a.U = c.U, a.W = c.W, a.g = c.g, a.state = c.state, a.O = c.O, a.final_state = c.final_state;
    const int64_t heads = (int64_t)c.n_seq * c.H;
    a.seg_state = reinterpret_cast<float*>(c.workspace);
    float* const first = a.seg_state + (c.n_seg - 1) * heads * c.d_k * c.d_v;
    a.seg_first = c.n_seg > 1 && c.state == c.final_state && c.state ? first : nullptr;
    a.seg_trans = first + heads * c.d_k * c.d_v;
    a.seg_decay = a.seg_trans;  // (one or the other)
    a.map = SeqMap{c.cu_seqlens, c.cu_chunks, c.Tlen, c.n_seq};
    a.H = c.H, a.group = c.H / c.H_k, a.d_k = c.d_k, a.d_v = c.d_v, a.C = c.C, a.n_seg = c.n_seg, a.scale = c.scale;
    return a;
}

template <int MT, int KP, bool DELTA, bool TWO> int go(const AttnCall& c)
{
    AttnArgs a = args_of(c);
    const unsigned heads = (unsigned)(c.n_seq * c.H), groups = (unsigned)((c.d_v + ATTN_COLS - 1) / ATTN_COLS);
    if (c.n_seg > 1) {
        const auto by = [&](unsigned cols) { return dim3(heads * ((c.d_v + cols - 1) / cols + (DELTA ? (c.d_k + cols - 1) / cols : 0)), (unsigned)c.n_seg - 1); };
        int rc = c.d_v > 64 ? launch_kernel(false, k_attn_states<OP, MT, KP, DELTA, ATTN_SEGMENT, TWO, 8>, by(128), dim3(512), 0, c.stream, a)
                            : launch_kernel(false, k_attn_states<OP, MT, KP, DELTA, ATTN_SEGMENT, TWO, 4>, by(64), dim3(256), 0, c.stream, a);
        if (rc != LAUNCHED) return rc;
        rc = DELTA ? launch_kernel(false, k_attn_join<KP>, dim3(heads * ((c.d_v + 15) / 16)), dim3(128 * KP), 0, c.stream, a)
                   : launch_kernel(false, k_attn_join_plain, dim3((unsigned)(((int64_t)heads * c.d_k * c.d_v + 255) / 256)), dim3(256), 0, c.stream, a);
        if (rc != LAUNCHED) return rc;
        if (a.seg_first) a.state = a.seg_first;
    }
    return launch_kernel(false, k_chunk_attn<OP, MT, KP, DELTA, TWO>, dim3(heads * groups, (unsigned)c.n_seg), dim3(512), 0, c.stream, a);
}
template <int MT, bool DELTA, bool TWO> int go_k(const AttnCall& c) { return c.d_k <= 64 ? go<MT, 2, DELTA, TWO>(c) : go<MT, 4, DELTA, TWO>(c); }
template <int MT, bool TWO> int go_delta(const AttnCall& c) { return c.W ? go_k<MT, true, TWO>(c) : go_k<MT, false, false>(c); }

}  // namespace

#if TRIINV_INST_OP == 1
#define LAUNCHER launch_chunk_attn_f16
#else
#define LAUNCHER launch_chunk_attn_bf16
#endif
int LAUNCHER(const AttnCall& c) { return c.C <= 32 ? go_delta<2, false>(c) : c.C == 64 ? go_delta<4, false>(c) : go_delta<4, true>(c); }

}  // namespace triinv
