// Gradient of the chunk attention (attn.hpp).  With the state S before a chunk, its values V' = U - W S, P = scale Q K^T . D and the gradient dS'
// that arrives at the state after it:
//     dV' = diag(e) K dS' + P^T dO                         e_i = exp(g_C - g_i),   dU = dV'
//     dS  = G_C dS' + scale Q^T diag(G) dO - W^T dV'       (arrives at the chunk before)
//     dW  = -dV' S^T
//     M   = scale (dO V'^T) . D
//     dQ  = scale diag(G) dO S^T + M K,   dK = diag(e) V' dS'^T + M^T Q
//     dg_i = <q_i, dQ_i> - <k_i, dK_i>,   and at the chunk's last token + <S', dS'>,  S' = G_C S + K^T diag(e) V' the state after it.
// In steps as there: inside a chunk of two, S and dS are those at the step's ends, W and dW go with the state before the chunk.
// Two kernels: the walks over the steps (k_attn_bwd_walks: half of its workgroups take the states and values again, half dS, last step first, with dU); everything
// else, all steps at once (k_attn_bwd_chunk).  The states between them go through memory in fp32: 0.74 GB written and 1.1 GB read for
// 4 x 4096 tokens of 16 heads of 128, where inputs and results are 0.61 GB.  The walks are bound by a step's chain (4.8 us) and what it moves (3.8 TB/s), the other by its instructions (half of the
// vector unit's cycles, a quarter of the matrix unit's) and that traffic.  Measured there: 304 and 260 us at the shortest, 376 and 302 at the median of calls under the profiler,
// 562 to 576 in all (one walk after the other: 214 + 336 us).
// dg is the difference of large sums, so what enters it (dO S^T, V' dS'^T, M) is formed from all 24 bits (fp16: 22, in its range by powers of two) of its fp32 operands, with decays
// as in the forward pass; dW ends in 16 bits and is formed from dU as it is written and 16 bits (fp16: 22) of the state (its error is that of two roundings to the type in place of
// one: 2.3e-3 against 1.7e-3 in bf16; the unrounded gradient would be 4 bytes more an element to write and to read).
#pragma once
#include "attn.hpp"

namespace triinv {

struct AttnBwdArgs {
    const void *Q, *K, *U, *W, *dO;
    const float *g, *dstate;
    void *dQ, *dK, *dU, *dW;
    float *dg, *dstate0;
    const float *rec_state, *rec_value;  // states before the steps, values (with W)
    float* rec_dstate;                   // gradients at the states after the steps
    SeqMap map;
    int H, group, d_k, d_v, C;
    float scale;
};

template <int OP, int MT, int KP, bool DELTA> struct BwdStateLayout {
    static constexpr int R = 16 * MT, PIECES = 4 * KP, UPIECES = ATTN_COLS / 8, ROWS = R * PIECES * 16;
    // Pairs of tiles of P (two tile rows, one tile column jt), tile columns one after the other.
    static constexpr int units_before(int jt)
    {
        int n = 0;
        for (int j = 0; j < jt; ++j) n += MT / 2 - j / 2;
        return n;
    }
    static constexpr int UNIT = 1024 * FULL_PARTS<OP>;
    // fp16: the wavefront that forms the pair of tiles tp, jt and brings it into range: tiles (0, 0), (1, 0), (1, 1) | (2, 0), (3, 0), (3, 3) | (2, 1), (3, 1) | (2, 2), (3, 2).
    static constexpr int maker(int tp, int jt) { return MT == 2 ? jt : tp == 0 ? 0 : jt == 3 ? 1 : jt + 1; }
    static constexpr int K_AT = 0, W_AT = 2 * ROWS, Q_AT = W_AT + (DELTA ? ROWS : 0), O_AT = Q_AT + ROWS, O_ROWS = R * UPIECES * 16, P_AT = O_AT + 2 * O_ROWS;
    static constexpr int X_AT = P_AT + units_before(MT) * UNIT, X_WAVE = 2 * KP * 1024;  // fp32 tiles, a wavefront's columns
    static constexpr int G_AT = X_AT + 4 * X_WAVE, SHIFT_AT = G_AT + 2 * StepGates<R>::FLOATS * 4, BYTES = SHIFT_AT + 16;
};

template <class LY> __device__ __forceinline__ int unit_at(int jt)  // units_before at run time
{
    int n = 0;
    for (int j = 0; j < jt; ++j) n += LY::R / 32 - j / 2;
    return n;
}

// dS from the last step to the first, a workgroup per head and 64 columns as in the forward pass.  Four wavefronts carry the recursion; four others are a step
// ahead with what does not depend on it: P, whose parts go round through LDS, and X = scale Q^T diag(G) dO in fp32.
//     first half     K dS', dV', G_C dS' + X            W and the rows of the step before to LDS
//     second half    dU, W^T dV', the parts of dS       P and X of the step before
template <int OP, int MT, int KP, bool DELTA, bool TWO>
__device__ __forceinline__ void attn_bwd_state(const AttnBwdArgs& a, char* const lds, unsigned b, unsigned n)
{
    typedef BwdStateLayout<OP, MT, KP, DELTA> LY;
    constexpr int R = LY::R, FP = FULL_PARTS<OP>, PIECES = LY::PIECES, TILES = MT * (MT + 1) / 2;
    float* const gates = reinterpret_cast<float*>(lds + LY::G_AT);
    int* const shifts = reinterpret_cast<int*>(lds + LY::SHIFT_AT);  // fp16: of the parts of P, by the wavefronts that form them
    const Lane ln = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane16 = 16 * (16 * ln.q + ln.n);
    const unsigned groups = (a.d_v + ATTN_COLS - 1) / ATTN_COLS;
    const SeqUnit mine = seq_unit(a.map, b, n, groups * a.H, by_length(a.map, 2 * n), lds);
    const unsigned cg = mine.unit % groups;
    const int h = mine.unit / groups, s = mine.seq, hs = s * a.H + h, wg_col = cg * ATTN_COLS;
    const SeqPos sq = seq_pos(a.map, s);
    const int64_t n_chunk = pieces_of(sq.len, a.C);
    const int tokens = a.C < R ? a.C : R, steps = a.C > R ? a.C / R : 1;
    const int64_t k1 = pieces_of(sq.len, tokens);
    const uint32_t stride_u = 2u * a.H * a.d_v;
    const MinusOne<OP> minus(ln);

    if (wave < 4) {
        const int col0 = wg_col + 16 * wave;
        const TurnOne<OP> one_k(ln, true);
        const int64_t rec0 = (a.map.cu_chunks ? a.map.cu_chunks[s] : s * n_chunk) * steps;
        v4f S[2 * KP], E[TWO ? 2 * KP : 1];  // dS; what the chunk's values pass on to the state before it
        get_state<KP>(a.dstate ? a.dstate + (int64_t)hs * a.d_k * a.d_v : nullptr, S, a.d_k, a.d_v, col0, false, ln);
        if constexpr (TWO) {
#pragma unroll
            for (int i = 0; i < 2 * KP; ++i) E[i] = zero4();
        }
        Parts<FP> sp[KP];
        int s_shift = 0;
        auto parts_of_state = [&]() {
            if constexpr (OP == OP_F16) s_shift = f16_shift(wave_max(most_of(S)));
            v4f x[2 * KP];
#pragma unroll
            for (int i = 0; i < 2 * KP; ++i) x[i] = OP == OP_F16 ? times(S[i], pow2(s_shift)) : S[i];
            split_pairs<OP, FP, KP>(x, sp, minus);
        };
        parts_of_state();
        __syncthreads();
        __syncthreads();  // the last step's rows, P and X are in LDS
        for (int64_t k = k1 - 1; k >= 0; --k) {
            const float* const gl = gates + (k & 1) * StepGates<R>::FLOATS;
            const char* const rows_k = lds + LY::K_AT + (k & 1) * LY::ROWS;
            v4f dv[MT];
            rows_times<OP, MT, KP>(dv, rows_k, sp, ln, [&](int p) {
                put_turned<OP>(a.rec_dstate + ((rec0 + k) * a.H + h) * a.d_k * a.d_v, p, sp[p], pow2(-s_shift), a.d_k, a.d_v, col0, one_k, ln);
            });
            v4u pt[MT / 2][FP][MT], o[MT / 2];
#pragma unroll
            for (int tp = 0; tp < MT / 2; ++tp) {
                const char* const rows_o = lds + LY::O_AT + (k & 1) * LY::O_ROWS;
                const int row = 32 * tp + 4 * ln.q + (ln.n >> 2), col4 = 4 * wave + (ln.n & 3);
                const v2u u = lds_turned<LY::UPIECES>(rows_o, row, col4), v = lds_turned<LY::UPIECES>(rows_o, row + 16, col4);
                o[tp] = v4u{u[0], u[1], v[0], v[1]};
#pragma unroll
                for (int part = 0; part < FP; ++part)
#pragma unroll
                    for (int jt = 0; jt <= 2 * tp + 1; ++jt) pt[tp][part][jt] = *reinterpret_cast<const v4u*>(lds + LY::P_AT + LY::UNIT * (LY::units_before(jt) + tp - jt / 2) + 1024 * part + lane16);
            }
            typedef int v4i __attribute__((ext_vector_type(4)));
            v4i p_shift = {0, 0, 0, 0};
            if constexpr (OP == OP_F16) p_shift = *reinterpret_cast<const v4i*>(shifts);
            const float decay = gl[3 * R];
#pragma unroll
            for (int tb = 0; tb < MT; ++tb) {
                const v4f e = *reinterpret_cast<const v4f*>(gl + R + 16 * tb + 4 * ln.q);
                const float f = OP == OP_F16 ? pow2(-s_shift) * pow2(p_shift[LY::maker(tb / 2, tb)]) : 1.f;
#pragma unroll
                for (int r = 0; r < 4; ++r) dv[tb][r] *= OP == OP_F16 ? e[r] * f : e[r];
            }
            in_order();
#pragma unroll
            for (int tp = 0; tp < MT / 2; ++tp) {
                if constexpr (OP == OP_F16) {
#pragma unroll
                    for (int jt = 0; jt < 2 * tp; ++jt) dv[jt] = times(dv[jt], pow2(p_shift[LY::maker(tp, jt)] - p_shift[LY::maker(tp - 1, jt)]));
                }
#pragma unroll
                for (int part = FP - 1; part >= 0; --part)
#pragma unroll
                    for (int jt = 0; jt <= 2 * tp + 1; ++jt) dv[jt] = mfma32<OP>(pt[tp][part][jt], o[tp], dv[jt]);
            }
            if constexpr (OP == OP_F16) {
#pragma unroll
                for (int jt = 0; jt < MT; ++jt) dv[jt] = times(dv[jt], pow2(-p_shift[LY::maker(MT / 2 - 1, jt)]));
            }
#pragma unroll
            for (int i = 0; i < 2 * KP; ++i) {
                const v4f x = *reinterpret_cast<const v4f*>(lds + LY::X_AT + LY::X_WAVE * wave + 1024 * i + lane16);
#pragma unroll
                for (int r = 0; r < 4; ++r) S[i][r] = decay * S[i][r] + x[r];
            }
            __syncthreads();  // this step's P, X, K and dO are used up, W is in LDS
            {
                const StepPos at = step_pos<R>(sq, k, k1, a.C);
                const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(a.dU) + at.row * stride_u + 2 * ((int64_t)h * a.d_v), 0,
                                                                    (uint32_t)(at.valid - 1) * stride_u + 2u * a.d_v, 0x00020000);
                uint32_t to = col0 + ln.n < a.d_v ? 4 * ln.q * stride_u + 2u * (col0 + ln.n) : 0x80000000u;
#pragma unroll
                for (int tb = 0; tb < MT; ++tb, to += 12 * stride_u) {
                    const v2u x = pack4<OP>(dv[tb]);
#pragma unroll
                    for (int r = 0; r < 4; ++r, to += stride_u) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(x[r >> 1] >> (16 * (r & 1))), rsrc, to, 0, 0);
                }
            }
            if constexpr (DELTA) {
                int shift = 0;
                if constexpr (OP == OP_F16) shift = f16_shift(wave_max(most_of(dv)));
                const float up = OP == OP_F16 ? -pow2(shift) : -1.f;
#pragma unroll
                for (int tb = 0; tb < MT; ++tb) dv[tb] = times(dv[tb], up);
                Parts<FP> vp[MT / 2];
                split_pairs<OP, FP, MT / 2>(dv, vp, minus);
                if constexpr (TWO) {  // dS takes it at the chunk's first step
#pragma unroll
                    for (int i = 0; i < 2 * KP; ++i) E[i] = OP == OP_F16 ? times(E[i], pow2(shift)) : E[i];
                    add_turned<OP, MT, KP>(E, lds + LY::W_AT, vp, ln);
#pragma unroll
                    for (int i = 0; i < 2 * KP; ++i) {
                        if constexpr (OP == OP_F16) E[i] = times(E[i], pow2(-shift));
                        if ((k & 1) == 0) {
#pragma unroll
                            for (int r = 0; r < 4; ++r) S[i][r] += E[i][r];
                            E[i] = zero4();
                        }
                    }
                } else {
                    if constexpr (OP == OP_F16) {
#pragma unroll
                        for (int i = 0; i < 2 * KP; ++i) S[i] = times(S[i], pow2(shift));
                    }
                    add_turned<OP, MT, KP>(S, lds + LY::W_AT, vp, ln);
                    if constexpr (OP == OP_F16) {
#pragma unroll
                        for (int i = 0; i < 2 * KP; ++i) S[i] = times(S[i], pow2(-shift));
                    }
                }
            }
            parts_of_state();
            __syncthreads();  // P and X of the next step are in LDS
        }
        if (a.dstate0) put_state<KP>(a.dstate0 + (int64_t)hs * a.d_k * a.d_v, S, a.d_k, a.d_v, col0, ln);
        return;
    }

    // A step ahead: what does not depend on dS.
    const int tid = threadIdx.x - 256, w4 = wave - 4, hk = h / a.group, H_k = a.H / a.group, cols = a.d_v - wg_col < ATTN_COLS ? a.d_v - wg_col : ATTN_COLS;
    RowLoader<PIECES, R, 256> lq, lk, lw;
    RowLoader<LY::UPIECES, R, 256> lo;
    StepGates<R> lg;
    const uint32_t stride_k = 2u * H_k * a.d_k, stride_w = 2u * a.H * a.d_k;
    auto request = [&](int64_t k) {
        const StepPos at = step_pos<R>(sq, k, k1, a.C);
        lk.load(static_cast<const char*>(a.K) + at.row * stride_k + 2 * hk * a.d_k, stride_k, a.d_k, at.valid, tid);
        lq.load(static_cast<const char*>(a.Q) + at.row * stride_k + 2 * hk * a.d_k, stride_k, a.d_k, at.valid, tid);
        lo.load(static_cast<const char*>(a.dO) + at.row * stride_u + 2 * ((int64_t)h * a.d_v + wg_col), stride_u, cols, at.valid, tid);
        lg.load(a.g, at, a.H, h, tid);
    };
    auto bring = [&](int64_t k) {
        lk.store(lds + LY::K_AT + (k & 1) * LY::ROWS, tid);
        lq.store(lds + LY::Q_AT, tid);
        lo.store(lds + LY::O_AT + (k & 1) * LY::O_ROWS, tid);
        lg.store(gates + (k & 1) * StepGates<R>::FLOATS, a.scale, tid);
    };
    auto request_w = [&](int64_t k) {
        if constexpr (DELTA) {
            const StepPos at = step_pos<R>(sq, k, k1, a.C);
            lw.load(static_cast<const char*>(a.W) + at.row * stride_w + 2 * (int64_t)h * a.d_k, stride_w, a.d_k, at.valid, tid);
        }
    };
    // P, as operands of P^T: token rows 4 q + r, column n; a share of the tiles a wavefront (one without a tile forms the last one again); fp16: both tiles of a pair
    // by one wavefront, which brings what it forms into range by one power of two.
    constexpr int SHARE = OP == OP_F16 && MT == 2 ? 2 : (TILES + 3) / 4;
    int its[SHARE], jts[SHARE], units[SHARE];
#pragma unroll
    for (int j = 0; j < SHARE; ++j) {
        int idx = j * 4 + w4 < TILES ? j * 4 + w4 : TILES - 1, it = 0;
        while (idx > it) idx -= ++it;
        if constexpr (OP == OP_F16 && MT == 2) it = w4 == 0 ? j : 1, idx = w4 == 0 ? 0 : 1;
        if constexpr (OP == OP_F16 && MT == 4) it = w4 == 0 ? (j + 1) / 2 : j == 0 ? 2 : 3, idx = w4 == 0 ? j / 2 : j == 2 && w4 == 1 ? 3 : w4 - 1;
        its[j] = it, jts[j] = idx, units[j] = LY::UNIT * (unit_at<LY>(idx) + (it >> 1) - (idx >> 1)) + 8 * (it & 1);
    }
    auto scores = [&](int64_t k) {
        const float* const gl = gates + (k & 1) * StepGates<R>::FLOATS;
        const char* const rows_k = lds + LY::K_AT + (k & 1) * LY::ROWS;
        v4f x[SHARE], gi[SHARE];
        float gj[SHARE];
        v4u qs[2][SHARE], ks[2][SHARE];
        auto rows_of = [&](int p) {
            const uint32_t at = in_place(LdsRows<PIECES>::at(ln.n, 4 * p + ln.q));
#pragma unroll
            for (int j = 0; j < SHARE; ++j) {
                qs[p & 1][j] = *reinterpret_cast<const v4u*>(lds + LY::Q_AT + 16 * LdsRows<PIECES>::BYTES * its[j] + at);
                ks[p & 1][j] = *reinterpret_cast<const v4u*>(rows_k + 16 * LdsRows<PIECES>::BYTES * jts[j] + at);
            }
        };
        rows_of(0);
#pragma unroll
        for (int j = 0; j < SHARE; ++j) {
            gj[j] = gl[16 * jts[j] + ln.n];
            gi[j] = *reinterpret_cast<const v4f*>(gl + 16 * its[j] + 4 * ln.q);
            x[j] = zero4();
        }
#pragma unroll
        for (int p = 0; p < KP; ++p) {
            if (p + 1 < KP) rows_of(p + 1);
            in_order();
#pragma unroll
            for (int j = 0; j < SHARE; ++j) x[j] = mfma32<OP>(qs[p & 1][j], ks[p & 1][j], x[j]);
        }
#pragma unroll
        for (int j = 0; j < SHARE; ++j) {
#pragma unroll
            for (int r = 0; r < 4; ++r) x[j][r] *= a.scale * __expf(jts[j] == its[j] && ln.n > 4 * ln.q + r ? -__builtin_inff() : gi[j][r] - gj[j]);
        }
        if constexpr (OP == OP_F16) {
            const int shift = f16_shift(wave_max(most_of(x)));
            if (ln.q == 0 && ln.n == 0) shifts[MT == 2 && w4 > 1 ? 1 : w4] = shift;
#pragma unroll
            for (int j = 0; j < SHARE; ++j) x[j] = times(x[j], pow2(shift));
        }
#pragma unroll
        for (int j = 0; j < SHARE; ++j) {
            const bool on = jts[j] == its[j];
            char* unit = lds + LY::P_AT + units[j] + in_place(lane16);
#pragma unroll
            for (int part = 0; part < FP; ++part) {
                const v2u u = pack4<OP>(x[j]);
                *reinterpret_cast<v2u*>(unit + 1024 * part) = u;
                if (on && (its[j] & 1)) *reinterpret_cast<v2u*>(unit + 1024 * part - 8) = v2u{0u, 0u};  // the pair's other tile lies above the diagonal
                x[j] = minus16<OP>(x[j], u);
            }
        }
    };
    auto products = [&](int64_t k) {  // X of this wavefront's columns
        const float* const gl = gates + (k & 1) * StepGates<R>::FLOATS;
        const char* const rows_o = lds + LY::O_AT + (k & 1) * LY::O_ROWS;
        v4f od[MT], x[2 * KP];
#pragma unroll
        for (int tb = 0; tb < MT; ++tb) {
            const v4f u = unpack4<OP>(lds_turned<LY::UPIECES>(rows_o, 16 * tb + 4 * ln.q + (ln.n >> 2), 4 * w4 + (ln.n & 3)));
            const v4f e = *reinterpret_cast<const v4f*>(gl + 2 * R + 16 * tb + 4 * ln.q);
#pragma unroll
            for (int r = 0; r < 4; ++r) od[tb][r] = u[r] * e[r];
        }
        int shift = 0;
        if constexpr (OP == OP_F16) {
            shift = f16_shift(wave_max(most_of(od)));
#pragma unroll
            for (int tb = 0; tb < MT; ++tb) od[tb] = times(od[tb], pow2(shift));
        }
        Parts<FP> vp[MT / 2];
        split_pairs<OP, FP, MT / 2>(od, vp, minus);
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i) x[i] = zero4();
        add_turned<OP, MT, KP>(x, lds + LY::Q_AT, vp, ln);
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i) *reinterpret_cast<v4f*>(lds + LY::X_AT + LY::X_WAVE * w4 + 1024 * i + lane16) = OP == OP_F16 ? times(x[i], pow2(-shift)) : x[i];
    };
    request(k1 - 1);
    request_w(k1 - 1);
    bring(k1 - 1);
    __syncthreads();
    request(k1 - 2);
    scores(k1 - 1);
    products(k1 - 1);
    __syncthreads();
    for (int64_t k = k1 - 1; k >= 0; --k) {
        if constexpr (DELTA) lw.store(lds + LY::W_AT, tid);
        bring(k - 1);
        __syncthreads();  // P and X in LDS are used up, the rows are there
        request_w(k - 1);
        scores(k - 1);
        request(k - 2);
        products(k - 1);
        __syncthreads();
    }
}

// The two walks do not need each other: the first half of the grid takes dS, the longer one, the second half the states.
template <int OP, int MT, int KP, bool DELTA, bool TWO>
__global__ __launch_bounds__(512) void k_attn_bwd_walks(AttnBwdArgs a, AttnArgs f)
{
    constexpr int OF_STATES = StatesLayout<OP, MT, KP, DELTA, 4>::BYTES, OF_DS = BwdStateLayout<OP, MT, KP, DELTA>::BYTES;
    __shared__ __attribute__((aligned(16))) char lds[OF_DS > OF_STATES ? OF_DS : OF_STATES];
    const unsigned units = gridDim.x / 2;
    if (blockIdx.x < units) {
        attn_bwd_state<OP, MT, KP, DELTA, TWO>(a, lds, blockIdx.x, units);
    } else {
        attn_states<OP, MT, KP, DELTA, ATTN_RECORD, TWO, 4>(f, lds, blockIdx.x - units, units, by_length(f.map, 2 * units), 0);
    }
}

// Everything that needs the states at both ends of a step: a workgroup per step and key head, which takes the heads that share it one
// after the other and d_v in blocks of 64 columns.  A wavefront has KT tiles of 16 channels of all tokens; the products stand turned
// (channels down, tokens across), so that a lane's four values are neighbours in memory.  The next block's rows are requested before one is used.
template <int OP, int MT, int WAVES, bool DELTA> struct BwdChunkLayout {
    static constexpr int R = 16 * MT, PIECES = 2 * WAVES, CB = 8;  // pieces of a row of channels; of a block of d_v
    static constexpr int VP = DELTA ? FULL_PARTS<OP> : 1;
    static constexpr int ROWS = R * PIECES * 16, BLOCK = R * CB * 16;
    static constexpr int TILES = MT * (MT + 1) / 2, M_BYTES = TILES * FULL_PARTS<OP> * TURN16_BYTES;
    static constexpr int COLS_BYTES = (1 + VP + (DELTA ? 1 : 0)) * BLOCK;  // dO, V', dV'
    static constexpr int K_AT = 0, Q_AT = ROWS, O_AT = 2 * ROWS, V_AT = O_AT + BLOCK, DV_AT = V_AT + VP * BLOCK;
    static constexpr int M_AT = O_AT;  // when the blocks of d_v are used up
    static constexpr int G_AT = O_AT + (COLS_BYTES > M_BYTES ? COLS_BYTES : M_BYTES), RED_AT = G_AT + StepGates<R>::FLOATS * 4;
    static constexpr int BYTES = RED_AT + (2 * R + 3) * WAVES * 4, SUM_BYTES = 2 * WAVES * MT * 1024;
};

// Recorded values, as put_turned left them, on their way to LDS as rows of 16-bit parts: 64 columns a time.
template <int OP, int N, int MT, int THREADS> struct ValueLoader {
    static constexpr int BAND = THREADS / 128, COUNT = (MT + BAND - 1) / BAND;  // tiles of tokens at once
    v4f v[COUNT][2];
    __device__ __forceinline__ void load(const float* first, int v0, int d_v, int valid, int tid)
    {
        const int n = tid & 15, col = v0 + 8 * ((tid >> 4) & 7);
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(first), 0, (uint32_t)valid * d_v * 4u, 0x00020000);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int band = (tid >> 7) + i * BAND, of_band = valid - 16 * band < 16 ? valid - 16 * band : 16;
            const uint32_t at = n < of_band && col < d_v ? 4u * (16 * band * d_v + col * of_band + 4 * n) : 0x80000000u;
            v[i][0] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0));
            v[i][1] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at + 16u * of_band, 0, 0));
        }
    }
    __device__ __forceinline__ float most() const
    {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) x = fmaxf(x, most_of(v[i]));
        return x;
    }
    // (fp16: times 2^shift)
    __device__ __forceinline__ void store(char* m, int plane, int shift, int tid) const
    {
        const int tb = tid >> 7;
        if (MT < BAND && tb >= MT) return;
        char* const to = m + LdsRows<8>::at(16 * tb + (tid & 15), (tid >> 4) & 7);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const Parts<N> p = OP == OP_F16 ? split_pair<OP, N>(times(v[i][0], pow2(shift)), times(v[i][1], pow2(shift))) : split_pair<OP, N>(v[i][0], v[i][1]);
#pragma unroll
            for (int j = 0; j < N; ++j) *reinterpret_cast<v4u*>(to + j * plane + i * BAND * 16 * LdsRows<8>::BYTES) = p.u[j];
        }
    }
};

// fp16: the power of two of a block of columns when those before it (v0 of them) took `before`.  It only falls: what has been summed up is never
// scaled past what fp32 holds, and a block of less than the largest needs no more bits than those.
__device__ __forceinline__ int shift_so_far(int shift, int before, int v0) { return v0 && before < shift ? before : shift; }

__device__ __forceinline__ float wave_sum(float x)
{
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}

// Tokens 32 tp .. 32 tp + 31 of the channels ch .. ch + 15, as an operand over the tokens.
template <int PIECES> __device__ __forceinline__ v4u lds_turned_channels(const char* m, int tp, int ch, Lane ln)
{
    const int row = 32 * tp + 4 * ln.q + (ln.n >> 2), col4 = (ch >> 2) + (ln.n & 3);
    const v2u a = lds_turned<PIECES>(m, row, col4), b = lds_turned<PIECES>(m, row + 16, col4);
    return v4u{a[0], a[1], b[0], b[1]};
}

// SHARED: heads share a key head, whose dQ and dK are summed in LDS.
template <int OP, int MT, int KP, bool DELTA, bool TWO, bool SHARED, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void k_attn_bwd_chunk(AttnBwdArgs a)
{
    typedef BwdChunkLayout<OP, MT, WAVES, DELTA> LY;
    constexpr int R = LY::R, THREADS = 64 * WAVES, KT = 1, SHARE = (LY::TILES + WAVES - 1) / WAVES, FP = FULL_PARTS<OP>;
    __shared__ __attribute__((aligned(16))) char lds[LY::BYTES + (SHARED ? LY::SUM_BYTES : 0)];
    float* const gl = reinterpret_cast<float*>(lds + LY::G_AT);
    float* const red = reinterpret_cast<float*>(lds + LY::RED_AT);  // sums over channels: [2][wavefront][token], then [3][wavefront]
    float* const red1 = red + 2 * WAVES * R;
    const Lane ln = lane_id();
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), H_k = a.H / a.group;
    constexpr int HALVES = 2 * KP / WAVES;
    const unsigned bh = xcd_neighbours(blockIdx.x, gridDim.x), b = bh / HALVES;
    const int half0 = 64 * (bh % HALVES);  // the workgroup's first channel
    const int hk = b % H_k, steps = a.C > R ? a.C / R : 1, tokens = a.C < R ? a.C : R;
    const unsigned id = b / H_k, chunk = id >> (steps - 1);  // of the step, and its chunk
    SeqPos sq;
    int64_t k;  // the step in its sequence
    if (a.map.cu_chunks) {
        int lo = 0, hi = a.map.n_seq - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (a.map.cu_chunks[mid] <= chunk) lo = mid;
            else hi = mid - 1;
        }
        sq = seq_pos(a.map, lo), k = (int64_t)id - a.map.cu_chunks[lo] * steps;
    } else {
        const unsigned cps = (unsigned)pieces_of(a.map.Tlen, a.C);
        sq = SeqPos{(int64_t)(chunk / cps) * a.map.Tlen, a.map.Tlen}, k = (int64_t)(chunk % cps) * steps + (id & (steps - 1));
    }
    const int64_t all = pieces_of(sq.len, tokens);
    if (k >= all) return;  // (the second step of a chunk that ends in its first)
    const StepPos at = step_pos<R>(sq, k, all, a.C);
    const bool chunk_ends = steps == 1 || (k & 1) || k + 1 == all;
    const int ch0 = 16 * KT * wave;  // this wavefront's first, of those
    const uint32_t stride_k = 2u * H_k * a.d_k, stride_u = 2u * a.H * a.d_v;
    const MinusOne<OP> minus(ln);
    RowLoader<LY::CB, R, THREADS> lo, lu;  // dO; dV', or V' itself
    ValueLoader<OP, FP, MT, THREADS> lv;
    StepGates<R> lg;
    auto request = [&](int h, int v0) {
        const int cols = a.d_v - v0 < 64 ? a.d_v - v0 : 64;
        const int64_t first = (at.row * a.H + h) * a.d_v + v0;
        lo.load(static_cast<const uint16_t*>(a.dO) + first, stride_u, cols, at.valid, tid);
        lu.load(static_cast<const uint16_t*>(DELTA ? a.dU : a.U) + first, stride_u, cols, at.valid, tid);
        if constexpr (DELTA) lv.load(a.rec_value + (at.row * a.H + h * at.valid) * a.d_v, v0, a.d_v, at.valid, tid);
    };
    v4f sv[KT][2][2], dsv[KT][2][2];  // this wavefront's rows of S and dS', the block's columns
    v4f szv[TWO ? KT : 1][2][2];      // of the state before the chunk, in its second step
    const bool second = TWO && (k & 1);
    auto request_states = [&](int h, int v0) {
        const int64_t size = a.d_k * a.d_v;
        const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(a.rec_state) + ((int64_t)id * a.H + h) * size, 0, (uint32_t)size * 4u, 0x00020000);
        const auto rd = __builtin_amdgcn_make_buffer_rsrc(a.rec_dstate + ((int64_t)id * a.H + h) * size, 0, (uint32_t)size * 4u, 0x00020000);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const int ch = half0 + ch0 + 16 * kt, col = v0 + 32 * ks + 8 * ln.q;
                const uint32_t from = ch < a.d_k && col < a.d_v ? 4u * (ch * a.d_v + 16 * col + 4 * ln.n) : 0x80000000u;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    sv[kt][ks][half] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(rs, from + 256u * half, 0, 0));
                    dsv[kt][ks][half] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(rd, from + 256u * half, 0, 0));
                    if constexpr (TWO) {
                        const auto rz = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(a.rec_state) + ((int64_t)(id - second) * a.H + h) * size, 0, (uint32_t)size * 4u, 0x00020000);
                        szv[kt][ks][half] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(rz, from + 256u * half, 0, 0));
                    }
                }
            }
    };
    const int h0 = hk * a.group;
    request(h0, 0);
    {
        RowLoader<LY::PIECES, R, THREADS> lk, lq;
        lk.load(static_cast<const char*>(a.K) + at.row * stride_k + 2 * (hk * a.d_k + half0), stride_k, a.d_k - half0, at.valid, tid);
        lq.load(static_cast<const char*>(a.Q) + at.row * stride_k + 2 * (hk * a.d_k + half0), stride_k, a.d_k - half0, at.valid, tid);
        lg.load(a.g, at, a.H, h0, tid);
        request_states(h0, 0);
        lk.store(lds + LY::K_AT, tid);
        lq.store(lds + LY::Q_AT, tid);
    }
    auto put_rows = [&](void* to, const v4f x, int heads, int head, int ch, int it) {
        const uint32_t stride = 2u * heads * a.d_k;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(to) + at.row * stride + 2 * head * a.d_k, 0, (uint32_t)(at.valid - 1) * stride + 2u * a.d_k, 0x00020000);
        __builtin_amdgcn_raw_buffer_store_b64(pack4<OP>(x), rsrc, in_place(ch < a.d_k ? ln.n * stride + 2u * ch : 0x80000000u) + 16 * it * stride, 0, 0);
    };

    for (int h = h0; h < h0 + (SHARED ? a.group : 1); ++h) {
        const bool last_h = !SHARED || h + 1 == h0 + a.group;
        lg.store(gl, a.scale, tid);
        v4f X[KT][MT], Y[KT][MT], Z[KT][MT], M[SHARE];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int it = 0; it < MT; ++it) X[kt][it] = Y[kt][it] = Z[kt][it] = zero4();
#pragma unroll
        for (int j = 0; j < SHARE; ++j) M[j] = zero4();
        // this wavefront's tiles of M (one without a tile forms the last one again, and writes the same)
        int its[SHARE], jts[SHARE], idx[SHARE];
#pragma unroll
        for (int j = 0; j < SHARE; ++j) {
            int x = j * WAVES + wave < LY::TILES ? j * WAVES + wave : LY::TILES - 1, it = 0;
            idx[j] = x;
            while (x > it) x -= ++it;
            its[j] = it, jts[j] = x;
        }
        float s_ds = 0.f;
        int s_shift = 0, d_shift = 0, z_shift = 0, v_shift = 0;
        for (int v0 = 0; v0 < a.d_v; v0 += 64) {
            lo.store(lds + LY::O_AT, tid);
            if constexpr (DELTA) {
                lu.store(lds + LY::DV_AT, tid);
                if constexpr (OP == OP_F16) {  // V' into fp16's range, by a power of two that all wavefronts agree on, and what there is of the products with it
                    const float mine = wave_max(lv.most());
                    if (ln.q == 0 && ln.n == 0) red1[wave] = mine;
                    __syncthreads();
                    float most = red1[0];
#pragma unroll
                    for (int w = 1; w < WAVES; ++w) most = fmaxf(most, red1[w]);
                    const int nv = shift_so_far(__builtin_amdgcn_readfirstlane(f16_shift(most)), v_shift, v0);
                    const float cv = v0 ? pow2(nv - v_shift) : 1.f;
                    v_shift = nv;
#pragma unroll
                    for (int j = 0; j < SHARE; ++j) M[j] = times(M[j], cv);
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int it = 0; it < MT; ++it) Y[kt][it] = times(Y[kt][it], cv);
                }
                lv.store(lds + LY::V_AT, LY::BLOCK, v_shift, tid);
            } else {
                lu.store(lds + LY::V_AT, tid);
            }
            __syncthreads();
            const bool last_block = v0 + 64 >= a.d_v;
            const int next_h = last_block ? (SHARED && h + 1 < h0 + a.group ? h + 1 : h) : h, next_v = last_block ? (SHARED && h + 1 < h0 + a.group ? 0 : a.d_v) : v0 + 64;
            if (next_v < a.d_v) request(next_h, next_v);
            if constexpr (OP == OP_F16) in_order();  // (registers, as below)
            // dO V'^T, turned: value tokens down, output tokens across
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int part = LY::VP - 1; part >= 0; --part)
#pragma unroll
                    for (int j = 0; j < SHARE; ++j)
                        M[j] = mfma32<OP>(lds_row<LY::CB>(lds + LY::V_AT + part * LY::BLOCK, 16 * jts[j] + ln.n, 4 * ks + ln.q), lds_row<LY::CB>(lds + LY::O_AT, 16 * its[j] + ln.n, 4 * ks + ln.q), M[j]);
            // S dO^T, S dV'^T and dS' V'^T
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) s_ds += sv[kt][i >> 3][i >> 2 & 1][i & 3] * dsv[kt][i >> 3][i >> 2 & 1][i & 3];
            if constexpr (OP == OP_F16) {  // both into fp16's range, and what there is of the products with them
                float most_s = 0.f, most_d = 0.f;
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) most_s = fmaxf(most_s, fabsf(sv[kt][i >> 3][i >> 2 & 1][i & 3])), most_d = fmaxf(most_d, fabsf(dsv[kt][i >> 3][i >> 2 & 1][i & 3]));
                const int ns = shift_so_far(f16_shift(wave_max(most_s)), s_shift, v0), nd = shift_so_far(f16_shift(wave_max(most_d)), d_shift, v0);
                const float us = pow2(ns), ud = pow2(nd), cs = v0 ? pow2(ns - s_shift) : 1.f, cd = v0 ? pow2(nd - d_shift) : 1.f;
                s_shift = ns, d_shift = nd;
                float cz = cs;
                if constexpr (TWO) {
                    float most_z = 0.f;
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int i = 0; i < 16; ++i) most_z = fmaxf(most_z, fabsf(szv[kt][i >> 3][i >> 2 & 1][i & 3]));
                    const int nz = shift_so_far(f16_shift(wave_max(most_z)), z_shift, v0);
                    cz = v0 ? pow2(nz - z_shift) : 1.f;
                    z_shift = nz;
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int i = 0; i < 16; ++i) szv[kt][i >> 3][i >> 2 & 1][i & 3] *= pow2(nz);
                } else {
                    z_shift = ns;
                }
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) sv[kt][i >> 3][i >> 2 & 1][i & 3] *= us, dsv[kt][i >> 3][i >> 2 & 1][i & 3] *= ud;
#pragma unroll
                    for (int it = 0; it < MT; ++it)
#pragma unroll
                        for (int r = 0; r < 4; ++r) X[kt][it][r] *= cs, Z[kt][it][r] *= cz, Y[kt][it][r] *= cd;
                }
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                // (Left alone it takes registers for all of it at once; what fp16 scales by leaves it fewer of them.)
                in_order();
                Parts<FP> sp[KT], dp[KT];
                v4f x[2 * KT];
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) x[2 * kt] = sv[kt][ks][0], x[2 * kt + 1] = sv[kt][ks][1];
                split_pairs<OP, FP, KT>(x, sp, minus);
                if constexpr (DELTA) {
                    Parts<2> zp[KT];
                    if constexpr (TWO) {
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt) x[2 * kt] = szv[kt][ks][0], x[2 * kt + 1] = szv[kt][ks][1];
                        split_pairs<OP, 2, KT>(x, zp, minus);
                    } else {
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt) zp[kt].u[0] = sp[kt].u[0], zp[kt].u[1] = sp[kt].u[1];
                    }
                    if constexpr (OP == OP_F16) in_order();
                    v4u d[MT];
#pragma unroll
                    for (int it = 0; it < MT; ++it) d[it] = lds_row<LY::CB>(lds + LY::DV_AT, 16 * it + ln.n, 4 * ks + ln.q);
#pragma unroll
                    for (int part = 1; part >= 0; --part)
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                            for (int it = 0; it < MT; ++it) Z[kt][it] = mfma32<OP>(zp[kt].u[part], d[it], Z[kt][it]);
                }
                if constexpr (OP == OP_F16) in_order();
                v4u o[MT];
#pragma unroll
                for (int it = 0; it < MT; ++it) o[it] = lds_row<LY::CB>(lds + LY::O_AT, 16 * it + ln.n, 4 * ks + ln.q);
#pragma unroll
                for (int part = FP - 1; part >= 0; --part)
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int it = 0; it < MT; ++it) X[kt][it] = mfma32<OP>(sp[kt].u[part], o[it], X[kt][it]);
                if constexpr (OP == OP_F16) in_order();
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) x[2 * kt] = dsv[kt][ks][0], x[2 * kt + 1] = dsv[kt][ks][1];
                split_pairs<OP, FP, KT>(x, dp, minus);
                // parts of both sides: what is left out is below the last bit kept
#pragma unroll
                for (int j = LY::VP - 1; j >= 0; --j) {
                    if constexpr (OP == OP_F16) in_order();
                    v4u v[MT];
#pragma unroll
                    for (int it = 0; it < MT; ++it) v[it] = lds_row<LY::CB>(lds + LY::V_AT + j * LY::BLOCK, 16 * it + ln.n, 4 * ks + ln.q);
#pragma unroll
                    for (int i = FP - 1 - j; i >= 0; --i)
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                            for (int it = 0; it < MT; ++it) Y[kt][it] = mfma32<OP>(dp[kt].u[i], v[it], Y[kt][it]);
                }
            }
            if (next_v < a.d_v) request_states(next_h, next_v);
            __syncthreads();  // the block is used up
        }
        if (SHARED && h + 1 < h0 + a.group) lg.load(a.g, at, a.H, h + 1, tid);
        // M = scale (dO V'^T) . D, in parts; fp16: times a power of two that all wavefronts agree on
#pragma unroll
        for (int j = 0; j < SHARE; ++j) {
            const float gi = gl[16 * its[j] + ln.n];
            const v4f gj = *reinterpret_cast<const v4f*>(gl + 16 * jts[j] + 4 * ln.q);
#pragma unroll
            for (int r = 0; r < 4; ++r) M[j][r] *= (OP == OP_F16 && DELTA ? pow2(-v_shift) : 1.f) * a.scale * __expf(jts[j] < its[j] || 4 * ln.q + r <= ln.n ? gi - gj[r] : -__builtin_inff());
        }
        int m_shift = 0;
        if constexpr (OP == OP_F16) {
            const float mine = wave_max(most_of(M));
            if (ln.q == 0 && ln.n == 0) red1[wave] = mine;
            __syncthreads();
            float most = red1[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) most = fmaxf(most, red1[w]);
            m_shift = f16_shift(most);
        }
        const Turn16 turn(reinterpret_cast<float*>(lds + LY::M_AT), ln);
#pragma unroll
        for (int j = 0; j < SHARE; ++j) {
            v4f m = OP == OP_F16 ? times(M[j], pow2(m_shift)) : M[j];
#pragma unroll
            for (int part = 0; part < FP; ++part) {
                const v2u x = pack4<OP>(m);
                turn.put(part * LY::TILES + idx[j], x);
                m = minus16<OP>(m, x);
            }
        }
        __syncthreads();
        // dQ (turned): lanes are tokens i, K^T M^T over the tokens j <= i.   dK: lanes are tokens j, Q^T M over i >= j.
        const float up = OP == OP_F16 ? pow2(m_shift) : 1.f, down = OP == OP_F16 ? pow2(-m_shift) : 1.f;
        const float s_down = OP == OP_F16 ? pow2(-s_shift) : 1.f, d_down = OP == OP_F16 ? pow2(-d_shift) * pow2(-v_shift) : 1.f;
        float inter = 0.f;
        v4u kt_op[KT][MT / 2], qt_op[KT][MT / 2];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int tp = 0; tp < MT / 2; ++tp) {
                kt_op[kt][tp] = lds_turned_channels<LY::PIECES>(lds + LY::K_AT, tp, ch0 + 16 * kt, ln);
                qt_op[kt][tp] = lds_turned_channels<LY::PIECES>(lds + LY::Q_AT, tp, ch0 + 16 * kt, ln);
            }
#pragma unroll
        for (int it = 0; it < MT; ++it) {
            v4f q[KT], kk[KT];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const int ch = ch0 + 16 * kt, piece = (ch >> 3) + (ln.q >> 1), byte = 8 * (ln.q & 1);
                q[kt] = unpack4<OP>(*reinterpret_cast<const v2u*>(lds + LY::Q_AT + LdsRows<LY::PIECES>::at(16 * it + ln.n, piece) + byte));
                kk[kt] = unpack4<OP>(*reinterpret_cast<const v2u*>(lds + LY::K_AT + LdsRows<LY::PIECES>::at(16 * it + ln.n, piece) + byte));
                const float gx = gl[2 * R + 16 * it + ln.n] * s_down, gy = gl[R + 16 * it + ln.n] * d_down;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    X[kt][it][r] *= gx, Y[kt][it][r] *= gy;
                    inter += kk[kt][r] * Y[kt][it][r];
                    if constexpr (OP == OP_F16) X[kt][it][r] *= up, Y[kt][it][r] *= up;
                }
            }
#pragma unroll
            for (int tp = 0; tp < MT / 2; ++tp)
#pragma unroll
                for (int part = FP - 1; part >= 0; --part) {
                    if (tp <= it / 2) {
                        const v2u m0 = *reinterpret_cast<const v2u*>(turn.put_at + (part * LY::TILES + tix(it, 2 * tp)) * TURN16_BYTES);
                        v2u m1 = {0u, 0u};
                        if (2 * tp + 1 <= it) m1 = *reinterpret_cast<const v2u*>(turn.put_at + (part * LY::TILES + tix(it, 2 * tp + 1)) * TURN16_BYTES);
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt) X[kt][it] = mfma32<OP>(kt_op[kt][tp], v4u{m0[0], m0[1], m1[0], m1[1]}, X[kt][it]);
                    }
                    if (tp >= it / 2) {
                        v2u m0 = {0u, 0u};
                        if (2 * tp >= it) m0 = turn.get(part * LY::TILES + tix(2 * tp, it));
                        const v2u m1 = turn.get(part * LY::TILES + tix(2 * tp + 1, it));
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt) Y[kt][it] = mfma32<OP>(qt_op[kt][tp], v4u{m0[0], m0[1], m1[0], m1[1]}, Y[kt][it]);
                    }
                }
            float dot_q = 0.f, dot_k = 0.f;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const int ch = half0 + ch0 + 16 * kt + 4 * ln.q;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if constexpr (OP == OP_F16) X[kt][it][r] *= down, Y[kt][it][r] *= down;
                    dot_q += q[kt][r] * X[kt][it][r], dot_k += kk[kt][r] * Y[kt][it][r];
                }
                if constexpr (DELTA) put_rows(a.dW, times(Z[kt][it], OP == OP_F16 ? -pow2(-z_shift) : -1.f), a.H, h, ch, it);
                if constexpr (SHARED) {
                    v4f* const sum = reinterpret_cast<v4f*>(lds + LY::BYTES + 1024 * (2 * (wave * MT + it)) + 16 * (16 * ln.q + ln.n));  // the lane's own
                    if (h > h0) {
                        const v4f x = sum[0], y = sum[64];
#pragma unroll
                        for (int r = 0; r < 4; ++r) X[kt][it][r] += x[r], Y[kt][it][r] += y[r];
                    }
                    if (!last_h) sum[0] = X[kt][it], sum[64] = Y[kt][it];
                }
                if (last_h) put_rows(a.dQ, X[kt][it], H_k, hk, ch, it), put_rows(a.dK, Y[kt][it], H_k, hk, ch, it);
            }
            dot_q += __shfl_xor(dot_q, 16), dot_k += __shfl_xor(dot_k, 16);
            dot_q += __shfl_xor(dot_q, 32), dot_k += __shfl_xor(dot_k, 32);
            if (ln.q == 0) red[wave * R + 16 * it + ln.n] = dot_q, red[(WAVES + wave) * R + 16 * it + ln.n] = dot_k;
        }
        if (a.dg) {
            const float x = wave_sum(inter), y = wave_sum(s_ds);
            if (ln.q == 0 && ln.n == 0) red1[WAVES + wave] = x, red1[2 * WAVES + wave] = y;
            __syncthreads();
            if (tid < at.valid) {
                float q = 0.f, kd = 0.f, last = 0.f;
                for (int w = 0; w < WAVES; ++w) q += red[w * R + tid], kd += red[(WAVES + w) * R + tid];
                if (chunk_ends && tid == at.valid - 1) {
                    float t = 0.f;
                    for (int w = 0; w < WAVES; ++w) last += red1[WAVES + w], t += red1[2 * WAVES + w];
                    last += gl[3 * R] * t;
                }
                float* const to = a.dg + (at.row + tid) * a.H + h;
                if constexpr (HALVES == 1) *to = q - kd + last;
                else unsafeAtomicAdd(to, q - kd + last);  // two terms on a zero: the same whichever comes first
            }
        }
        if constexpr (SHARED) __syncthreads();  // M, the gates and the sums are not needed any more
    }
}

}  // namespace triinv
