// Attention over chunks of C tokens with one decay per head: what a layer computes from the solved right-hand sides.
//
// Per head, chunk after chunk, with the state S (d_k x d_v) before the chunk, G = exp(g), D_ij = exp(g_i - g_j) for i >= j:
//     V' = U - W S                                     (plain decay, no W: V' = U)
//     O  = scale (diag(G) Q S + (Q K^T . D) V')
//     S <- G_C S + K^T diag(exp(g_C - g)) V'
// A workgroup takes some columns of one head through all its chunks (or those of its segment), a wavefront 16 NT of them, S in its
// registers; what all columns share (rows of Q, K, W; the tiles of (Q K^T . D)^T, formed once a workgroup, a share per wavefront)
// goes through LDS.  Rows of the next chunk are requested before one is computed.
#pragma once
#include "attn_ops.hpp"

namespace triinv {

struct AttnArgs {
    const void *Q, *K, *U, *W;
    const float *g, *state;
    void* O;
    float* final_state;
    // Segments of the sequences (a workgroup each), where there are too few heads: what a segment adds to a state and what it does to
    // the one before it, or the states before the segments from them.
    float *seg_state, *seg_trans, *seg_decay;
    float *rec_state, *rec_value;  // for the gradient: the states before the chunks [chunk][H][d_k][d_v], and V' [token][H][d_v] where it is not U
    SeqMap map;
    int H, group, d_k, d_v, C;  // group: heads that share a key head
    int n_seg;
    float scale;
};

// Chunks of segment `seg` of a sequence of n.
__device__ __forceinline__ void segment_chunks(int64_t n, int n_seg, int seg, int64_t& first, int64_t& last)
{
    const int64_t per = (n + n_seg - 1) / n_seg;
    first = per * seg < n ? per * seg : n;
    last = first + per < n ? first + per : n;
}

// Channel of row `row` (0..15) of state tile t (attn_ops.hpp).
__device__ __forceinline__ int state_channel(int t, int row) { return 32 * (t >> 1) + 8 * (row >> 2) + 4 * (t & 1) + (row & 3); }

// State tiles of a wavefront's columns from `col0` on, from and to memory [d_k][d_v].  No address: zeros, or the identity.
template <int KP, int NT> __device__ __forceinline__ void get_state(const float* from, v4f (&S)[NT][2 * KP], int d_k, int d_v, int col0, bool identity, Lane ln)
{
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int ch = state_channel(i, 4 * ln.q + r), col = col0 + 16 * t + ln.n;
                S[t][i][r] = from && ch < d_k && col < d_v ? from[(int64_t)ch * d_v + col] : identity && ch == col ? 1.f : 0.f;
            }
}
template <int KP, int NT> __device__ __forceinline__ void put_state(float* to, const v4f (&S)[NT][2 * KP], int d_k, int d_v, int col0, Lane ln)
{
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int ch = state_channel(i, 4 * ln.q + r), col = col0 + 16 * t + ln.n;
                if (ch < d_k && col < d_v) to[(int64_t)ch * d_v + col] = S[t][i][r];
            }
}

// MT tiles of 16 token rows, KP pairs of tiles of 16 channels, NT column tiles a wavefront, WAVES wavefronts.
template <int OP, int MT, int KP, int NT, int WAVES, bool DELTA> struct AttnLayout {
    static constexpr int R = 16 * MT, PIECES = 4 * KP, COLS = 16 * NT * WAVES, UPIECES = COLS / 8;
    static constexpr int ROWS_BYTES = R * PIECES * 16, U_BYTES = R * UPIECES * 16;
    static constexpr int units_before(int it) { return (it / 2) * (it / 2 + 1) + (it % 2) * (it / 2 + 1); }  // pairs of tiles of P^T before tile column it
    static constexpr int P_UNITS = units_before(MT), P_BYTES = P_UNITS * 2048;
    static constexpr int K_AT = 0, Q_AT = ROWS_BYTES, W_AT = 2 * ROWS_BYTES, U_AT = (DELTA ? 3 : 2) * ROWS_BYTES, P_AT = U_AT + U_BYTES, G_AT = P_AT + P_BYTES;
    static constexpr int BYTES = G_AT + 3 * R * 4;
};

// What a wavefront keeps of one chunk's rows of its columns.
template <int OP, int MT, int KP, int NT, bool DELTA> struct ChunkValues {
    v4f v[NT][MT];  // V', in units of 2^-shift
    int shift;      // fp16: V' = v as it is; its parts are of v 2^shift
};

// V' of a chunk: U from LDS, minus W S.  sp: parts of S 2^s_shift.
template <int OP, int MT, int KP, int NT, bool DELTA, class LY>
__device__ __forceinline__ void chunk_values(ChunkValues<OP, MT, KP, NT, DELTA>& c, const char* lds, const Parts<FULL_PARTS<OP>> (&sp)[NT][KP], int s_shift, int col0, Lane ln)
{
    const float down = OP == OP_F16 ? pow2(-s_shift) : 1.f;
#pragma unroll
    for (int tb = 0; tb < MT; ++tb) {
        v4f acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = zero4();
        if constexpr (DELTA) {
#pragma unroll
            for (int p = 0; p < KP; ++p) {
                const v4u w = lds_row<LY::PIECES>(lds + LY::W_AT, 16 * tb + ln.n, 4 * p + ln.q);
#pragma unroll
                for (int part = FULL_PARTS<OP> - 1; part >= 0; --part)
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[t] = mfma32<OP>(w, sp[t][p].u[part], acc[t]);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const v2u raw = lds_turned<LY::UPIECES>(lds + LY::U_AT, 16 * tb + 4 * ln.q + (ln.n >> 2), (col0 >> 2) + 4 * t + (ln.n & 3));
            v4f u;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint16_t x = (uint16_t)(raw[r >> 1] >> (16 * (r & 1)));
                u[r] = OP == OP_F16 ? f16_to_f32(x) : bf16_to_f32(x);
            }
            if constexpr (DELTA) {
#pragma unroll
                for (int r = 0; r < 4; ++r) u[r] -= OP == OP_F16 ? acc[t][r] * down : acc[t][r];
            }
            c.v[t][tb] = u;
        }
    }
    c.shift = 0;
    if constexpr (OP == OP_F16) {
        float most = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int tb = 0; tb < MT; ++tb)
#pragma unroll
                for (int r = 0; r < 4; ++r) most = fmaxf(most, fabsf(c.v[t][tb][r]));
        c.shift = f16_shift(wave_max(most));
    }
}

// S <- G_C S + K^T diag(e) V'.  e: exp(g_C - g) of the chunk's rows, in LDS.
template <int OP, int MT, int KP, int NT, bool DELTA, class LY>
__device__ __forceinline__ void chunk_state(v4f (&S)[NT][2 * KP], const ChunkValues<OP, MT, KP, NT, DELTA>& c, const char* lds, const float* e, float decay, Lane ln)
{
    const float up = OP == OP_F16 ? pow2(c.shift) : 1.f, a = decay * up;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][i][r] *= a;
#pragma unroll
    for (int tp = 0; tp < MT / 2; ++tp) {
        Parts<FULL_PARTS<OP>> vp[NT];
        const v4f e0 = *reinterpret_cast<const v4f*>(e + 32 * tp + 4 * ln.q), e1 = *reinterpret_cast<const v4f*>(e + 32 * tp + 16 + 4 * ln.q);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            v4f x = c.v[t][2 * tp], y = c.v[t][2 * tp + 1];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] *= e0[r] * up, y[r] *= e1[r] * up;
            vp[t] = split_pair<OP, FULL_PARTS<OP>>(x, y);
        }
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i) {
            const int col4 = 8 * (i >> 1) + 2 * (ln.n & 3) + (i & 1), row = 32 * tp + 4 * ln.q + (ln.n >> 2);
            const v2u k0 = lds_turned<LY::PIECES>(lds + LY::K_AT, row, col4), k1 = lds_turned<LY::PIECES>(lds + LY::K_AT, row + 16, col4);
            const v4u k = {k0[0], k0[1], k1[0], k1[1]};
#pragma unroll
            for (int part = FULL_PARTS<OP> - 1; part >= 0; --part)
#pragma unroll
                for (int t = 0; t < NT; ++t) S[t][i] = mfma32<OP>(k, vp[t].u[part], S[t][i]);
        }
    }
    if constexpr (OP == OP_F16) {
        const float down = pow2(-c.shift);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[t][i][r] *= down;
    }
}

// Parts of S, fp16: of S 2^shift.
template <int OP, int KP, int NT> __device__ __forceinline__ int split_state(const v4f (&S)[NT][2 * KP], Parts<FULL_PARTS<OP>> (&sp)[NT][KP])
{
    int shift = 0;
    float up = 1.f;
    if constexpr (OP == OP_F16) {
        float most = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) most = fmaxf(most, fabsf(S[t][i][r]));
        shift = f16_shift(wave_max(most));
        up = pow2(shift);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int p = 0; p < KP; ++p) {
            v4f x = S[t][2 * p], y = S[t][2 * p + 1];
            if constexpr (OP == OP_F16) {
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] *= up, y[r] *= up;
            }
            sp[t][p] = split_pair<OP, FULL_PARTS<OP>>(x, y);
        }
    return shift;
}

// The tiles of (scale Q K^T . D)^T that this wavefront forms, two parts each, into LDS as operands.
template <int OP, int MT, int KP, int WAVES, class LY>
__device__ __forceinline__ void chunk_scores(char* lds, const float* gl, float scale, int wave, Lane ln)
{
#pragma unroll
    for (int k = 0; k < (MT * (MT + 1) / 2 + WAVES - 1) / WAVES; ++k) {
        int idx = k * WAVES + wave, it = 0;
        if (idx >= MT * (MT + 1) / 2) break;
        while (idx > it) idx -= ++it;  // tile row idx <= it of tile column it
        const int jt = idx;
        v4f acc = zero4();
#pragma unroll
        for (int p = 0; p < KP; ++p)
            acc = mfma32<OP>(lds_row<LY::PIECES>(lds + LY::K_AT, 16 * jt + ln.n, 4 * p + ln.q), lds_row<LY::PIECES>(lds + LY::Q_AT, 16 * it + ln.n, 4 * p + ln.q), acc);
        const float gi = gl[16 * it + ln.n];
        const v4f gj = *reinterpret_cast<const v4f*>(gl + 16 * jt + 4 * ln.q);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] = jt < it || 4 * ln.q + r <= ln.n ? acc[r] * (scale * __expf(gi - gj[r])) : 0.f;
        const v2u hi = pack4<OP>(acc), lo = pack4<OP>(minus16<OP>(acc, hi));
        char* unit = lds + LY::P_AT + 2048 * (LY::units_before(it) + (jt >> 1)) + 16 * (16 * ln.q + ln.n) + 8 * (jt & 1);
        *reinterpret_cast<v2u*>(unit) = hi;
        *reinterpret_cast<v2u*>(unit + 1024) = lo;
        if (jt == it && !(it & 1)) {  // the pair's other tile lies behind the diagonal
            *reinterpret_cast<v2u*>(unit + 8) = v2u{0u, 0u};
            *reinterpret_cast<v2u*>(unit + 1024 + 8) = v2u{0u, 0u};
        }
    }
}

// ATTN_OUT: the outputs and the final state.  ATTN_SEGMENT: what a segment adds to a state (column groups of d_v) and, with W, what it does to
// the one before it: the same recursion from the identity with U = 0 (column groups of d_k behind them).  ATTN_RECORD: the states before
// the chunks and the chunks' values, for the gradient.
enum : int { ATTN_OUT = 0, ATTN_SEGMENT = 1, ATTN_RECORD = 2 };
template <int OP, int MT, int KP, int NT, int WAVES, bool DELTA, int MODE>
__global__ __launch_bounds__(64 * WAVES) void k_chunk_attn(AttnArgs a)
{
    typedef AttnLayout<OP, MT, KP, NT, WAVES, DELTA> LY;
    constexpr bool OUT = MODE == ATTN_OUT, SEGMENT = MODE == ATTN_SEGMENT;
    constexpr int THREADS = 64 * WAVES, R = LY::R;
    __shared__ __attribute__((aligned(16))) char lds[LY::BYTES];
    float* const gl = reinterpret_cast<float*>(lds + LY::G_AT);  // g, exp(g_C - g), scale exp(g)
    const Lane ln = lane_id();
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    const unsigned groups_v = (a.d_v + LY::COLS - 1) / LY::COLS, groups = groups_v + (SEGMENT && DELTA ? (a.d_k + LY::COLS - 1) / LY::COLS : 0);
    const unsigned b = xcd_neighbours(blockIdx.x, gridDim.x);
    const unsigned cg = b % groups, hs = b / groups;
    const int seg = blockIdx.y;
    const int h = hs % a.H, s = hs / a.H;
    const bool trans = SEGMENT && cg >= groups_v;
    const int d_v = trans ? a.d_k : a.d_v;
    const int wg_col = (trans ? cg - groups_v : cg) * LY::COLS, col0 = 16 * NT * wave;  // of the workgroup, of the wavefront in it
    const SeqPos sq = seq_pos(a.map, s);
    const int64_t n_chunk = (sq.len + a.C - 1) / a.C;
    int64_t c0, c1;
    segment_chunks(n_chunk, a.n_seg, seg, c0, c1);
    const int hk = h / a.group, H_k = a.H / a.group;

    v4f S[NT][2 * KP];
    const float* from = !SEGMENT ? (seg == 0 ? a.state : a.seg_state + (int64_t)(seg - 1) * a.map.n_seq * a.H * a.d_k * a.d_v) : nullptr;
    get_state<KP, NT>(from ? from + (int64_t)hs * a.d_k * a.d_v : nullptr, S, a.d_k, d_v, wg_col + col0, trans, ln);

    RowLoader<LY::PIECES, R, THREADS> lq, lk, lw;
    RowLoader<LY::UPIECES, R, THREADS> lu;
    float g_row = 0.f, g_end = 0.f;
    auto request = [&](int64_t c) {
        const int64_t left = sq.len - c * a.C;
        const int valid = left < a.C ? (int)left : a.C;
        const int64_t row = sq.tok0 + c * a.C;
        lk.load(a.K, (row * H_k + hk) * a.d_k, H_k * a.d_k, a.d_k, valid, tid);
        if constexpr (DELTA) lw.load(a.W, (row * a.H + h) * a.d_k, a.H * a.d_k, a.d_k, valid, tid);
        const int cols = a.d_v - wg_col;
        lu.load(a.U, (row * a.H + h) * a.d_v + wg_col, a.H * a.d_v, cols < LY::COLS ? cols : LY::COLS, trans ? 0 : valid, tid);
        if constexpr (OUT) lq.load(a.Q, (row * H_k + hk) * a.d_k, H_k * a.d_k, a.d_k, valid, tid);
        if (a.g && tid < R) {
            g_row = a.g[(row + (tid < valid ? tid : valid - 1)) * a.H + h];
            g_end = a.g[(row + valid - 1) * a.H + h];
        }
    };
    float total = 0.f;
    if (c0 < c1) request(c0);
    for (int64_t c = c0; c < c1; ++c) {
        const int64_t left = sq.len - c * a.C;
        const int valid = left < a.C ? (int)left : a.C;
        lk.store(lds + LY::K_AT, tid);
        if constexpr (OUT) lq.store(lds + LY::Q_AT, tid);
        if constexpr (DELTA) lw.store(lds + LY::W_AT, tid);
        lu.store(lds + LY::U_AT, tid);
        if (tid < R) {
            gl[tid] = g_row;
            gl[R + tid] = expf(g_end - g_row);
            gl[2 * R + tid] = a.scale * expf(g_row);
        }
        __syncthreads();
        if (c + 1 < c1) request(c + 1);
        if constexpr (OUT) chunk_scores<OP, MT, KP, WAVES, LY>(lds, gl, a.scale, wave, ln);

        const float g_last = gl[R - 1], decay = expf(g_last);
        total += g_last;
        if constexpr (MODE == ATTN_RECORD) {
            const int64_t id = (a.map.cu_chunks ? a.map.cu_chunks[s] : s * n_chunk) + c;
            put_state<KP, NT>(a.rec_state + (id * a.H + h) * a.d_k * a.d_v, S, a.d_k, a.d_v, wg_col + col0, ln);
        }
        Parts<FULL_PARTS<OP>> sp[NT][KP];
        int s_shift = 0;
        if constexpr (DELTA || OUT) s_shift = split_state<OP, KP, NT>(S, sp);
        ChunkValues<OP, MT, KP, NT, DELTA> cv;
        chunk_values<OP, MT, KP, NT, DELTA, LY>(cv, lds, sp, s_shift, col0, ln);
        if constexpr (MODE == ATTN_RECORD && DELTA) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int tb = 0; tb < MT; ++tb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int i = 16 * tb + 4 * ln.q + r, col = wg_col + col0 + 16 * t + ln.n;
                        if (i < valid && col < a.d_v) a.rec_value[((sq.tok0 + c * a.C + i) * a.H + h) * a.d_v + col] = cv.v[t][tb][r];
                    }
        }
        chunk_state<OP, MT, KP, NT, DELTA, LY>(S, cv, lds, gl + R, decay, ln);
        if constexpr (OUT) __syncthreads();  // the scores are in LDS
        if constexpr (OUT) {
            Parts<2> vp[NT][MT / 2];
            const float up = OP == OP_F16 ? pow2(cv.shift) : 1.f, down = OP == OP_F16 ? pow2(-cv.shift) : 1.f;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int tp = 0; tp < MT / 2; ++tp) {
                    v4f x = cv.v[t][2 * tp], y = cv.v[t][2 * tp + 1];
                    if constexpr (OP == OP_F16) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[r] *= up, y[r] *= up;
                    }
                    vp[t][tp] = split_pair<OP, 2>(x, y);
                }
            const float across = OP == OP_F16 ? pow2(cv.shift - s_shift) : 1.f;
#pragma unroll
            for (int it = 0; it < MT; ++it) {
                v4f acc[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = zero4();
#pragma unroll
                for (int p = 0; p < KP; ++p) {
                    const v4u q = lds_row<LY::PIECES>(lds + LY::Q_AT, 16 * it + ln.n, 4 * p + ln.q);
#pragma unroll
                    for (int part = 1; part >= 0; --part)
#pragma unroll
                        for (int t = 0; t < NT; ++t) acc[t] = mfma32<OP>(sp[t][p].u[part], q, acc[t]);
                }
                const float gate = gl[2 * R + 16 * it + ln.n] * across;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[t][r] *= gate;
#pragma unroll
                for (int tp = 0; tp <= it / 2; ++tp) {
                    const char* unit = lds + LY::P_AT + 2048 * (LY::units_before(it) + tp) + 16 * (16 * ln.q + ln.n);
                    const v4u hi = *reinterpret_cast<const v4u*>(unit), lo = *reinterpret_cast<const v4u*>(unit + 1024);
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[t] = mfma32<OP>(vp[t][tp].u[0], lo, acc[t]);
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[t] = mfma32<OP>(vp[t][tp].u[1], hi, acc[t]);
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[t] = mfma32<OP>(vp[t][tp].u[0], hi, acc[t]);
                }
                const int i = 16 * it + ln.n;
                if (i < valid) {
                    uint16_t* o = static_cast<uint16_t*>(a.O) + ((sq.tok0 + c * a.C + i) * a.H + h) * a.d_v + wg_col + col0 + 4 * ln.q;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if constexpr (OP == OP_F16) {
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[t][r] *= down;
                        }
                        if (wg_col + col0 + 16 * t + 4 * ln.q < a.d_v) *reinterpret_cast<v2u*>(o + 16 * t) = pack4<OP>(acc[t]);
                    }
                }
            }
        }
        __syncthreads();  // the rows are not needed any more
    }

    if (!SEGMENT && seg != a.n_seg - 1) return;
    float* to = !SEGMENT ? a.final_state : trans ? a.seg_trans : a.seg_state;
    if (!to) return;
    if (SEGMENT) to += (int64_t)seg * a.map.n_seq * a.H * a.d_k * d_v;
    put_state<KP, NT>(to + (int64_t)hs * a.d_k * d_v, S, a.d_k, d_v, wg_col + col0, ln);
    if (SEGMENT && !DELTA && cg == 0 && tid == 0) a.seg_decay[(int64_t)seg * a.map.n_seq * a.H + hs] = expf(total);
}

// States before the segments, in place of what the segments add: S <- M_seg S + L_seg from the sequence's initial state.  M and S as
// three bf16 parts each, the six products that matter.
template <int KP, int WAVES, bool DELTA> __global__ __launch_bounds__(64 * WAVES) void k_attn_join(AttnArgs a)
{
    constexpr int COLS = 16 * WAVES;
    const Lane ln = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned groups = (a.d_v + COLS - 1) / COLS, cg = blockIdx.x % groups, hs = blockIdx.x / groups;
    const int col = cg * COLS + 16 * wave + ln.n;
    const int64_t heads = (int64_t)a.map.n_seq * a.H;
    const bool mine = col < a.d_v;
    v4f S[2 * KP];
#pragma unroll
    for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int ch = state_channel(i, 4 * ln.q + r);
            S[i][r] = a.state && mine && ch < a.d_k ? a.state[((int64_t)hs * a.d_k + ch) * a.d_v + col] : 0.f;
        }
    for (int seg = 0; seg + 1 < a.n_seg; ++seg) {
        float* const L = a.seg_state + (seg * heads + hs) * a.d_k * a.d_v;
        v4f next[2 * KP];
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int ch = state_channel(i, 4 * ln.q + r);
                next[i][r] = mine && ch < a.d_k ? L[(int64_t)ch * a.d_v + col] : 0.f;
            }
        if constexpr (DELTA) {
            const float* const M = a.seg_trans + (seg * heads + hs) * a.d_k * a.d_k;
            Parts<3> sp[KP];
#pragma unroll
            for (int p = 0; p < KP; ++p) sp[p] = split_pair<OP_BF16, 3>(S[2 * p], S[2 * p + 1]);
#pragma unroll
            for (int i = 0; i < 2 * KP; ++i) {
                const int ch = state_channel(i, ln.n);
#pragma unroll
                for (int p = 0; p < KP; ++p) {
                    v4f x = zero4(), y = zero4();
                    if (ch < a.d_k && 32 * p < a.d_k) {
                        const float* m = M + (int64_t)ch * a.d_k + 32 * p + 8 * ln.q;
                        x = *reinterpret_cast<const v4f*>(m), y = *reinterpret_cast<const v4f*>(m + 4);
                    }
                    const Parts<3> mp = split_pair<OP_BF16, 3>(x, y);
                    next[i] = mfma32<OP_BF16>(mp.u[2], sp[p].u[0], next[i]);
                    next[i] = mfma32<OP_BF16>(mp.u[0], sp[p].u[2], next[i]);
                    next[i] = mfma32<OP_BF16>(mp.u[1], sp[p].u[1], next[i]);
                    next[i] = mfma32<OP_BF16>(mp.u[1], sp[p].u[0], next[i]);
                    next[i] = mfma32<OP_BF16>(mp.u[0], sp[p].u[1], next[i]);
                    next[i] = mfma32<OP_BF16>(mp.u[0], sp[p].u[0], next[i]);
                }
            }
        } else {
            const float decay = a.seg_decay[seg * heads + hs];
#pragma unroll
            for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) next[i][r] += decay * S[i][r];
        }
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i) {
            S[i] = next[i];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int ch = state_channel(i, 4 * ln.q + r);
                if (mine && ch < a.d_k) L[(int64_t)ch * a.d_v + col] = S[i][r];
            }
        }
    }
}

}  // namespace triinv
