// Gradient of the chunk attention (attn.hpp).  With the state S before a chunk, its values V' = U - W S, P = scale Q K^T . D and the gradient dS'
// that arrives at the state after it:
//     dV' = diag(e) K dS' + P^T dO                         e_i = exp(g_C - g_i),   dU = dV'
//     dS  = G_C dS' + scale Q^T diag(G) dO - W^T dV'       (arrives at the chunk before)
//     dW  = -dV' S^T
//     M   = scale (dO V'^T) . D
//     dQ  = scale diag(G) dO S^T + M K,   dK = diag(e) V' dS'^T + M^T Q
//     dg_i = <q_i, dQ_i> - <k_i, dK_i>,   and at the chunk's last token + <S', dS'>,  S' = G_C S + K^T diag(e) V' the state after it.
// Three kernels: the states and values again, chunk after chunk (k_chunk_attn, ATTN_RECORD); dS, last chunk first, with dU (k_attn_bwd_state);
// everything else, all chunks at once (k_attn_bwd_chunk).  The first two are the walk of the forward pass, bound by the chain from chunk
// to chunk; the states between them go through memory in fp32.  dg is the difference of large sums, so what enters it (dO S^T, V' dS'^T, M) is
// formed from all 24 bits (fp16: 22) of its fp32 operands; what only ends in 16 bits (dW) from 16 of them.
#pragma once
#include "attn.hpp"

namespace triinv {

struct AttnBwdArgs {
    const void *Q, *K, *U, *W, *dO;
    const float *g, *dstate;
    void *dQ, *dK, *dU, *dW;
    float *dg, *dstate0;
    const float *rec_state, *rec_value;  // states before the chunks, values (rec_value null: U)
    float* rec_dstate;                   // gradients at the states after the chunks
    SeqMap map;
    int64_t n_chunk;
    int H, group, d_k, d_v, C;
    float scale;
};

template <int OP, int MT, int KP, int NT, int WAVES, bool DELTA> struct BwdStateLayout {
    static constexpr int R = 16 * MT, PIECES = 4 * KP, COLS = 16 * NT * WAVES, UPIECES = COLS / 8;
    static constexpr int ROWS_BYTES = R * PIECES * 16, O_BYTES = R * UPIECES * 16;
    // Pairs of tiles of P (two tile rows, one tile column jt), tile columns one after the other.
    static constexpr int units_before(int jt)
    {
        int n = 0;
        for (int j = 0; j < jt; ++j) n += MT / 2 - j / 2;
        return n;
    }
    static constexpr int UNIT = 1024 * FULL_PARTS<OP>, P_BYTES = units_before(MT) * UNIT;
    static constexpr int PW_BYTES = DELTA && ROWS_BYTES > P_BYTES ? ROWS_BYTES : P_BYTES;  // W takes P's place when that is used up
    static constexpr int K_AT = 0, Q_AT = ROWS_BYTES, O_AT = 2 * ROWS_BYTES, P_AT = O_AT + O_BYTES, G_AT = P_AT + PW_BYTES, BYTES = G_AT + 3 * R * 4;
};

template <class LY> __device__ __forceinline__ int unit_at(int jt)  // units_before at run time
{
    int n = 0;
    for (int j = 0; j < jt; ++j) n += LY::R / 32 - j / 2;
    return n;
}

template <int OP> __device__ __forceinline__ v4f unpack4(v2u raw)
{
    v4f u;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const uint16_t x = (uint16_t)(raw[r >> 1] >> (16 * (r & 1)));
        u[r] = OP == OP_F16 ? f16_to_f32(x) : bf16_to_f32(x);
    }
    return u;
}

// acc + X^T V (channels x columns): rows of X read turned, vp the parts of V.
template <int OP, int MT, int KP, int NT, class LY>
__device__ __forceinline__ void add_turned(v4f (&S)[NT][2 * KP], const char* rows, const Parts<FULL_PARTS<OP>> (&vp)[NT], int tp, Lane ln)
{
#pragma unroll
    for (int i = 0; i < 2 * KP; ++i) {
        const int col4 = 8 * (i >> 1) + 2 * (ln.n & 3) + (i & 1), row = 32 * tp + 4 * ln.q + (ln.n >> 2);
        const v2u k0 = lds_turned<LY::PIECES>(rows, row, col4), k1 = lds_turned<LY::PIECES>(rows, row + 16, col4);
        const v4u k = {k0[0], k0[1], k1[0], k1[1]};
#pragma unroll
        for (int part = FULL_PARTS<OP> - 1; part >= 0; --part)
#pragma unroll
            for (int t = 0; t < NT; ++t) S[t][i] = mfma32<OP>(k, vp[t].u[part], S[t][i]);
    }
}

// dS from the last chunk to the first, a workgroup per head and column group as in the forward pass.
template <int OP, int MT, int KP, int NT, int WAVES, bool DELTA>
__global__ __launch_bounds__(64 * WAVES) void k_attn_bwd_state(AttnBwdArgs a)
{
    typedef BwdStateLayout<OP, MT, KP, NT, WAVES, DELTA> LY;
    constexpr int THREADS = 64 * WAVES, R = LY::R, TILES = MT * (MT + 1) / 2;
    __shared__ __attribute__((aligned(16))) char lds[LY::BYTES];
    float* const gl = reinterpret_cast<float*>(lds + LY::G_AT);  // g, exp(g_C - g), scale exp(g)
    const Lane ln = lane_id();
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned groups = (a.d_v + LY::COLS - 1) / LY::COLS;
    const unsigned b = xcd_neighbours(blockIdx.x, gridDim.x);
    const unsigned cg = b % groups, hs = b / groups;
    const int h = hs % a.H, s = hs / a.H;
    const int wg_col = cg * LY::COLS, col0 = 16 * NT * wave;
    const SeqPos sq = seq_pos(a.map, s);
    const int64_t n_chunk = (sq.len + a.C - 1) / a.C, first_id = a.map.cu_chunks ? a.map.cu_chunks[s] : s * n_chunk;
    const int hk = h / a.group, H_k = a.H / a.group;

    v4f S[NT][2 * KP];
    get_state<KP, NT>(a.dstate ? a.dstate + (int64_t)hs * a.d_k * a.d_v : nullptr, S, a.d_k, a.d_v, wg_col + col0, false, ln);

    RowLoader<LY::PIECES, R, THREADS> lq, lk, lw;
    RowLoader<LY::UPIECES, R, THREADS> lo;
    float g_row = 0.f, g_end = 0.f;
    auto request = [&](int64_t c) {
        const int64_t left = sq.len - c * a.C;
        const int valid = left < a.C ? (int)left : a.C;
        const int64_t row = sq.tok0 + c * a.C;
        lk.load(a.K, (row * H_k + hk) * a.d_k, H_k * a.d_k, a.d_k, valid, tid);
        lq.load(a.Q, (row * H_k + hk) * a.d_k, H_k * a.d_k, a.d_k, valid, tid);
        const int cols = a.d_v - wg_col;
        lo.load(a.dO, (row * a.H + h) * a.d_v + wg_col, a.H * a.d_v, cols < LY::COLS ? cols : LY::COLS, valid, tid);
        if constexpr (DELTA) lw.load(a.W, (row * a.H + h) * a.d_k, a.H * a.d_k, a.d_k, valid, tid);
        if (a.g && tid < R) {
            g_row = a.g[(row + (tid < valid ? tid : valid - 1)) * a.H + h];
            g_end = a.g[(row + valid - 1) * a.H + h];
        }
    };
    if (n_chunk > 0) request(n_chunk - 1);
    for (int64_t c = n_chunk - 1; c >= 0; --c) {
        const int64_t left = sq.len - c * a.C;
        const int valid = left < a.C ? (int)left : a.C;
        lk.store(lds + LY::K_AT, tid);
        lq.store(lds + LY::Q_AT, tid);
        lo.store(lds + LY::O_AT, tid);
        if (tid < R) {
            gl[tid] = g_row;
            gl[R + tid] = expf(g_end - g_row);
            gl[2 * R + tid] = a.scale * expf(g_row);
        }
        __syncthreads();
        // P, as operands of P^T: token rows 4 q + r, column n.
#pragma unroll
        for (int k = 0; k < (TILES + WAVES - 1) / WAVES; ++k) {
            int idx = k * WAVES + wave, it = 0;
            if (idx >= TILES) break;
            while (idx > it) idx -= ++it;
            const int jt = idx;
            v4f acc = zero4();
#pragma unroll
            for (int p = 0; p < KP; ++p)
                acc = mfma32<OP>(lds_row<LY::PIECES>(lds + LY::Q_AT, 16 * it + ln.n, 4 * p + ln.q), lds_row<LY::PIECES>(lds + LY::K_AT, 16 * jt + ln.n, 4 * p + ln.q), acc);
            const float gj = gl[16 * jt + ln.n];
            const v4f gi = *reinterpret_cast<const v4f*>(gl + 16 * it + 4 * ln.q);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[r] = jt < it || ln.n <= 4 * ln.q + r ? acc[r] * (a.scale * expf(gi[r] - gj)) : 0.f;
            char* unit = lds + LY::P_AT + LY::UNIT * (unit_at<LY>(jt) + (it >> 1) - (jt >> 1)) + 16 * (16 * ln.q + ln.n) + 8 * (it & 1);
#pragma unroll
            for (int part = 0; part < FULL_PARTS<OP>; ++part) {
                const v2u x = pack4<OP>(acc);
                *reinterpret_cast<v2u*>(unit + 1024 * part) = x;
                if (jt == it && (it & 1)) *reinterpret_cast<v2u*>(unit + 1024 * part - 8) = v2u{0u, 0u};  // the pair's other tile lies above the diagonal
                acc = minus16<OP>(acc, x);
            }
        }
        put_state<KP, NT>(a.rec_dstate + ((first_id + c) * a.H + h) * a.d_k * a.d_v, S, a.d_k, a.d_v, wg_col + col0, ln);
        Parts<FULL_PARTS<OP>> sp[NT][KP];
        const int s_shift = split_state<OP, KP, NT>(S, sp);
        const float s_down = OP == OP_F16 ? pow2(-s_shift) : 1.f;
        v4f dv[NT][MT];
#pragma unroll
        for (int tb = 0; tb < MT; ++tb) {
            v4f acc[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = zero4();
#pragma unroll
            for (int p = 0; p < KP; ++p) {
                const v4u k = lds_row<LY::PIECES>(lds + LY::K_AT, 16 * tb + ln.n, 4 * p + ln.q);
#pragma unroll
                for (int part = FULL_PARTS<OP> - 1; part >= 0; --part)
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[t] = mfma32<OP>(k, sp[t][p].u[part], acc[t]);
            }
            const v4f e = *reinterpret_cast<const v4f*>(gl + R + 16 * tb + 4 * ln.q);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) dv[t][tb][r] = acc[t][r] * (e[r] * s_down);
        }
        __syncthreads();  // P is in LDS
        v4u o[NT][MT / 2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int tp = 0; tp < MT / 2; ++tp) {
                const int row = 32 * tp + 4 * ln.q + (ln.n >> 2), col4 = (col0 >> 2) + 4 * t + (ln.n & 3);
                const v2u x = lds_turned<LY::UPIECES>(lds + LY::O_AT, row, col4), y = lds_turned<LY::UPIECES>(lds + LY::O_AT, row + 16, col4);
                o[t][tp] = v4u{x[0], x[1], y[0], y[1]};
            }
#pragma unroll
        for (int jt = 0; jt < MT; ++jt)
#pragma unroll
            for (int tp = jt / 2; tp < MT / 2; ++tp) {
                const char* unit = lds + LY::P_AT + LY::UNIT * (LY::units_before(jt) + tp - jt / 2) + 16 * (16 * ln.q + ln.n);
#pragma unroll
                for (int part = FULL_PARTS<OP> - 1; part >= 0; --part) {
                    const v4u p = *reinterpret_cast<const v4u*>(unit + 1024 * part);
#pragma unroll
                    for (int t = 0; t < NT; ++t) dv[t][jt] = mfma32<OP>(p, o[t][tp], dv[t][jt]);
                }
            }
        // dU
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int tb = 0; tb < MT; ++tb) {
                const v2u x = pack4<OP>(dv[t][tb]);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * tb + 4 * ln.q + r, col = wg_col + col0 + 16 * t + ln.n;
                    if (i < valid && col < a.d_v) static_cast<uint16_t*>(a.dU)[((sq.tok0 + c * a.C + i) * a.H + h) * a.d_v + col] = (uint16_t)(x[r >> 1] >> (16 * (r & 1)));
                }
            }
        const float decay = expf(gl[R - 1]);
        // scale G dO in place of dO, row by row; the shift that suits it and dV'.
        v4f od[NT][MT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int tb = 0; tb < MT; ++tb) {
                const v4f e = *reinterpret_cast<const v4f*>(gl + 2 * R + 16 * tb + 4 * ln.q);
                od[t][tb] = unpack4<OP>(v2u{o[t][tb / 2][2 * (tb & 1)], o[t][tb / 2][2 * (tb & 1) + 1]});
#pragma unroll
                for (int r = 0; r < 4; ++r) od[t][tb][r] *= e[r];
            }
        int shift = 0;
        if constexpr (OP == OP_F16) {
            float most = 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int tb = 0; tb < MT; ++tb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        most = fmaxf(most, fabsf(od[t][tb][r]));
                        if (DELTA) most = fmaxf(most, fabsf(dv[t][tb][r]));
                    }
            shift = f16_shift(wave_max(most));
        }
        const float up = OP == OP_F16 ? pow2(shift) : 1.f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[t][i][r] *= decay * up;
#pragma unroll
        for (int tp = 0; tp < MT / 2; ++tp) {
            Parts<FULL_PARTS<OP>> vp[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                v4f x = od[t][2 * tp], y = od[t][2 * tp + 1];
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] *= up, y[r] *= up;
                vp[t] = split_pair<OP, FULL_PARTS<OP>>(x, y);
            }
            add_turned<OP, MT, KP, NT, LY>(S, lds + LY::Q_AT, vp, tp, ln);
        }
        if constexpr (DELTA) {
            __syncthreads();  // P is used up
            lw.store(lds + LY::P_AT, tid);
            __syncthreads();
        }
        if (c > 0) request(c - 1);
        if constexpr (DELTA) {
#pragma unroll
            for (int tp = 0; tp < MT / 2; ++tp) {
                Parts<FULL_PARTS<OP>> vp[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    v4f x = dv[t][2 * tp], y = dv[t][2 * tp + 1];
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] *= -up, y[r] *= -up;
                    vp[t] = split_pair<OP, FULL_PARTS<OP>>(x, y);
                }
                add_turned<OP, MT, KP, NT, LY>(S, lds + LY::P_AT, vp, tp, ln);
            }
        }
        if constexpr (OP == OP_F16) {
            const float down = pow2(-shift);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[t][i][r] *= down;
        }
        __syncthreads();  // the rows are not needed any more
    }
    if (a.dstate0) put_state<KP, NT>(a.dstate0 + (int64_t)hs * a.d_k * a.d_v, S, a.d_k, a.d_v, wg_col + col0, ln);
}

// Everything that needs the states at both ends of a chunk: a workgroup per chunk and key head, which takes the heads that share it one
// after the other and d_v in blocks of 64 columns.  A wavefront has KT tiles of 16 channels of all tokens; the products stand turned
// (channels down, tokens across), so that a lane's four values are neighbours in memory.
template <int OP, int MT, int KT, int WAVES, bool DELTA> struct BwdChunkLayout {
    static constexpr int R = 16 * MT, PIECES = 2 * KT * WAVES, CB = 8;  // CB: pieces of a block of d_v
    static constexpr int VP = DELTA ? FULL_PARTS<OP> : 1;
    static constexpr int ROWS_BYTES = R * PIECES * 16, BLOCK = R * CB * 16;
    static constexpr int TILES = MT * (MT + 1) / 2, M_BYTES = TILES * FULL_PARTS<OP> * TURN16_BYTES;
    static constexpr int COLS_BYTES = (1 + VP + (DELTA ? 1 : 0)) * BLOCK;  // dO, V', dV'
    static constexpr int K_AT = 0, Q_AT = ROWS_BYTES, O_AT = 2 * ROWS_BYTES, V_AT = O_AT + BLOCK, DV_AT = V_AT + VP * BLOCK;
    static constexpr int M_AT = O_AT;  // when the blocks of d_v are used up
    static constexpr int G_AT = O_AT + (COLS_BYTES > M_BYTES ? COLS_BYTES : M_BYTES), RED_AT = G_AT + 3 * R * 4;
    static constexpr int BYTES = RED_AT + (2 * WAVES * R + 4 * WAVES) * 4;
};

// fp32 rows of a head on their way to LDS as 16-bit parts.
template <int OP, int N, int PIECES, int ROWS, int THREADS> struct SplitLoader {
    static constexpr int COUNT = (PIECES * ROWS + THREADS - 1) / THREADS;
    v4f v[COUNT][2];
    __device__ __forceinline__ void load(const float* base, int64_t first, int row_elems, int d, int valid, int tid)
    {
        const uint32_t stride = (uint32_t)row_elems * 4u, span = valid > 0 ? (uint32_t)(valid - 1) * stride + (uint32_t)d * 4u : 0u;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(reinterpret_cast<const char*>(base + first)), 0, span, 0x00020000);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int k = tid + i * THREADS, row = k / PIECES, piece = k % PIECES;
            const uint32_t at = row < ROWS && 8 * piece < d ? (uint32_t)row * stride + 32u * piece : 0x80000000u;
            v[i][0] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0));
            v[i][1] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 16, 0));
        }
    }
    __device__ __forceinline__ void store(char* m, int plane, int tid) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int k = tid + i * THREADS;
            if (k >= PIECES * ROWS) continue;
            const Parts<N> p = split_pair<OP, N>(v[i][0], v[i][1]);
#pragma unroll
            for (int j = 0; j < N; ++j) *reinterpret_cast<v4u*>(m + j * plane + LdsRows<PIECES>::at(k / PIECES, k % PIECES)) = p.u[j];
        }
    }
};

__device__ __forceinline__ float wave_sum(float x)
{
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}

template <int OP, int MT, int KT, int WAVES, bool DELTA>
__global__ __launch_bounds__(64 * WAVES) void k_attn_bwd_chunk(AttnBwdArgs a)
{
    typedef BwdChunkLayout<OP, MT, KT, WAVES, DELTA> LY;
    constexpr int THREADS = 64 * WAVES, R = LY::R, SHARE = (LY::TILES + WAVES - 1) / WAVES, FP = FULL_PARTS<OP>;
    __shared__ __attribute__((aligned(16))) char lds[LY::BYTES];
    float* const gl = reinterpret_cast<float*>(lds + LY::G_AT);    // g, exp(g_C - g), scale exp(g)
    float* const red = reinterpret_cast<float*>(lds + LY::RED_AT);  // sums over channels: [2][wavefront][token], then [4][wavefront]
    float* const red1 = red + 2 * WAVES * R;
    const Lane ln = lane_id();
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), H_k = a.H / a.group;
    const unsigned b = xcd_neighbours(blockIdx.x, gridDim.x);
    const int hk = b % H_k;
    const int64_t id = b / H_k;
    // which sequence and chunk
    int64_t c;
    SeqPos sq;
    if (a.map.cu_chunks) {
        int lo = 0, hi = a.map.n_seq - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (a.map.cu_chunks[mid] <= id) lo = mid;
            else hi = mid - 1;
        }
        sq = seq_pos(a.map, lo), c = id - a.map.cu_chunks[lo];
    } else {
        const int64_t cps = (a.map.Tlen + a.C - 1) / a.C;
        sq = SeqPos{id / cps * a.map.Tlen, a.map.Tlen}, c = id % cps;
    }
    const int64_t left = sq.len - c * a.C, row0 = sq.tok0 + c * a.C;
    const int valid = left < a.C ? (int)left : a.C;
    const int ch0 = 16 * KT * wave;  // this wavefront's first channel
    {
        RowLoader<LY::PIECES, R, THREADS> lk, lq;
        lk.load(a.K, (row0 * H_k + hk) * a.d_k, H_k * a.d_k, a.d_k, valid, tid);
        lq.load(a.Q, (row0 * H_k + hk) * a.d_k, H_k * a.d_k, a.d_k, valid, tid);
        lk.store(lds + LY::K_AT, tid);
        lq.store(lds + LY::Q_AT, tid);
    }
    v4f sum_q[KT][MT], sum_k[KT][MT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int it = 0; it < MT; ++it) sum_q[kt][it] = sum_k[kt][it] = zero4();

    for (int h = hk * a.group; h < (hk + 1) * a.group; ++h) {
        if (tid < R) {
            float g_row = 0.f, g_end = 0.f;
            if (a.g) g_row = a.g[(row0 + (tid < valid ? tid : valid - 1)) * a.H + h], g_end = a.g[(row0 + valid - 1) * a.H + h];
            gl[tid] = g_row, gl[R + tid] = expf(g_end - g_row), gl[2 * R + tid] = a.scale * expf(g_row);
        }
        const float* const S = a.rec_state + (id * a.H + h) * a.d_k * a.d_v;
        const float* const dS = a.rec_dstate + (id * a.H + h) * a.d_k * a.d_v;
        v4f X[KT][MT], Y[KT][MT], Z[KT][MT], M[SHARE];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int it = 0; it < MT; ++it) X[kt][it] = Y[kt][it] = Z[kt][it] = zero4();
#pragma unroll
        for (int k = 0; k < SHARE; ++k) M[k] = zero4();
        float s_ds = 0.f;
        int s_shift = 0, d_shift = 0;
        for (int v0 = 0; v0 < a.d_v; v0 += 64) {
            const int cols = a.d_v - v0 < 64 ? a.d_v - v0 : 64;
            {
                RowLoader<LY::CB, R, THREADS> lo;
                lo.load(a.dO, (row0 * a.H + h) * a.d_v + v0, a.H * a.d_v, cols, valid, tid);
                if constexpr (DELTA) {
                    RowLoader<LY::CB, R, THREADS> ld;
                    SplitLoader<OP, FP, LY::CB, R, THREADS> lv;
                    ld.load(a.dU, (row0 * a.H + h) * a.d_v + v0, a.H * a.d_v, cols, valid, tid);
                    lv.load(a.rec_value, (row0 * a.H + h) * a.d_v + v0, a.H * a.d_v, cols, valid, tid);
                    lo.store(lds + LY::O_AT, tid);
                    ld.store(lds + LY::DV_AT, tid);
                    lv.store(lds + LY::V_AT, LY::BLOCK, tid);
                } else {
                    RowLoader<LY::CB, R, THREADS> lv;
                    lv.load(a.U, (row0 * a.H + h) * a.d_v + v0, a.H * a.d_v, cols, valid, tid);
                    lo.store(lds + LY::O_AT, tid);
                    lv.store(lds + LY::V_AT, tid);
                }
            }
            __syncthreads();
            // dO V'^T, turned: value tokens down, output tokens across
#pragma unroll
            for (int k = 0; k < SHARE; ++k) {
                int idx = k * WAVES + wave, it = 0;
                if (idx >= LY::TILES) break;
                while (idx > it) idx -= ++it;
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    const v4u o = lds_row<LY::CB>(lds + LY::O_AT, 16 * it + ln.n, 4 * ks + ln.q);
#pragma unroll
                    for (int part = LY::VP - 1; part >= 0; --part)
                        M[k] = mfma32<OP>(lds_row<LY::CB>(lds + LY::V_AT + part * LY::BLOCK, 16 * idx + ln.n, 4 * ks + ln.q), o, M[k]);
                }
            }
            // S dO^T, S dV'^T and dS' V'^T
            v4f sv[KT][2][2], dsv[KT][2][2];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    const int ch = ch0 + 16 * kt + ln.n, col = v0 + 32 * ks + 8 * ln.q;
                    const bool there = ch < a.d_k && col < a.d_v;
                    const int64_t at = (int64_t)ch * a.d_v + col;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        sv[kt][ks][half] = there ? *reinterpret_cast<const v4f*>(S + at + 4 * half) : zero4();
                        dsv[kt][ks][half] = there ? *reinterpret_cast<const v4f*>(dS + at + 4 * half) : zero4();
#pragma unroll
                        for (int r = 0; r < 4; ++r) s_ds += sv[kt][ks][half][r] * dsv[kt][ks][half][r];
                    }
                }
            if constexpr (OP == OP_F16) {  // both into fp16's range, and what there is of the products with them
                float most_s = 0.f, most_d = 0.f;
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) most_s = fmaxf(most_s, fabsf(sv[kt][i >> 3][i >> 2 & 1][i & 3])), most_d = fmaxf(most_d, fabsf(dsv[kt][i >> 3][i >> 2 & 1][i & 3]));
                const int ns = f16_shift(wave_max(most_s)), nd = f16_shift(wave_max(most_d));
                const float us = pow2(ns), ud = pow2(nd), cs = v0 ? pow2(ns - s_shift) : 1.f, cd = v0 ? pow2(nd - d_shift) : 1.f;
                s_shift = ns, d_shift = nd;
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) sv[kt][i >> 3][i >> 2 & 1][i & 3] *= us, dsv[kt][i >> 3][i >> 2 & 1][i & 3] *= ud;
#pragma unroll
                    for (int it = 0; it < MT; ++it)
#pragma unroll
                        for (int r = 0; r < 4; ++r) X[kt][it][r] *= cs, Z[kt][it][r] *= cs, Y[kt][it][r] *= cd;
                }
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    const Parts<FP> sp = split_pair<OP, FP>(sv[kt][ks][0], sv[kt][ks][1]), dp = split_pair<OP, FP>(dsv[kt][ks][0], dsv[kt][ks][1]);
#pragma unroll
                    for (int it = 0; it < MT; ++it) {
                        const v4u o = lds_row<LY::CB>(lds + LY::O_AT, 16 * it + ln.n, 4 * ks + ln.q);
#pragma unroll
                        for (int part = FP - 1; part >= 0; --part) X[kt][it] = mfma32<OP>(sp.u[part], o, X[kt][it]);
                        if constexpr (DELTA) {
                            const v4u d = lds_row<LY::CB>(lds + LY::DV_AT, 16 * it + ln.n, 4 * ks + ln.q);
                            Z[kt][it] = mfma32<OP>(sp.u[1], d, Z[kt][it]);
                            Z[kt][it] = mfma32<OP>(sp.u[0], d, Z[kt][it]);
                        }
                        // parts of both sides: what is left out is below the last bit kept
#pragma unroll
                        for (int order = FP - 1; order >= 0; --order)
#pragma unroll
                            for (int j = order < LY::VP - 1 ? order : LY::VP - 1; j >= 0; --j)
                                Y[kt][it] = mfma32<OP>(dp.u[order - j], lds_row<LY::CB>(lds + LY::V_AT + j * LY::BLOCK, 16 * it + ln.n, 4 * ks + ln.q), Y[kt][it]);
                    }
                }
            __syncthreads();  // the block is used up
        }
        // M = scale (dO V'^T) . D, in parts; fp16: times a power of two that all wavefronts agree on
        float most = 0.f;
#pragma unroll
        for (int k = 0; k < SHARE; ++k) {
            int idx = k * WAVES + wave, it = 0;
            if (idx >= LY::TILES) break;
            while (idx > it) idx -= ++it;
            const float gi = gl[16 * it + ln.n];
            const v4f gj = *reinterpret_cast<const v4f*>(gl + 16 * idx + 4 * ln.q);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                M[k][r] = idx < it || 4 * ln.q + r <= ln.n ? M[k][r] * (a.scale * expf(gi - gj[r])) : 0.f;
                most = fmaxf(most, fabsf(M[k][r]));
            }
        }
        int m_shift = 0;
        if constexpr (OP == OP_F16) {
            most = wave_max(most);
            if (ln.q == 0 && ln.n == 0) red1[wave] = most;
            __syncthreads();
            for (int w = 0; w < WAVES; ++w) most = fmaxf(most, red1[w]);
            m_shift = f16_shift(most);
        }
        const Turn16 turn(reinterpret_cast<float*>(lds + LY::M_AT), ln);
#pragma unroll
        for (int k = 0; k < SHARE; ++k) {
            const int idx = k * WAVES + wave;
            if (idx >= LY::TILES) break;
            v4f m = M[k];
            if constexpr (OP == OP_F16) {
#pragma unroll
                for (int r = 0; r < 4; ++r) m[r] *= pow2(m_shift);
            }
#pragma unroll
            for (int part = 0; part < FP; ++part) {
                const v2u x = pack4<OP>(m);
                turn.put(part * LY::TILES + idx, x);
                m = minus16<OP>(m, x);
            }
        }
        __syncthreads();
        // dQ (turned): lanes are tokens i, K^T M^T over the tokens j <= i.   dK: lanes are tokens j, Q^T M over i >= j.
        const float up = OP == OP_F16 ? pow2(m_shift) : 1.f, down = OP == OP_F16 ? pow2(-m_shift) : 1.f;
        const float s_down = OP == OP_F16 ? pow2(-s_shift) : 1.f, d_down = OP == OP_F16 ? pow2(-d_shift) : 1.f;
        float inter = 0.f;
#pragma unroll
        for (int it = 0; it < MT; ++it) {
            float dot_q = 0.f, dot_k = 0.f;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                v4f x = X[kt][it], y = Y[kt][it];
                const float gx = gl[2 * R + 16 * it + ln.n] * s_down, gy = gl[R + 16 * it + ln.n] * d_down;
                const int ch = ch0 + 16 * kt, piece = (ch >> 3) + (ln.q >> 1), byte = 8 * (ln.q & 1);
                const v4f q = unpack4<OP>(*reinterpret_cast<const v2u*>(lds + LY::Q_AT + LdsRows<LY::PIECES>::at(16 * it + ln.n, piece) + byte));
                const v4f kk = unpack4<OP>(*reinterpret_cast<const v2u*>(lds + LY::K_AT + LdsRows<LY::PIECES>::at(16 * it + ln.n, piece) + byte));
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[r] *= gx, y[r] *= gy;
                    inter += kk[r] * y[r];
                    if constexpr (OP == OP_F16) x[r] *= up, y[r] *= up;
                }
#pragma unroll
                for (int tp = 0; tp < MT / 2; ++tp) {
                    const int row = 32 * tp + 4 * ln.q + (ln.n >> 2), col4 = (ch >> 2) + (ln.n & 3);
                    if (tp <= it / 2) {
                        const v2u k0 = lds_turned<LY::PIECES>(lds + LY::K_AT, row, col4), k1 = lds_turned<LY::PIECES>(lds + LY::K_AT, row + 16, col4);
#pragma unroll
                        for (int part = FP - 1; part >= 0; --part) {
                            const v2u m0 = *reinterpret_cast<const v2u*>(turn.put_at + (part * LY::TILES + tix(it, 2 * tp)) * TURN16_BYTES);
                            v2u m1 = {0u, 0u};
                            if (2 * tp + 1 <= it) m1 = *reinterpret_cast<const v2u*>(turn.put_at + (part * LY::TILES + tix(it, 2 * tp + 1)) * TURN16_BYTES);
                            x = mfma32<OP>(v4u{k0[0], k0[1], k1[0], k1[1]}, v4u{m0[0], m0[1], m1[0], m1[1]}, x);
                        }
                    }
                    if (tp >= it / 2) {
                        const v2u q0 = lds_turned<LY::PIECES>(lds + LY::Q_AT, row, col4), q1 = lds_turned<LY::PIECES>(lds + LY::Q_AT, row + 16, col4);
#pragma unroll
                        for (int part = FP - 1; part >= 0; --part) {
                            v2u m0 = {0u, 0u};
                            if (2 * tp >= it) m0 = turn.get(part * LY::TILES + tix(2 * tp, it));
                            const v2u m1 = turn.get(part * LY::TILES + tix(2 * tp + 1, it));
                            y = mfma32<OP>(v4u{q0[0], q0[1], q1[0], q1[1]}, v4u{m0[0], m0[1], m1[0], m1[1]}, y);
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if constexpr (OP == OP_F16) x[r] *= down, y[r] *= down;
                    dot_q += q[r] * x[r], dot_k += kk[r] * y[r];
                    sum_q[kt][it][r] += x[r], sum_k[kt][it][r] += y[r];
                }
                const int i = 16 * it + ln.n;
                if constexpr (DELTA) {
                    v4f z = Z[kt][it];
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[r] *= -s_down;
                    if (i < valid && ch + 4 * ln.q < a.d_k) *reinterpret_cast<v2u*>(static_cast<uint16_t*>(a.dW) + ((row0 + i) * a.H + h) * a.d_k + ch + 4 * ln.q) = pack4<OP>(z);
                }
            }
            dot_q += __shfl_xor(dot_q, 16), dot_k += __shfl_xor(dot_k, 16);
            dot_q += __shfl_xor(dot_q, 32), dot_k += __shfl_xor(dot_k, 32);
            if (ln.q == 0) red[wave * R + 16 * it + ln.n] = dot_q, red[(WAVES + wave) * R + 16 * it + ln.n] = dot_k;
        }
        if (a.dg) {
            const float x = wave_sum(inter), y = wave_sum(s_ds);
            if (ln.q == 0 && ln.n == 0) red1[wave] = x, red1[WAVES + wave] = y;
            __syncthreads();
            if (tid < valid) {
                float q = 0.f, k = 0.f, last = 0.f;
                for (int w = 0; w < WAVES; ++w) q += red[w * R + tid], k += red[(WAVES + w) * R + tid];
                if (tid == valid - 1) {
                    float t = 0.f;
                    for (int w = 0; w < WAVES; ++w) last += red1[w], t += red1[WAVES + w];
                    last += expf(gl[R - 1]) * t;
                }
                a.dg[(row0 + tid) * a.H + h] = q - k + last;
            }
        }
        __syncthreads();  // M and the sums are not needed any more
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int it = 0; it < MT; ++it) {
            const int i = 16 * it + ln.n, ch = ch0 + 16 * kt + 4 * ln.q;
            if (i >= valid || ch >= a.d_k) continue;
            const int64_t at = ((row0 + i) * H_k + hk) * a.d_k + ch;
            *reinterpret_cast<v2u*>(static_cast<uint16_t*>(a.dQ) + at) = pack4<OP>(sum_q[kt][it]);
            *reinterpret_cast<v2u*>(static_cast<uint16_t*>(a.dK) + at) = pack4<OP>(sum_k[kt][it]);
        }
}

}  // namespace triinv
