// Attention over chunks of C tokens with one decay per head: what a layer computes from the solved right-hand sides.
//
// Per head, chunk after chunk, with the state S (d_k x d_v) before the chunk, G = exp(g), D_ij = exp(g_i - g_j) for i >= j:
//     V' = U - W S                                     (plain decay, no W: V' = U)
//     O  = scale (diag(G) Q S + (Q K^T . D) V')
//     S <- G_C S + K^T diag(exp(g_C - g)) V'
// Everything but W S may be taken in smaller steps: a chunk of 128 goes in two of 64 tokens, with g counted from the step's beginning,
// and W S with the state before the chunk for both.
//
// A workgroup takes 64 columns of one head through all its steps (or those of its segment).  Four wavefronts carry the recursion, 16 columns each,
// S in their registers; four others form the scores and the outputs, one product behind.  Each brings the rows of the next step that it uses to LDS:
//     first half     W S, V'                                         scores V' and the store of the step before, Q S
//     second half    K^T V', the new S and its parts; W and U        K and Q, scores
// The halves are separated by barriers, across which V' and the parts of S go through LDS.  A wavefront per SIMD that waits needs another to take its place,
// which is what the second four are for.
//
// Bound by the chain of a step: d_k = d_v = 128 takes 3.3 thousand cycles of matrix instructions a SIMD and step of 64 tokens, half of them for the second and
// third parts of S (products of fp32 states), and a step lasts 7: of a SIMD's 204 of them 124 stand in the one wavefront of the recursion, behind each other and behind two splits
// of V', and the matrix unit works half of the time.  A chip full of it runs at 1.6 to 1.9 GHz.  Measured: 8 x 8192 tokens, 16 heads, bf16 447 to 473 us from card to card (the
// bytes at the rate of a copy: 246); 48 packed sequences of 1100 on average, 4 heads, fp16, no W 105 to 107 (44).
// Decays of scores by __expf: |g_i - g_j| 2^-24 of the value and a bit, which the difference in its exponent is no better than.
#pragma once

#include <type_traits>

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
    float* seg_first;  // a copy of `state` for the first segment, which runs beside the last one that writes over it; or null
    float *rec_state, *rec_value;  // for the gradient: the states before the steps [step][H], and V' where it is not U, [first token of the step][H], as put_turned leaves them
    float* rec_dg;                 // zeroed where two workgroups add to it
    SeqMap map;
    int H, group, d_k, d_v, C;  // group: heads that share a key head
    int n_seg;
    float scale;
};

// Chunks of segment `seg` of a sequence of n.
__device__ __forceinline__ void segment_chunks(int64_t n, int n_seg, int seg, int64_t& first, int64_t& last)
{
    const int64_t per = ((uint32_t)n + n_seg - 1u) / (uint32_t)n_seg;  // (a sequence of 2^31 chunks fits in no memory)
    first = per * seg < n ? per * seg : n;
    last = first + per < n ? first + per : n;
}

// (By value: the cast of an element of a vector where it stands takes the vector's first.)
__device__ __forceinline__ uint32_t bits(float x) { return __builtin_bit_cast(uint32_t, x); }
// State tiles of a wavefront's 16 columns from `col0` on, from and to memory [d_k][d_v].  No address: zeros, or the identity.
template <int KP> __device__ __forceinline__ void get_state(const float* from, v4f (&S)[2 * KP], int d_k, int d_v, int col0, bool identity, Lane ln)
{
#pragma unroll
    for (int i = 0; i < 2 * KP; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int ch = state_channel(i, 4 * ln.q + r), col = col0 + ln.n;
            S[i][r] = from && ch < d_k && col < d_v ? from[(int64_t)ch * d_v + col] : identity && ch == col ? 1.f : 0.f;
        }
}
// (Buffer stores: what belongs to every lane of an address goes as a scalar, columns that are not there lie outside the buffer.)
template <int KP> __device__ __forceinline__ void put_state(float* to, const v4f (&S)[2 * KP], int d_k, int d_v, int col0, Lane ln)
{
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(to, 0, (uint32_t)d_k * d_v * 4u, 0x00020000);
    const uint32_t at = col0 + ln.n < d_v ? (uint32_t)(8 * ln.q * d_v + col0 + ln.n) * 4u : 0x80000000u;
#pragma unroll
    for (int i = 0; i < 2 * KP; ++i) {
        if (32 * (i >> 1) >= d_k) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r) __builtin_amdgcn_raw_buffer_store_b32(bits(S[i][r]), rsrc, at, (state_channel(i, 0) + r) * d_v * 4, 0);
    }
}

// Largest magnitude of some tiles.
template <int N> __device__ __forceinline__ float most_of(const v4f (&x)[N])
{
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) most = fmaxf(most, fabsf(x[i][r]));
    return most;
}
__device__ __forceinline__ v4f times(v4f x, float a)
{
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] *= a;
    return x;
}

// S + X^T V (channels x columns): rows of X read turned, vp the parts of V.  Here as everywhere, products that add to one tile are kept apart by those of
// other tiles, so that none waits for the one before it.
template <int OP, int MT, int KP>
__device__ __forceinline__ void add_turned(v4f (&S)[2 * KP], const char* rows, const Parts<FULL_PARTS<OP>> (&vp)[MT / 2], Lane ln)
{
    // the next KP tiles are requested before one is used
    v4u k[2][KP];
    auto rows_of = [&](int stage) {
#pragma unroll
        for (int i = 0; i < KP; ++i) k[stage & 1][i] = lds_turned_tile<4 * KP>(rows, stage >> 1, KP * (stage & 1) + i, ln);
    };
    rows_of(0);
#pragma unroll
    for (int stage = 0; stage < MT; ++stage) {
        if (stage + 1 < MT) rows_of(stage + 1);
        in_order();
#pragma unroll
        for (int part = FULL_PARTS<OP> - 1; part >= 0; --part)
#pragma unroll
            for (int i = 0; i < KP; ++i) S[KP * (stage & 1) + i] = mfma32<OP>(k[stage & 1][i], vp[stage >> 1].u[part], S[KP * (stage & 1) + i]);
    }
}

// v = X S (tokens x columns), sp the parts of S: rows of X, the next pair's requested before one is used; `also` follows each pair's products.
template <int OP, int MT, int KP, class Also> __device__ __forceinline__ void rows_times(v4f (&v)[MT], const char* rows, const Parts<FULL_PARTS<OP>> (&sp)[KP], Lane ln, Also also)
{
    v4u w[2][MT];
    auto rows_of = [&](int p) {
#pragma unroll
        for (int tb = 0; tb < MT; ++tb) w[p & 1][tb] = lds_row<4 * KP>(rows, 16 * tb + ln.n, 4 * p + ln.q);
    };
    rows_of(0);
#pragma unroll
    for (int tb = 0; tb < MT; ++tb) v[tb] = zero4();
#pragma unroll
    for (int p = 0; p < KP; ++p) {
        if (p + 1 < KP) rows_of(p + 1);
        in_order();
#pragma unroll
        for (int part = FULL_PARTS<OP> - 1; part >= 0; --part)
#pragma unroll
            for (int tb = 0; tb < MT; ++tb) v[tb] = mfma32<OP>(w[p & 1][tb], sp[p].u[part], v[tb]);
        also(p);
    }
}
// V' = U - W S of 16 columns from LDS; v holds W S 2^shift (DELTA).
template <int OP, int MT, int UPIECES, bool DELTA> __device__ __forceinline__ void values_of(v4f (&v)[MT], const v2u (&u)[MT], int shift)
{
    const float down = OP == OP_F16 ? pow2(-shift) : 1.f;
#pragma unroll
    for (int tb = 0; tb < MT; ++tb) {
        const v4f x = unpack4<OP>(u[tb]);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[tb][r] = DELTA ? x[r] - (OP == OP_F16 ? v[tb][r] * down : v[tb][r]) : x[r];
    }
}
// S <- decay S + K^T diag(e) V'; v is used up.
template <int OP, int MT, int KP> __device__ __forceinline__ void state_after(v4f (&S)[2 * KP], v4f (&v)[MT], int shift, const char* rows_k, const float* e, float decay, const MinusOne<OP>& minus, Lane ln)
{
    const float up = OP == OP_F16 ? pow2(shift) : 1.f;
    Parts<FULL_PARTS<OP>> vp[MT / 2];
#pragma unroll
    for (int tb = 0; tb < MT; ++tb) {
        const v4f x = *reinterpret_cast<const v4f*>(e + 16 * tb + 4 * ln.q);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[tb][r] *= OP == OP_F16 ? x[r] * up : x[r];
    }
    split_pairs<OP, FULL_PARTS<OP>, MT / 2>(v, vp, minus);
#pragma unroll
    for (int i = 0; i < 2 * KP; ++i) S[i] = times(S[i], decay * up);
    add_turned<OP, MT, KP>(S, rows_k, vp, ln);
    if constexpr (OP == OP_F16) {
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i) S[i] = times(S[i], pow2(-shift));
    }
}

// A step's tokens: what of them there is, and their gates.
struct StepPos {
    int64_t row;  // of its first token
    int valid;    // 0: no such step
    bool inner;   // not a chunk's first step: g counts from the token before
};
template <int R> __device__ __forceinline__ StepPos step_pos(const SeqPos& sq, int64_t step, int64_t last, int C)
{
    const int tokens = C < R ? C : R;
    const int64_t left = step >= 0 && step < last ? sq.len - step * tokens : 0;
    return {sq.tok0 + step * tokens, left < tokens ? (int)left : tokens, C > R && (step & 1)};
}
__device__ __forceinline__ float buffer_float(const void* base, uint32_t span, uint32_t at)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, span, 0x00020000), at, 0, 0));
}
// g, exp(g_end - g), scale exp(g - base) of a step's tokens, its whole decay and that one's logarithm.  (Loads without a branch around them: what is not there,
// or no g at all, lies outside a buffer of no bytes and reads as 0.  Behind a branch they made the wavefront wait for its stores.)
template <int R> struct StepGates {
    static constexpr int FLOATS = 3 * R + 4;
    float g_row, g_end, g_base;
    __device__ __forceinline__ void load(const float* g, const StepPos& at, int H, int h, int i)
    {
        const float* const first = g + at.row * H + h;
        const uint32_t span = g && at.valid > 0 ? (uint32_t)(at.valid - 1) * H * 4u + 4u : 0u, end = (uint32_t)(at.valid > 0 ? at.valid - 1 : 0) * H * 4u;
        g_row = buffer_float(first, span, i < at.valid ? (uint32_t)i * H * 4u : end);
        g_end = buffer_float(first, span, end);
        g_base = buffer_float(first - H, at.inner ? span : 0u, 0u);
    }
    __device__ __forceinline__ void store(float* gl, float scale, int i) const
    {
        if (i >= R) return;
        gl[i] = g_row;
        gl[R + i] = expf(g_end - g_row);
        gl[2 * R + i] = scale * expf(g_row - g_base);
        if (i == 0) gl[3 * R] = expf(g_end - g_base), gl[3 * R + 1] = g_end - g_base;
    }
};

// MT tiles of 16 token rows a step, KP pairs of tiles of 16 channels; 64 columns, four wavefronts of 16.
constexpr int ATTN_COLS = 64;
template <int OP, int MT, int KP, bool DELTA> struct AttnLayout {
    static constexpr int R = 16 * MT, PIECES = 4 * KP, UPIECES = ATTN_COLS / 8;
    static constexpr int ROWS = R * PIECES * 16, U_BYTES = R * UPIECES * 16;
    static constexpr int K_AT = 0;  // twice: the second half of a step reads it while the next is brought
    static constexpr int W_AT = 2 * ROWS, Q_AT = W_AT + (DELTA ? ROWS : 0), U_AT = Q_AT + ROWS;
    static constexpr int S_AT = U_AT + U_BYTES, S_WAVE = KP * 2048;  // two parts of S, a wavefront's columns one after the other
    static constexpr int V_AT = S_AT + 4 * S_WAVE, V_WAVE = MT * 1024;  // of V', twice
    static constexpr int G_AT = V_AT + 8 * V_WAVE, SHIFT_AT = G_AT + 2 * StepGates<R>::FLOATS * 4, BYTES = SHIFT_AT + 64;
};

// Outputs and the final state.
template <int OP, int MT, int KP, bool DELTA, bool TWO>
__global__ __launch_bounds__(512) void k_chunk_attn(AttnArgs a)
{
    typedef AttnLayout<OP, MT, KP, DELTA> LY;
    constexpr int R = LY::R, FP = FULL_PARTS<OP>, PIECES = LY::PIECES;
    __shared__ __attribute__((aligned(16))) char lds[LY::BYTES];
    float* const gates = reinterpret_cast<float*>(lds + LY::G_AT);
    int* const shifts = reinterpret_cast<int*>(lds + LY::SHIFT_AT);  // fp16: of the parts of S and V', by wavefront
    const Lane ln = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane16 = 16 * (16 * ln.q + ln.n);

    const unsigned groups = (a.d_v + ATTN_COLS - 1) / ATTN_COLS;
    const SeqUnit mine = seq_unit(a.map, blockIdx.x, gridDim.x, groups * a.H, by_length(a.map, gridDim.x) && a.n_seg == 1, lds);
    const unsigned cg = mine.unit % groups;
    const int seg = blockIdx.y;
    const int h = mine.unit / groups, s = mine.seq, hs = s * a.H + h;
    const int wg_col = cg * ATTN_COLS;
    const SeqPos sq = seq_pos(a.map, s);
    const int64_t n_chunk = pieces_of(sq.len, a.C);
    int64_t c0, c1;
    segment_chunks(n_chunk, a.n_seg, seg, c0, c1);
    const int tokens = a.C < R ? a.C : R, steps = a.C > R ? a.C / R : 1;  // of a step; of a chunk
    const int64_t all = pieces_of(sq.len, tokens), k0 = c0 * steps, k1 = c1 * steps < all ? c1 * steps : all;

    const int cols = a.d_v - wg_col < ATTN_COLS ? a.d_v - wg_col : ATTN_COLS;
    const uint32_t stride_w = 2u * a.H * a.d_k, stride_u = 2u * a.H * a.d_v;
    const int64_t row0 = sq.tok0 + k0 * tokens;

    if (wave < 4) {
        // The recursion, and W and U.
        const int col0 = wg_col + 16 * wave;
        RowLoader<PIECES, R, 256> lw;
        RowLoader<LY::UPIECES, R, 256> lu;
        const char *at_w = static_cast<const char*>(a.W) + row0 * stride_w + 2 * h * a.d_k, *at_u = static_cast<const char*>(a.U) + row0 * stride_u + 2 * (h * a.d_v + wg_col);
        auto request = [&](int64_t k) {
            const StepPos at = step_pos<R>(sq, k, k1, a.C);
            if constexpr (DELTA) lw.load(at_w, stride_w, a.d_k, at.valid, threadIdx.x);
            lu.load(at_u, stride_u, cols, at.valid, threadIdx.x);
            at_w += (int64_t)tokens * stride_w, at_u += (int64_t)tokens * stride_u;
        };
        auto bring = [&]() {
            if constexpr (DELTA) lw.store(lds + LY::W_AT, threadIdx.x);
            lu.store(lds + LY::U_AT, threadIdx.x);
        };
        request(k0);
        const MinusOne<OP> minus(ln);
        v4f S[2 * KP];
        const float* from = seg == 0 ? a.state : a.seg_state + (int64_t)(seg - 1) * a.map.n_seq * a.H * a.d_k * a.d_v;
        get_state<KP>(from ? from + (int64_t)hs * a.d_k * a.d_v : nullptr, S, a.d_k, a.d_v, col0, false, ln);
        Parts<FP> sp[KP];
        int s_shift = 0;
        // The parts of S: of the state before a chunk for W, two of them for Q in every step.
        auto parts_of_state = [&](bool first) {
            float up = 1.f;
            int shift = 0;
            if constexpr (OP == OP_F16) shift = f16_shift(wave_max(most_of(S))), up = pow2(shift);
            v4f x[2 * KP];
#pragma unroll
            for (int i = 0; i < 2 * KP; ++i) x[i] = OP == OP_F16 ? times(S[i], up) : S[i];
            Parts<DELTA ? FP : 2> t[KP];
            split_pairs<OP, DELTA ? FP : 2, KP>(x, t, minus);
#pragma unroll
            for (int p = 0; p < KP; ++p) {
                char* const to = lds + LY::S_AT + LY::S_WAVE * wave + 2048 * p + lane16;
                *reinterpret_cast<v4u*>(to) = t[p].u[0];
                *reinterpret_cast<v4u*>(to + 1024) = t[p].u[1];
                if constexpr (DELTA) {
                    if (!TWO || first) sp[p] = t[p];
                }
            }
            if (!TWO || first) s_shift = shift;
            if (OP == OP_F16 && ln.q == 0 && ln.n == 0) shifts[wave] = shift;
        };
        parts_of_state(true);
        bring();
        __syncthreads();  // the first rows are in LDS
        for (int64_t k = k0; k < k1; ++k) {
            const float* const gl = gates + (k & 1) * StepGates<R>::FLOATS;
            v4f v[MT];
            v2u u[MT];
#pragma unroll
            for (int tb = 0; tb < MT; ++tb) u[tb] = lds_turned<LY::UPIECES>(lds + LY::U_AT, 16 * tb + 4 * ln.q + (ln.n >> 2), 4 * wave + (ln.n & 3));
            if constexpr (DELTA) rows_times<OP, MT, KP>(v, lds + LY::W_AT, sp, ln, [](int) {});
            request(k + 1);
            __syncthreads();  // W, U, Q and the parts of S are in registers
            values_of<OP, MT, LY::UPIECES, DELTA>(v, u, s_shift);
            int v_shift = 0;
            if constexpr (OP == OP_F16) v_shift = f16_shift(wave_max(most_of(v)));
            {
                if (OP == OP_F16 && ln.q == 0 && ln.n == 0) shifts[4 + 4 * (k & 1) + wave] = v_shift;
                v4f x[MT];
#pragma unroll
                for (int tb = 0; tb < MT; ++tb) x[tb] = OP == OP_F16 ? times(v[tb], pow2(v_shift)) : v[tb];
                Parts<2> t[MT / 2];
                split_pairs<OP, 2, MT / 2>(x, t, minus);
#pragma unroll
                for (int tp = 0; tp < MT / 2; ++tp) {
                    char* const to = lds + LY::V_AT + LY::V_WAVE * (4 * (k & 1) + wave) + 2048 * tp + lane16;
                    *reinterpret_cast<v4u*>(to) = t[tp].u[0];
                    *reinterpret_cast<v4u*>(to + 1024) = t[tp].u[1];
                }
            }
            state_after<OP, MT, KP>(S, v, v_shift, lds + LY::K_AT + (k & 1) * LY::ROWS, gl + R, gl[3 * R], minus, ln);
            parts_of_state(((k + 1) & 1) == 0);
            bring();
            __syncthreads();  // the parts of S and the next rows are in LDS
        }
        if (seg == a.n_seg - 1 && a.final_state) put_state<KP>(a.final_state + (int64_t)hs * a.d_k * a.d_v, S, a.d_k, a.d_v, col0, ln);
        return;
    }

    // K, Q and the gates, scores and outputs.
    const int tid = threadIdx.x - 256;
    const int hk = h / a.group, H_k = a.H / a.group;
    RowLoader<PIECES, R, 256> lq, lk;
    StepGates<R> lg;
    // addresses of the next step to be requested
    const uint32_t stride_k = 2u * H_k * a.d_k;
    const char *at_k = static_cast<const char*>(a.K) + row0 * stride_k + 2 * hk * a.d_k, *at_q = static_cast<const char*>(a.Q) + row0 * stride_k + 2 * hk * a.d_k;
    auto request = [&](int64_t k) {
        const StepPos at = step_pos<R>(sq, k, k1, a.C);
        lk.load(at_k, stride_k, a.d_k, at.valid, tid);
        lq.load(at_q, stride_k, a.d_k, at.valid, tid);
        lg.load(a.g, at, a.H, h, tid);
        at_k += (int64_t)tokens * stride_k, at_q += (int64_t)tokens * stride_k;
    };
    auto bring = [&](int64_t k) {
        lk.store(lds + LY::K_AT + (k & 1) * LY::ROWS, tid);
        lq.store(lds + LY::Q_AT, tid);
        lg.store(gates + (k & 1) * StepGates<R>::FLOATS, a.scale, tid);
    };
    request(k0);
    bring(k0);
    __syncthreads();
    request(k0 + 1);
    const MinusOne<OP> minus(ln);
    // This wavefront's outputs: two column tiles, and of MT = 4 token tiles the outer or the inner two (so that all have six pairs' worth of scores).
    constexpr int NI = MT / 2;
    const int ct = 2 * (wave & 1), half = (wave >> 1) & 1;
    // What is added to the exponents of its score tiles 2 tp and 2 tp + 1 next to the diagonal: nothing, or minus infinity behind it.
    v4f edge[NI][2];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float none = -__builtin_inff(), on = 4 * ln.q + r <= ln.n ? 0.f : none;
        edge[0][0][r] = half == 0 ? on : 0.f, edge[0][1][r] = half == 0 ? none : on;
        if constexpr (NI == 2) edge[1][0][r] = half == 1 ? on : 0.f, edge[1][1][r] = half == 1 ? none : on;
    }
    v4f acc[NI][2];
    Parts<2> pp[NI][NI];  // scores: pairs of tiles, two parts
    int p_shift[NI] = {};  // fp16: of those (a score may lie anywhere, and 22 bits of it are there only in fp16's range)
    // The outputs of step k, whose Q S and scores are there: the scores' product with V', and the store.
    auto finish = [&](int64_t k) {
        const StepPos at = step_pos<R>(sq, k, k1, a.C);
        v4f sum[NI][2];  // (fp16: apart from Q S, for the powers of two of scores and values together may pass what fp32 holds)
#pragma unroll
        for (int ii = 0; ii < NI; ++ii)
#pragma unroll
            for (int t = 0; t < 2; ++t) sum[ii][t] = OP == OP_F16 ? zero4() : acc[ii][t];
        v4u vs[NI][2][2];
#pragma unroll
        for (int tp = 0; tp < NI; ++tp)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int part = 0; part < 2; ++part)
                    vs[tp][t][part] = *reinterpret_cast<const v4u*>(lds + LY::V_AT + LY::V_WAVE * (4 * (k & 1) + ct + t) + 2048 * tp + 1024 * part + lane16);
        in_order();
#pragma unroll
        for (int tp = 0; tp < NI; ++tp)
#pragma unroll
            for (int order = 0; order < 3; ++order)
#pragma unroll
                for (int ii = tp; ii < NI; ++ii)
#pragma unroll
                    for (int t = 0; t < 2; ++t) sum[ii][t] = mfma32<OP>(vs[tp][t][order == 1], pp[ii][tp].u[order == 0], sum[ii][t]);
        const int left = a.d_v - wg_col;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(a.O) + at.row * stride_u + 2 * ((int64_t)h * a.d_v + wg_col), 0,
                                                            at.valid > 0 ? (uint32_t)(at.valid - 1) * stride_u + 2u * left : 0u, 0x00020000);
#pragma unroll
        for (int ii = 0; ii < NI; ++ii)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int i = 16 * (ii == 0 ? half : 3 - half) + ln.n, col = 16 * (ct + t) + 4 * ln.q;
                v4f x = sum[ii][t];
                if constexpr (OP == OP_F16) {
                    const float of_v = pow2(-shifts[4 + 4 * (k & 1) + ct + t]), of_p = pow2(-p_shift[ii]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = acc[ii][t][r] + x[r] * of_v * of_p;
                }
                __builtin_amdgcn_raw_buffer_store_b64(pack4<OP>(x), rsrc, col < left ? (uint32_t)i * stride_u + 2u * col : 0x80000000u, 0, 0);
            }
    };
    for (int64_t k = k0; k < k1; ++k) {
        const float* const gl = gates + (k & 1) * StepGates<R>::FLOATS;
        const char* const rows_k = lds + LY::K_AT + (k & 1) * LY::ROWS;
        v4u q[NI][KP];
        {
            if (k > k0) finish(k - 1);
            v4u sf[2][2][2];
            auto parts_of = [&](int p) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int part = 0; part < 2; ++part) sf[p & 1][t][part] = *reinterpret_cast<const v4u*>(lds + LY::S_AT + LY::S_WAVE * (ct + t) + 2048 * p + 1024 * part + lane16);
            };
#pragma unroll
            for (int p = 0; p < KP; ++p)
#pragma unroll
                for (int ii = 0; ii < NI; ++ii) q[ii][p] = lds_row<PIECES>(lds + LY::Q_AT, 16 * (ii == 0 ? half : 3 - half) + ln.n, 4 * p + ln.q);
            parts_of(0);
#pragma unroll
            for (int ii = 0; ii < NI; ++ii) acc[ii][0] = acc[ii][1] = zero4();
#pragma unroll
            for (int p = 0; p < KP; ++p) {
                if (p + 1 < KP) parts_of(p + 1);
                in_order();
#pragma unroll
                for (int part = 1; part >= 0; --part)
#pragma unroll
                    for (int ii = 0; ii < NI; ++ii)
#pragma unroll
                        for (int t = 0; t < 2; ++t) acc[ii][t] = mfma32<OP>(sf[p & 1][t][part], q[ii][p], acc[ii][t]);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float down = OP == OP_F16 ? pow2(-shifts[ct + t]) : 1.f;  // (fp16: Q S is of S 2^shift)
#pragma unroll
                for (int ii = 0; ii < NI; ++ii) acc[ii][t] = times(acc[ii][t], gl[2 * R + 16 * (ii == 0 ? half : 3 - half) + ln.n] * down);
            }
        }
        __syncthreads();  // W, U, Q and the parts of S are in registers
        bring(k + 1);
        request(k + 2);
        in_order();
        {
            v4u kf[2][2 * NI];
            v4f x[NI][2 * NI];  // scores, turned: x[ii][jt], jt <= 2 ii + 1
            auto keys_of = [&](int p) {
#pragma unroll
                for (int jt = 0; jt < 2 * NI; ++jt) kf[p & 1][jt] = lds_row<PIECES>(rows_k, 16 * jt + ln.n, 4 * p + ln.q);
            };
            keys_of(0);
#pragma unroll
            for (int ii = 0; ii < NI; ++ii)
#pragma unroll
                for (int jt = 0; jt < 2 * NI; ++jt) x[ii][jt] = zero4();
#pragma unroll
            for (int p = 0; p < KP; ++p) {
                if (p + 1 < KP) keys_of(p + 1);
                in_order();
#pragma unroll
                for (int ii = 0; ii < NI; ++ii)
#pragma unroll
                    for (int jt = 0; jt < 2 * ii + 2; ++jt) x[ii][jt] = mfma32<OP>(kf[p & 1][jt], q[ii][p], x[ii][jt]);
            }
            v4f gj[2 * NI];
#pragma unroll
            for (int jt = 0; jt < 2 * NI; ++jt) gj[jt] = *reinterpret_cast<const v4f*>(gl + 16 * jt + 4 * ln.q);
#pragma unroll
            for (int ii = 0; ii < NI; ++ii) {
                const float gi = gl[16 * (ii == 0 ? half : 3 - half) + ln.n];
#pragma unroll
                for (int jt = 0; jt < 2 * ii + 2; ++jt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[ii][jt][r] *= a.scale * __expf(jt >= 2 * ii ? gi - gj[jt][r] + edge[ii][jt & 1][r] : gi - gj[jt][r]);
                if constexpr (OP == OP_F16) {
                    float most = 0.f;
#pragma unroll
                    for (int jt = 0; jt < 2 * ii + 2; ++jt)
#pragma unroll
                        for (int r = 0; r < 4; ++r) most = fmaxf(most, fabsf(x[ii][jt][r]));
                    p_shift[ii] = f16_shift(wave_max(most));
#pragma unroll
                    for (int jt = 0; jt < 2 * ii + 2; ++jt) x[ii][jt] = times(x[ii][jt], pow2(p_shift[ii]));
                }
#pragma unroll
                for (int tp = 0; tp <= ii; ++tp) {
                    v4f two[2] = {x[ii][2 * tp], x[ii][2 * tp + 1]};
                    Parts<2> one[1];
                    split_pairs<OP, 2, 1>(two, one, minus);
                    pp[ii][tp] = one[0];
                }
            }
        }
        __syncthreads();
    }
    if (k0 < k1) finish(k1 - 1);
}

// The recursion alone, 16 WAVES columns of a head, every wavefront with a share of the rows to bring.  ATTN_SEGMENT: what a segment adds to a state (column groups
// of d_v) and, with W, what it does to the one before it: the same recursion from the identity with U = 0 (column groups of d_k behind them).
// ATTN_RECORD: the states before the steps and the values, for the gradient.
enum : int { ATTN_SEGMENT = 1, ATTN_RECORD = 2 };
template <int OP, int MT, int KP, bool DELTA, int WAVES> struct StatesLayout {
    static constexpr int R = 16 * MT, PIECES = 4 * KP, COLS = 16 * WAVES, UPIECES = COLS / 8, ROWS = R * PIECES * 16;
    static constexpr int K_AT = 0, W_AT = 2 * ROWS, U_AT = W_AT + (DELTA ? ROWS : 0), G_AT = U_AT + R * UPIECES * 16, BYTES = G_AT + 2 * StepGates<R>::FLOATS * 4;
};

template <int OP, int MT, int KP, bool DELTA, int MODE, bool TWO, int WAVES>
__device__ __forceinline__ void attn_states(const AttnArgs& a, char* const lds, unsigned b, unsigned n, bool sorted, int seg)
{
    typedef StatesLayout<OP, MT, KP, DELTA, WAVES> LY;
    constexpr bool SEGMENT = MODE == ATTN_SEGMENT;
    constexpr int R = LY::R, FP = FULL_PARTS<OP>, THREADS = 64 * WAVES;  // that bring rows
    float* const gates = reinterpret_cast<float*>(lds + LY::G_AT);
    const Lane ln = lane_id();
    const int tid = threadIdx.x & (THREADS - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool brings = SEGMENT || threadIdx.x >= THREADS;

    const unsigned groups_v = (a.d_v + LY::COLS - 1) / LY::COLS, groups = groups_v + (SEGMENT && DELTA ? (a.d_k + LY::COLS - 1) / LY::COLS : 0);
    const SeqUnit mine = seq_unit(a.map, b, n, groups * a.H, sorted, lds);
    const unsigned cg = mine.unit % groups;
    const int h = mine.unit / groups, s = mine.seq, hs = s * a.H + h, hk = h / a.group, H_k = a.H / a.group;
    const bool trans = SEGMENT && cg >= groups_v;
    const int d_v = trans ? a.d_k : a.d_v, wg_col = (trans ? cg - groups_v : cg) * LY::COLS, col0 = wg_col + 16 * wave;
    const SeqPos sq = seq_pos(a.map, s);
    const int64_t n_chunk = pieces_of(sq.len, a.C);
    int64_t c0, c1;
    segment_chunks(n_chunk, a.n_seg, seg, c0, c1);
    const int tokens = a.C < R ? a.C : R, steps = a.C > R ? a.C / R : 1;
    const int64_t all = pieces_of(sq.len, tokens), k0 = c0 * steps, k1 = c1 * steps < all ? c1 * steps : all;
    const int64_t rec0 = (!SEGMENT && a.map.cu_chunks ? a.map.cu_chunks[s] : s * n_chunk) * steps;

    RowLoader<LY::PIECES, R, THREADS> lk, lw;
    RowLoader<LY::UPIECES, R, THREADS> lu;
    StepGates<R> lg;
    const int cols = a.d_v - wg_col < LY::COLS ? a.d_v - wg_col : LY::COLS;
    const uint32_t stride_k = 2u * H_k * a.d_k, stride_w = 2u * a.H * a.d_k, stride_u = 2u * a.H * a.d_v;
    const int64_t row0 = sq.tok0 + k0 * tokens;
    const char *at_k = static_cast<const char*>(a.K) + row0 * stride_k + 2 * hk * a.d_k, *at_w = static_cast<const char*>(a.W) + row0 * stride_w + 2 * h * a.d_k,
               *at_u = static_cast<const char*>(a.U) + row0 * stride_u + 2 * (h * a.d_v + (trans ? 0 : wg_col));
    auto request = [&](int64_t k) {
        const StepPos at = step_pos<R>(sq, k, k1, a.C);
        lk.load(at_k, stride_k, a.d_k, at.valid, tid);
        if constexpr (DELTA) lw.load(at_w, stride_w, a.d_k, at.valid, tid);
        lu.load(at_u, stride_u, cols, trans ? 0 : at.valid, tid);
        lg.load(a.g, at, a.H, h, tid);
        at_k += (int64_t)tokens * stride_k, at_w += (int64_t)tokens * stride_w, at_u += (int64_t)tokens * stride_u;
    };
    auto bring = [&](int64_t k) {
        lk.store(lds + LY::K_AT + (k & 1) * LY::ROWS, tid);
        if constexpr (DELTA) lw.store(lds + LY::W_AT, tid);
        lu.store(lds + LY::U_AT, tid);
        lg.store(gates + (k & 1) * StepGates<R>::FLOATS, a.scale, tid);
    };
    if (brings) {
        request(k0);
        bring(k0);
    }
    if (!SEGMENT && brings) {
        __syncthreads();
        request(k0 + 1);
        for (int64_t k = k0; k < k1; ++k) {
            __syncthreads();  // W and U are in registers
            bring(k + 1);
            request(k + 2);
            if constexpr (KP == 4) {
                const StepPos at = step_pos<R>(sq, k, k1, a.C);
                const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(a.rec_dg + at.row * a.H + h, 0, a.rec_dg && cg == 0 ? (uint32_t)(at.valid - 1) * a.H * 4u + 4u : 0u, 0x00020000);
                __builtin_amdgcn_raw_buffer_store_b32(0u, rsrc, tid < at.valid ? (uint32_t)tid * a.H * 4u : 0x80000000u, 0, 0);
            }
            __syncthreads();
        }
        return;
    }
    const MinusOne<OP> minus(ln);
    v4f S[2 * KP];
    const float* const from = SEGMENT || !a.state ? nullptr : a.state + (int64_t)hs * a.d_k * a.d_v;
    get_state<KP>(from, S, a.d_k, d_v, col0, trans, ln);
    Parts<FP> sp[KP];
    int s_shift = 0;
    auto parts_of_state = [&](Parts<FP>(&to)[KP], int& shift) {
        if constexpr (OP == OP_F16) shift = f16_shift(wave_max(most_of(S)));
        v4f x[2 * KP];
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i) x[i] = OP == OP_F16 ? times(S[i], pow2(shift)) : S[i];
        split_pairs<OP, FP, KP>(x, to, minus);
    };
    if constexpr (DELTA) parts_of_state(sp, s_shift);
    const TurnOne<OP> one_k(ln, true), one_t(ln, false);
    float total = 0.f;
    __syncthreads();
    if constexpr (SEGMENT) request(k0 + 1);
    for (int64_t k = k0; k < k1; ++k) {
        const float* const gl = gates + (k & 1) * StepGates<R>::FLOATS;
        float* const state_to = SEGMENT ? nullptr : a.rec_state + ((rec0 + k) * a.H + h) * a.d_k * a.d_v;
        if constexpr (!SEGMENT) {
            if constexpr (TWO || !DELTA) {
                Parts<FP> now[KP];
                int shift = 0;
                parts_of_state(now, shift);
#pragma unroll
                for (int p = 0; p < KP; ++p) put_turned<OP>(state_to, p, now[p], pow2(-shift), a.d_k, a.d_v, col0, one_k, ln);
            }
        }
        v4f v[MT];
        v2u u[MT];
#pragma unroll
        for (int tb = 0; tb < MT; ++tb) u[tb] = lds_turned<LY::UPIECES>(lds + LY::U_AT, 16 * tb + 4 * ln.q + (ln.n >> 2), 4 * wave + (ln.n & 3));
        if constexpr (DELTA) {
            rows_times<OP, MT, KP>(v, lds + LY::W_AT, sp, ln, [&](int p) {
                if constexpr (!SEGMENT && !TWO) put_turned<OP>(state_to, p, sp[p], pow2(-s_shift), a.d_k, a.d_v, col0, one_k, ln);
            });
        }
        __syncthreads();  // W and U are in registers
        if constexpr (SEGMENT) {
            bring(k + 1);
            request(k + 2);
        }
        values_of<OP, MT, LY::UPIECES, DELTA>(v, u, s_shift);
        int v_shift = 0;
        if constexpr (OP == OP_F16) v_shift = f16_shift(wave_max(most_of(v)));
        if constexpr (!SEGMENT && DELTA) {
            v4f x[MT];
            Parts<FP> vp[MT / 2];
#pragma unroll
            for (int tb = 0; tb < MT; ++tb) x[tb] = OP == OP_F16 ? times(v[tb], pow2(v_shift)) : v[tb];
            split_pairs<OP, FP, MT / 2>(x, vp, minus);
            const StepPos at = step_pos<R>(sq, k, k1, a.C);
#pragma unroll
            for (int tp = 0; tp < MT / 2; ++tp) put_turned<OP>(a.rec_value + (at.row * a.H + h * at.valid) * a.d_v, tp, vp[tp], pow2(-v_shift), at.valid, a.d_v, col0, one_t, ln);
        }
        if (SEGMENT && !DELTA) total += gl[3 * R + 1];
        state_after<OP, MT, KP>(S, v, v_shift, lds + LY::K_AT + (k & 1) * LY::ROWS, gl + R, gl[3 * R], minus, ln);
        if constexpr (DELTA) {
            if (!TWO || ((k + 1) & 1) == 0) parts_of_state(sp, s_shift);
        }
        __syncthreads();  // the next rows are in LDS
    }
    if constexpr (!SEGMENT) return;
    put_state<KP>((trans ? a.seg_trans : a.seg_state) + ((int64_t)seg * a.map.n_seq * a.H + hs) * a.d_k * d_v, S, a.d_k, d_v, col0, ln);
    if (!DELTA && cg == 0 && tid == 0) a.seg_decay[(int64_t)seg * a.map.n_seq * a.H + hs] = expf(total);
}

template <int OP, int MT, int KP, bool DELTA, int MODE, bool TWO, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_attn_states(AttnArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[StatesLayout<OP, MT, KP, DELTA, WAVES>::BYTES];
    attn_states<OP, MT, KP, DELTA, MODE, TWO, WAVES>(a, lds, blockIdx.x, gridDim.x, false, blockIdx.y);
}

// States before the segments, in place of what the segments add: S <- M S + L from the sequence's initial state, segment by segment.  M and S as three
// bf16 parts each, the six products that matter.  A workgroup takes 16 columns, a wavefront a tile of their rows; the parts of S go round
// through LDS.  M is asked for two segments ahead; a segment of 16 heads of 128 x 128 takes 2.6 us.
template <int KP> __global__ __launch_bounds__(128 * KP) void k_attn_join(AttnArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[2][KP * 3 * 1024];
    const Lane ln = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane16 = 16 * (16 * ln.q + ln.n);
    const unsigned groups = (a.d_v + 15) / 16, b = xcd_neighbours(blockIdx.x, gridDim.x), hs = b / groups;  // (a head's groups read the same M: from one L2)
    const int col = 16 * (b % groups) + ln.n;
    const int64_t heads = (int64_t)a.map.n_seq * a.H;
    auto place = [&](int r) { return col < a.d_v ? 4u * (state_channel(wave, 4 * ln.q + r) * a.d_v + col) : 0x80000000u; };  // (channels that are not there lie outside the buffer)
    v4f S;
    {
        const auto from = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(a.state) + (int64_t)hs * a.d_k * a.d_v, 0, a.state ? 4u * a.d_k * a.d_v : 0u, 0x00020000);
#pragma unroll
        for (int r = 0; r < 4; ++r) S[r] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from, place(r), 0, 0));
        const auto first = __builtin_amdgcn_make_buffer_rsrc(a.seg_first + (int64_t)hs * a.d_k * a.d_v, 0, a.seg_first ? 4u * a.d_k * a.d_v : 0u, 0x00020000);
#pragma unroll
        for (int r = 0; r < 4; ++r) __builtin_amdgcn_raw_buffer_store_b32(bits(S[r]), first, place(r), 0, 0);
    }
    const MinusOne<OP_BF16> minus(ln);
    v4f m[2][2 * KP], add[2];  // rows of M and L, of the next two segments
    auto request = [&](int seg, auto buffer) {
        constexpr int B = buffer;
        const bool there = seg + 1 < a.n_seg;
        const auto M = __builtin_amdgcn_make_buffer_rsrc(a.seg_trans + ((there ? seg : 0) * heads + hs) * a.d_k * a.d_k, 0, there ? 4u * a.d_k * a.d_k : 0u, 0x00020000);
        const auto L = __builtin_amdgcn_make_buffer_rsrc(a.seg_state + ((there ? seg : 0) * heads + hs) * a.d_k * a.d_v, 0, there ? 4u * a.d_k * a.d_v : 0u, 0x00020000);
        const uint32_t row = 4u * (state_channel(wave, ln.n) * a.d_k + 8 * ln.q);
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i)
            m[B][i] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(M, 16 * i < a.d_k ? row + 4u * (32 * (i >> 1) + 4 * (i & 1)) : 0x80000000u, 0, 0));
#pragma unroll
        for (int r = 0; r < 4; ++r) add[B][r] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(L, place(r), 0, 0));
    };
    auto pass = [&](int seg, auto buffer) {
        constexpr int B = buffer;
        Parts<3> mp[KP];
        v4f next = add[B], low = zero4();  // half of the products each, in chains of their own
        split_pairs<OP_BF16, 3, KP>(m[B], mp, minus);
        request(seg + 2, buffer);
        // this wavefront's parts of S: half a pair of tiles
        char* const buf = lds[seg & 1];
        v4f x = S;
#pragma unroll
        for (int part = 0; part < 3; ++part) {
            const v2u u = pack4<OP_BF16>(x);
            *reinterpret_cast<v2u*>(buf + ((wave >> 1) * 3 + part) * 1024 + lane16 + 8 * (wave & 1)) = u;
            x = minus16<OP_BF16>(x, u);
        }
        __syncthreads();
#pragma unroll
        for (int p = 0; p < KP; ++p) {
            v4u sp[3];
#pragma unroll
            for (int part = 0; part < 3; ++part) sp[part] = *reinterpret_cast<const v4u*>(buf + (p * 3 + part) * 1024 + lane16);
#pragma unroll
            for (int j = 0; j < 6; ++j) {
                constexpr int of_m[6] = {2, 0, 1, 1, 0, 0}, of_s[6] = {0, 2, 1, 0, 1, 0};
                (j & 1 ? next : low) = mfma32<OP_BF16>(mp[p].u[of_m[j]], sp[of_s[j]], j & 1 ? next : low);
            }
        }
        const auto L = __builtin_amdgcn_make_buffer_rsrc(a.seg_state + (seg * heads + hs) * a.d_k * a.d_v, 0, 4u * a.d_k * a.d_v, 0x00020000);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            S[r] = next[r] + low[r];
            __builtin_amdgcn_raw_buffer_store_b32(bits(S[r]), L, place(r), 0, 0);
        }
    };
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    request(0, even);
    request(1, odd);
    for (int seg = 0; seg + 1 < a.n_seg; seg += 2) {
        pass(seg, even);
        if (seg + 2 < a.n_seg) pass(seg + 1, odd);
    }
}

// The same without W, where a segment multiplies a state by one number: an element of the state a thread.
static __global__ __launch_bounds__(256) void k_attn_join_plain(AttnArgs a)
{
    const int64_t heads = (int64_t)a.map.n_seq * a.H, size = (int64_t)a.d_k * a.d_v, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= heads * size) return;
    const int64_t hs = i / size;
    float S = a.state ? a.state[i] : 0.f;
    if (a.seg_first) a.seg_first[i] = S;
    for (int seg = 0; seg + 1 < a.n_seg; ++seg) {
        float* const L = a.seg_state + seg * heads * size + i;
        S = a.seg_decay[seg * heads + hs] * S + *L;
        *L = S;
    }
}

}  // namespace triinv
