// What the chunk-attention kernels share: 16-bit parts of fp32 tiles, chunk rows staged in LDS, where a sequence's tokens are.
//
// The state S (d_k x d_v, fp32) stays in registers as 16 x 16 tiles in the accumulator layout (tile_ops.hpp): tile 2 p + e of a column tile holds, in
// register r of lane 16 q + n, channel 32 p + 8 q + 4 e + r of column n.  The two packed tiles of a pair then are, register for register, the operand
// that meets 16 consecutive bytes of a token's row (8 channels a lane), on either side of a product:
//   W S        A = rows of W,  B = tiles of S;       S^T Q^T    A = tiles of S,  B = rows of Q;
//   V'^T P^T   A = tiles of V', B = tiles of P^T;     K^T V'     A = K read transposed from LDS, B = tiles of V'.
// No accumulator crosses lanes on its way to the next product.
#pragma once
#include "tile_ops.hpp"

namespace triinv {

// Sequences of the call: fixed (cu_seqlens null, Tlen tokens each) or packed.
struct SeqMap {
    const int64_t* cu_seqlens;
    const int64_t* cu_chunks;  // packed, kernels over chunks only
    int64_t Tlen;
    int n_seq;
};
struct SeqPos {
    int64_t tok0;  // row of the sequence's first token
    int64_t len;
};
__device__ __forceinline__ SeqPos seq_pos(const SeqMap& m, int s)
{
    if (!m.cu_seqlens) return {(int64_t)s * m.Tlen, m.Tlen};
    const int64_t a = m.cu_seqlens[s];
    return {a, m.cu_seqlens[s + 1] - a};
}

// Pieces of a power of two in n tokens (a 64-bit division is 130 instructions, and a workgroup would begin with three of them).
__device__ __forceinline__ int64_t pieces_of(int64_t n, int size) { return (n + size - 1) >> __builtin_ctz((unsigned)size); }

// Workgroups go to the eight XCDs in turn; neighbours (column groups and heads that read the same rows) are put on one of them.
__device__ __forceinline__ unsigned xcd_neighbours(unsigned b, unsigned n)
{
    const unsigned x = b & 7u, q = n >> 3, r = n & 7u;
    return x * q + (x < r ? x : r) + (b >> 3);
}

// A workgroup's sequence, and its place among the `per` that a sequence has.  Where packed sequences need more than one round of the 256 compute units the longest begin
// (each of them on one XCD, the next on the next), so that none of them starts when the others are done.  Every workgroup ranks the lengths for itself, in time proportional to
// their number, and from the fourth round on the order of the call does as well.  In us, order of the call / by length, 128 channels and columns, W: lengths from 1 to 2200, 4
// heads, 48 sequences (384 workgroups) 143 / 113, 64 170 / 142, 96 (768) 236 / 207, 128 293 / 271, 160 (1280) 359 / 344; to 1000, 48 72 / 55, 96 115 / 107, 128 151 / 142, 160 181 / 182; of
// 16 heads 16 (512) 73 / 77, 24 111 / 105, 32 (1024) 132 / 144, 64 262 / 270; to 600, 2 heads, 128 (512) 58 / 52, 160 72 / 70, 250 (1000) 100 / 113.  Equal lengths, which gain
// nothing: 48 of 4 heads and 500 tokens 59 / 61, 128 128 / 140, 256 254 / 301.
constexpr int LENGTHS_SORTED = 128;  // sequences at most
__host__ __device__ __forceinline__ bool by_length(const SeqMap& m, unsigned n) { return m.cu_seqlens && n > 256u && n <= 768u && m.n_seq <= LENGTHS_SORTED; }
struct SeqUnit {
    int seq;
    unsigned unit;
};
__device__ __forceinline__ SeqUnit seq_unit(const SeqMap& m, unsigned b, unsigned n, unsigned per, bool sorted, char* lds)
{
    if (!sorted) {
        b = xcd_neighbours(b, n);
        return {(int)(b / per), b % per};
    }
    const unsigned eights = (unsigned)m.n_seq / 8u * 8u, in_eights = b >> 3, left = b - eights * per;
    const bool whole = b < eights * per;
    const unsigned place = whole ? in_eights / per * 8u + (b & 7u) : eights + left / per;
    int64_t* const lengths = reinterpret_cast<int64_t*>(lds);
    int* const found = reinterpret_cast<int*>(lengths + LENGTHS_SORTED);
    const int t = threadIdx.x;
    int64_t mine = 0;
    if (t < m.n_seq) lengths[t] = mine = m.cu_seqlens[t + 1] - m.cu_seqlens[t];
    __syncthreads();
    if (t < m.n_seq) {
        unsigned before = 0;
        for (int j = 0; j < m.n_seq; ++j) before += lengths[j] > mine || (lengths[j] == mine && j < t);
        if (before == place) *found = t;
    }
    __syncthreads();
    const int seq = __builtin_amdgcn_readfirstlane(*found);
    __syncthreads();
    return {seq, whole ? in_eights % per : left % per};
}

template <int OP> __device__ __forceinline__ v4f mfma32(v4u a, v4u b, v4f c)
{
    if constexpr (OP == OP_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

__device__ __forceinline__ v4f minus_f16(v4f x, v2u w)
{
#pragma clang fp contract(off)
    const v4h h = __builtin_bit_cast(v4h, w);
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] -= (float)h[r];
    return x;
}
template <int OP> __device__ __forceinline__ v2u pack4(v4f x) { return __builtin_bit_cast(v2u, pack<OP>(x).x); }
template <int OP> __device__ __forceinline__ v4f minus16(v4f x, v2u w)
{
    if constexpr (OP == OP_F16)
        return minus_f16(x, w);
    else
        return minus_bf16(x, Opnd<OP_BF16>{__builtin_bit_cast(v4s, w)});
}

// Parts that carry an fp32 value through 16-bit products: three bf16 (24 bits) or two fp16 (22 bits, for values brought into
// fp16's range by a power of two, see scale_to_f16).
template <int OP> constexpr int FULL_PARTS = OP == OP_F16 ? 2 : 3;

// N parts of two tiles, as operands: u[part] = (tile a, tile b).
template <int N> struct Parts {
    v4u u[N];
};
template <int OP, int N> __device__ __forceinline__ Parts<N> split_pair(v4f a, v4f b)
{
    Parts<N> o;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const v2u x = pack4<OP>(a), y = pack4<OP>(b);
        o.u[i] = v4u{x[0], x[1], y[0], y[1]};
        if (i + 1 < N) a = minus16<OP>(a, x), b = minus16<OP>(b, y);
    }
    return o;
}

// The same for some pairs at once, the rests formed by the matrix cores (x - part = x + (-1) part, exact): one instruction a tile in place of eight, and the
// vector unit is what these kernels run out of first.
template <int OP> struct MinusOne {
    v4u of_first, of_second;  // left operands that pick one tile of a pair, negated
    __device__ __forceinline__ explicit MinusOne(Lane ln)
    {
        constexpr uint32_t m = OP == OP_F16 ? 0xbc00u : 0xbf80u;
        const v2u one = {4 * ln.q == ln.n ? m : 4 * ln.q + 1 == ln.n ? m << 16 : 0u, 4 * ln.q + 2 == ln.n ? m : 4 * ln.q + 3 == ln.n ? m << 16 : 0u};
        of_first = v4u{one[0], one[1], 0u, 0u}, of_second = v4u{0u, 0u, one[0], one[1]};
    }
};
template <int OP, int N, int COUNT> __device__ __forceinline__ void split_pairs(v4f (&x)[2 * COUNT], Parts<N> (&o)[COUNT], const MinusOne<OP>& minus)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int k = 0; k < COUNT; ++k) {
            const v2u a = pack4<OP>(x[2 * k]), b = pack4<OP>(x[2 * k + 1]);
            o[k].u[i] = v4u{a[0], a[1], b[0], b[1]};
        }
        if (i + 1 < N) {
#pragma unroll
            for (int k = 0; k < COUNT; ++k) {
                x[2 * k] = mfma32<OP>(minus.of_first, o[k].u[i], x[2 * k]), x[2 * k + 1] = mfma32<OP>(minus.of_second, o[k].u[i], x[2 * k + 1]);
            }
        }
    }
}

// Tiles turned by the matrix cores, X^T 1 from parts of X, exact: columns down and rows across, so that a lane's four values are neighbours in a row.
// In memory a band of 16 rows is [4 columns][row of the band][4]: a tile is 1 KB in one piece, to be read by rows or by columns.
// Rows of a pair of tiles: 32 channels as they follow each other, or two tiles of 16 tokens.
template <int OP> struct TurnOne {
    v4u of[2];
    __device__ __forceinline__ TurnOne(Lane ln, bool channels)
    {
        constexpr uint32_t m = OP == OP_F16 ? 0x3c00u : 0x3f80u;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int first = channels ? 8 * ln.q + 2 * w : 16 * (w >> 1) + 4 * ln.q + 2 * (w & 1), row = ln.n + 16 * half;
                of[half][w] = first == row ? m : first + 1 == row ? m << 16 : 0u;
            }
    }
};
// The columns col0 .. col0 + 15 of pair number `pair` of tiles; `rows` of them there are in all, of d columns.
template <int OP, int N> __device__ __forceinline__ void put_turned(float* to, int pair, const Parts<N>& p, float down, int rows, int d, int col0, const TurnOne<OP>& one, Lane ln)
{
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(to, 0, (uint32_t)rows * d * 4u, 0x00020000);
    v4f x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int part = N - 1; part >= 0; --part)
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = mfma32<OP>(p.u[part], one.of[i], x[i]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int band = 2 * pair + i, of_band = rows - 16 * band < 16 ? rows - 16 * band : 16;
        const uint32_t at = ln.n < of_band && col0 + 4 * ln.q < d ? 4u * (16 * band * d + (col0 + 4 * ln.q) * of_band + 4 * ln.n) : 0x80000000u;
        if constexpr (OP == OP_F16) {
#pragma unroll
            for (int r = 0; r < 4; ++r) x[i][r] *= down;
        }
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, x[i]), rsrc, at, 0, 0);
    }
}

// Largest of a non-negative value over the wavefront, as a uniform value.
__device__ __forceinline__ float wave_max(float x)
{
    uint32_t u = __builtin_bit_cast(uint32_t, x);  // (magnitudes order like their bits; NaN comes out on top)
#define TRIINV_ROR(n)                                                                                       \
    {                                                                                                       \
        const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0x120 + n, 0xf, 0xf, true);     \
        u = u > y ? u : y;                                                                                  \
    }
    TRIINV_ROR(8) TRIINV_ROR(4) TRIINV_ROR(2) TRIINV_ROR(1)
#undef TRIINV_ROR
    const uint32_t a = __builtin_amdgcn_readlane(u, 0), b = __builtin_amdgcn_readlane(u, 16), c = __builtin_amdgcn_readlane(u, 32), d = __builtin_amdgcn_readlane(u, 48);
    const uint32_t e = a > b ? a : b, f = c > d ? c : d;
    return __builtin_bit_cast(float, e > f ? e : f);
}
// The power of two that brings magnitudes up to `most` below 2^14, where two fp16 parts hold 22 bits of everything above 2^-28 of
// it.  (Kept between 2^-60 and 2^60, so that scales can be multiplied and inverted; also for zeros, infinities and NaN.)
__device__ __forceinline__ int f16_shift(float most)
{
    const int e = 13 - (int)((__builtin_bit_cast(uint32_t, most) >> 23 & 0xffu) - 127u);
    return e < -60 ? -60 : e > 60 ? 60 : e;
}
__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// Rows of 16-byte pieces in LDS, a row's pieces permuted by the row: sixteen lanes that read one piece of sixteen rows find it in sixteen places, and eight
// rows of a transposing read lie as far apart as they can (with the low bits of the row alone four of them meet in the same banks: 4.1 of 7.1 thousand
// cycles of LDS a step were conflicts).
template <int PIECES> struct LdsRows {
    static constexpr int BYTES = PIECES * 16;
    static_assert(PIECES == 8 || PIECES == 16, "rows of 128 or 256 bytes");
    static __device__ __forceinline__ int at(int row, int piece)
    {
        const int turn = PIECES == 16 ? (row & 3) << 2 | (row >> 2 & 3) : (row << 1 & 4) | (row >> 1 & 2) | (row >> 3 & 1);
        return row * BYTES + ((piece ^ turn) << 4);
    }
};
// Eight columns from 8 `piece` on.
template <int PIECES> __device__ __forceinline__ v4u lds_row(const char* m, int row, int piece) { return *reinterpret_cast<const v4u*>(m + LdsRows<PIECES>::at(row, piece)); }
typedef __attribute__((address_space(3))) v4s* lds_v4s_ptr;
// Rows `row` .. `row` + 3 of a lane group, turned: the group's lane n points at row n / 4 of them and at the columns 4 col4 .. 4 col4 + 3, and receives
// column n % 16 of the four rows.
template <int PIECES> __device__ __forceinline__ v2u lds_turned(const char* m, int row, int col4)
{
    const char* p = m + LdsRows<PIECES>::at(row, col4 >> 1) + ((col4 & 1) << 3);
    return __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(p)));
}
// Tokens 32 tp .. 32 tp + 31 of the channels of state tile i, as an operand over the tokens.
template <int PIECES> __device__ __forceinline__ v4u lds_turned_tile(const char* m, int tp, int i, Lane ln)
{
    const int row = 32 * tp + 4 * ln.q + (ln.n >> 2), col4 = 8 * (i >> 1) + 2 * (ln.n & 3) + (i & 1);
    const v2u a = lds_turned<PIECES>(m, row, col4), b = lds_turned<PIECES>(m, row + 16, col4);
    return v4u{a[0], a[1], b[0], b[1]};
}
// Channel of row `row` of state tile i.
__device__ __forceinline__ int state_channel(int i, int row) { return 32 * (i >> 1) + 8 * (row >> 2) + 4 * (i & 1) + (row & 3); }

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

// Rows of one head of a [token][heads][d] tensor on their way from memory to LDS: `ROWS` of them, what is not there (rows from
// `valid` on, columns from d on) as zeros, by the bounds check of buffer loads.  A thread has one piece of every THREADS / PIECES-th row.
// The same value, as one that a loop must not take for its own: sums with it are formed where they are used instead of being kept in a register each.
__device__ __forceinline__ uint32_t in_place(uint32_t x)
{
    asm volatile("" : "+v"(x));
    return x;
}

template <int PIECES, int ROWS, int THREADS> struct RowLoader {
    static constexpr int STRIDE = THREADS / PIECES, N = (ROWS + STRIDE - 1) / STRIDE;
    static_assert(THREADS % PIECES == 0 && (STRIDE % 16 == 0 || N == 1), "a thread's rows are permuted alike");
    v4u v[N];
    __device__ __forceinline__ void load(const void* first, uint32_t stride, int d, int valid, int tid)
    {
        const uint32_t span = valid > 0 ? (uint32_t)(valid - 1) * stride + (uint32_t)d * 2u : 0u;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(first), 0, span, 0x00020000);
        const int row = tid / PIECES, piece = tid % PIECES;
        uint32_t at = in_place(8 * piece < d && (ROWS >= STRIDE || row < ROWS) ? (uint32_t)row * stride + 16u * piece : 0x80000000u);
#pragma unroll
        for (int i = 0; i < N; ++i, at += STRIDE * stride) v[i] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0));
    }
    __device__ __forceinline__ void store(char* m, int tid) const
    {
        const int row = tid / PIECES;
        if (ROWS < STRIDE && row >= ROWS) return;
        char* const to = m + LdsRows<PIECES>::at(row, tid % PIECES);
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<v4u*>(to + i * STRIDE * LdsRows<PIECES>::BYTES) = v[i];
    }
};

// Nothing is moved across: what stands before is issued before (the scheduler, left alone, waits for every read from LDS right where it asked for it).
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

}  // namespace triinv
