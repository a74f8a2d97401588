// What the chunk-attention kernels share: 16-bit parts of fp32 tiles, chunk rows staged in LDS, where a sequence's tokens are.
//
// The state S (d_k x d_v, fp32) stays in registers as 16 x 16 tiles in the accumulator layout (tile_ops.hpp), a wavefront holding all
// d_k rows of its columns.  Tile 2 p + h of a column holds, in row 4 q + r, channel 32 p + 8 q + 4 h + r: the two packed tiles of a
// pair then are, register for register, the operand that meets 16 consecutive bytes of a token's row (8 channels a lane), on either
// side of a product:
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

// Workgroups go to the eight XCDs in turn; neighbours (column groups and heads that read the same rows) are put on one of them.
__device__ __forceinline__ unsigned xcd_neighbours(unsigned b, unsigned n)
{
    const unsigned x = b & 7u, q = n >> 3, r = n & 7u;
    return x * q + (x < r ? x : r) + (b >> 3);
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

// Rows of 16-byte pieces in LDS; a row's pieces are permuted by the row, so that sixteen lanes reading one piece of sixteen rows, or
// transposing reads of four rows, meet different banks.
template <int PIECES> struct LdsRows {
    static constexpr int BYTES = PIECES * 16, TURN = (PIECES < 16 ? PIECES : 16) - 1;
    static_assert((PIECES & (PIECES - 1)) == 0, "a power of two");
    static __device__ __forceinline__ int at(int row, int piece) { return row * BYTES + ((piece ^ (row & TURN)) << 4); }
};
template <int PIECES> __device__ __forceinline__ v4u lds_row(const char* m, int row, int piece)
{
    return *reinterpret_cast<const v4u*>(m + LdsRows<PIECES>::at(row, piece));
}
typedef __attribute__((address_space(3))) v4s* lds_v4s_ptr;
// Rows 16 tb + 4 q + r (r = 0..3) of column 4 * (piece of lane n / 4) + n % 4: columns are given by the lane's own 4-column piece `col4`.
template <int PIECES> __device__ __forceinline__ v2u lds_turned(const char* m, int row, int col4)
{
    const char* p = m + LdsRows<PIECES>::at(row, col4 >> 1) + ((col4 & 1) << 3);
    return __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(p)));
}

// Rows of one head of a [token][heads][d] tensor on their way from memory to LDS: `rows` of them, what is not there (rows from
// `valid` on, columns from d on) as zeros, by the bounds check of buffer loads.
template <int PIECES, int ROWS, int THREADS> struct RowLoader {
    static constexpr int N = (PIECES * ROWS + THREADS - 1) / THREADS;
    v4u v[N];
    static __device__ __forceinline__ constexpr bool whole() { return PIECES * ROWS % THREADS == 0; }
    __device__ __forceinline__ void load(const void* base, int64_t first_elem, int row_elems, int d, int valid, int tid)
    {
        const uint32_t stride = (uint32_t)row_elems * 2u;
        const uint32_t span = valid > 0 ? (uint32_t)(valid - 1) * stride + (uint32_t)d * 2u : 0u;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base)) + first_elem * 2, 0, span, 0x00020000);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int k = tid + i * THREADS, row = k / PIECES, piece = k % PIECES;
            const bool there = (whole() || row < ROWS) && 8 * piece < d;
            v[i] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rsrc, there ? (uint32_t)row * stride + 16u * piece : 0x80000000u, 0, 0));
        }
    }
    __device__ __forceinline__ void store(char* m, int tid) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int k = tid + i * THREADS;
            if (whole() || k < PIECES * ROWS) *reinterpret_cast<v4u*>(m + LdsRows<PIECES>::at(k / PIECES, k % PIECES)) = v[i];
        }
    }
};

}  // namespace triinv
