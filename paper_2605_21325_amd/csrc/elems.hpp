// VEC elements of an operand type that stand side by side, as they are in memory and widened.
#pragma once
#include "tile_ops.hpp"

namespace triinv {

template <int DT, int VEC> struct Elems {
    static constexpr int SIZE = DT == OP_F32 ? 4 : 2, BYTES = VEC * SIZE, WORDS = (BYTES + 3) / 4;
    uint32_t w[WORDS];

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0u;
    }
    // From element i on; the address is a multiple of BYTES (of 16 where that is more).
    __device__ __forceinline__ void load(const void* p, int64_t i)
    {
        const char* const from = static_cast<const char*>(p) + i * SIZE;
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int j = 0; j < BYTES / 16; ++j) {
                const v4u x = reinterpret_cast<const v4u*>(from)[j];
                w[4 * j] = x[0], w[4 * j + 1] = x[1], w[4 * j + 2] = x[2], w[4 * j + 3] = x[3];
            }
        } else if constexpr (BYTES == 8) {
            const v2u x = *reinterpret_cast<const v2u*>(from);
            w[0] = x[0], w[1] = x[1];
        } else if constexpr (BYTES == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(from);
        } else {
            w[0] = *reinterpret_cast<const uint16_t*>(from);
        }
    }
    // From a buffer, `lane` bytes (of the lane) and `row` (of all of them) behind its beginning; nothing where `lane` is beyond the buffer's end: zeros.  Up to 8 bytes.
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, uint32_t lane, uint32_t row)
    {
        if constexpr (BYTES == 8) {
            const v2u x = __builtin_bit_cast(v2u, __builtin_amdgcn_raw_buffer_load_b64(from, lane, row, 0));
            w[0] = x[0], w[1] = x[1];
        } else if constexpr (BYTES == 4) {
            w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_raw_buffer_load_b32(from, lane, row, 0));
        } else {
            static_assert(BYTES == 2);
            w[0] = __builtin_bit_cast(uint16_t, __builtin_amdgcn_raw_buffer_load_b16(from, lane, row, 0));
        }
    }
    __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t to, uint32_t lane, uint32_t row) const
    {
        if constexpr (BYTES == 8)
            __builtin_amdgcn_raw_buffer_store_b64(v2u{w[0], w[1]}, to, lane, row, 0);
        else if constexpr (BYTES == 4)
            __builtin_amdgcn_raw_buffer_store_b32(w[0], to, lane, row, 0);
        else
            __builtin_amdgcn_raw_buffer_store_b16((uint16_t)w[0], to, lane, row, 0);
    }
    __device__ __forceinline__ float operator[](int e) const
    {
        if constexpr (DT == OP_F32) return __builtin_bit_cast(float, w[e]);
        const uint16_t x = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
        return DT == OP_F16 ? f16_to_f32(x) : bf16_to_f32(x);
    }
    // Rounded to the type, to nearest even.
    __device__ __forceinline__ void set(const float (&x)[VEC])
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if constexpr (DT == OP_F32) {
                w[i] = __builtin_bit_cast(uint32_t, x[i]);
            } else {
                const float hi = 2 * i + 1 < VEC ? x[(2 * i + 1) % VEC] : 0.f;
                w[i] = DT == OP_F16 ? pack2_f16(x[2 * i], hi) : pack2_bf16(x[2 * i], hi);
            }
        }
    }
    __device__ __forceinline__ void store(void* p, int64_t i) const
    {
        char* const to = static_cast<char*>(p) + i * SIZE;
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int j = 0; j < BYTES / 16; ++j) reinterpret_cast<v4u*>(to)[j] = v4u{w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]};
        } else if constexpr (BYTES == 8) {
            *reinterpret_cast<v2u*>(to) = v2u{w[0], w[1]};
        } else if constexpr (BYTES == 4) {
            *reinterpret_cast<uint32_t*>(to) = w[0];
        } else {
            *reinterpret_cast<uint16_t*>(to) = (uint16_t)w[0];
        }
    }
};

template <int DT, int VEC> __device__ __forceinline__ void store_rounded(void* p, int64_t i, const float (&x)[VEC])
{
    Elems<DT, VEC> e;
    e.set(x);
    e.store(p, i);
}

}  // namespace triinv
