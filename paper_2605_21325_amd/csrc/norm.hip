// Root-mean-square norm with the residual's addition in front:
//     s = x + residual (rounded to x's type and written),   y = s / sqrt(mean(s^2) + eps) . weight
// y in x's type, or in 8 bits (4 exponent and 3 mantissa bits, largest value 448) with an fp32 scale for every row or group of columns,
// scale = max |y| / 448 (1 where that is 0).  The gradient, from s as it was written, with r = 1 / sqrt(mean(s^2) + eps):
//     dx = dsum + r (dy . w - s r^2 mean(dy . w . s)),   dw = sum over the rows of dy . s r.
//
// Bound by memory, each element read once: a row stays in the registers of its wavefronts, 8 elements a piece, PIECES pieces a lane, all
// requested at once.  One wavefront takes a row where rows are short and many (no barrier anywhere), more of them where they are few or long.
// Measured: 65536 rows of 2048 with residual, bf16, 8 bits out 170 us (5.5 TB/s); the gradient of 16381 rows of 4096 77 us (5.2 TB/s; 96 without the
// next row's request ahead and with a barrier more a row).
#include "layer.hpp"
#include "tile_ops.hpp"

namespace triinv {

namespace {

typedef float v8f __attribute__((ext_vector_type(8)));

// Eight elements as they are in memory, and widened.
template <int DT> struct Raw8 {
    v4u u[DT == OP_F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void* p, int64_t i)
    {
        const v4u* const from = reinterpret_cast<const v4u*>(static_cast<const char*>(p) + i * (DT == OP_F32 ? 4 : 2));
        u[0] = from[0];
        if constexpr (DT == OP_F32) u[1] = from[1];
    }
    __device__ __forceinline__ void clear()
    {
        u[0] = v4u{0u, 0u, 0u, 0u};
        if constexpr (DT == OP_F32) u[1] = u[0];
    }
    __device__ __forceinline__ v8f wide() const
    {
        v8f o;
        if constexpr (DT == OP_F32) {
            o = __builtin_shufflevector(__builtin_bit_cast(v4f, u[0]), __builtin_bit_cast(v4f, u[1]), 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint16_t x = (uint16_t)(u[0][e >> 1] >> (16 * (e & 1)));
                o[e] = DT == OP_F16 ? f16_to_f32(x) : bf16_to_f32(x);
            }
        }
        return o;
    }
};
template <int DT> __device__ __forceinline__ v8f load8(const void* p, int64_t i)
{
    Raw8<DT> r;
    r.load(p, i);
    return r.wide();
}
// x rounded to the type, and written.
template <int DT> __device__ __forceinline__ v8f store8(void* p, int64_t i, v8f x)
{
    if constexpr (DT == OP_F32) {
        *reinterpret_cast<v4f*>(static_cast<float*>(p) + i) = __builtin_shufflevector(x, x, 0, 1, 2, 3);
        *reinterpret_cast<v4f*>(static_cast<float*>(p) + i + 4) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
    } else {
        v4u u;
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = DT == OP_F16 ? pack2_f16(x[2 * e], x[2 * e + 1]) : pack2_bf16(x[2 * e], x[2 * e + 1]);
        *reinterpret_cast<v4u*>(static_cast<uint16_t*>(p) + i) = u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint16_t h = (uint16_t)(u[e >> 1] >> (16 * (e & 1)));
            x[e] = DT == OP_F16 ? f16_to_f32(h) : bf16_to_f32(h);
        }
    }
    return x;
}

__device__ __forceinline__ float lanes_sum(float x, int width)
{
    for (int d = 1; d < width; d *= 2) x += __shfl_xor(x, d);
    return x;
}
// Largest magnitude over `width` lanes; as bit patterns, which puts NaN on top.
__device__ __forceinline__ uint32_t lanes_max(uint32_t x, int width)
{
    for (int d = 1; d < width; d *= 2) {
        const uint32_t y = __shfl_xor(x, d);
        x = x > y ? x : y;
    }
    return x;
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t magnitude(v8f x)
{
    uint32_t m = magnitude(x[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) m = m > magnitude(x[e]) ? m : magnitude(x[e]);
    return m;
}
__device__ __forceinline__ float scale_of(uint32_t most)
{
    const float s = __builtin_bit_cast(float, most) * (1.f / 448.f);
    return s == 0.f ? 1.f : s;
}
// y / scale in 8 bits: what rounding carries past the largest value stays there, NaN stays NaN.
__device__ __forceinline__ void store_fp8(void* p, int64_t i, v8f y, float scale)
{
    uint32_t u[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float z = y[e] / scale;
        y[e] = z > 448.f ? 448.f : z < -448.f ? -448.f : z;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
        u[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], w, true);
    }
    *reinterpret_cast<v2u*>(static_cast<uint8_t*>(p) + i) = v2u{u[0], u[1]};
}

// A value of all WAVES wavefronts of a row through LDS.
template <int WAVES, class T, class F> __device__ __forceinline__ T across_waves(T x, T* lds, F join)
{
    if constexpr (WAVES == 1) return x;
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[w] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) x = join(x, lds[i]);
    __syncthreads();
    return x;
}

// WAVES wavefronts a row; workgroups of 256 threads where that is one.
enum : int { OUT_SAME = 0, OUT_ROW = 1, OUT_GROUP = 2 };
template <int DT, int OUT, bool RESIDUAL, int WAVES, int PIECES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void k_norm(NormCall a)
{
    constexpr int ROWS = WAVES == 1 ? 4 : 1, LANES = 64 * WAVES;
    __shared__ float sums[WAVES];
    __shared__ uint32_t mosts[WAVES];
    const int lane = threadIdx.x % LANES;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ROWS + threadIdx.x / LANES;
    if (row >= a.N) return;  // (whole wavefronts; with more than one to a row there is one row a workgroup)
    const int64_t at = row * a.D;
    v8f x[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int c = 8 * (lane + LANES * i);
        x[i] = v8f{0, 0, 0, 0, 0, 0, 0, 0};
        if (c < a.D) x[i] = load8<DT>(a.x, at + c);
    }
    if constexpr (RESIDUAL) {
        v8f r[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int c = 8 * (lane + LANES * i);
            r[i] = v8f{0, 0, 0, 0, 0, 0, 0, 0};
            if (c < a.D) r[i] = load8<DT>(a.residual, at + c);
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int c = 8 * (lane + LANES * i);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] += r[i][e];
            if (c < a.D) x[i] = store8<DT>(a.sum, at + c, x[i]);
        }
    }
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sq += x[i][e] * x[i][e];
    sq = across_waves<WAVES>(lanes_sum(sq, 64), sums, [](float p, float q) { return p + q; });
    const float rstd = 1.f / sqrtf(sq / (float)a.D + a.eps);
    uint32_t most = 0u;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int c = 8 * (lane + LANES * i);
        if (c < a.D) {
            const v8f w = load8<DT>(a.weight, c);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = x[i][e] * rstd * w[e];
            if constexpr (OUT == OUT_SAME) store8<DT>(a.y, at + c, x[i]);
        }
        if constexpr (OUT == OUT_ROW) {
            const uint32_t m = magnitude(x[i]);
            most = most > m ? most : m;
        }
        if constexpr (OUT == OUT_GROUP) {  // 128 columns: sixteen lanes
            const float scale = scale_of(lanes_max(magnitude(x[i]), 16));
            if (c < a.D) {
                store_fp8(a.y, at + c, x[i], scale);
                if (lane % 16 == 0) a.scales[row * (a.D / 128) + c / 128] = scale;
            }
        }
    }
    if constexpr (OUT == OUT_ROW) {
        most = across_waves<WAVES>(lanes_max(most, 64), mosts, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
        const float scale = scale_of(most);
        if (lane == 0) a.scales[row] = scale;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int c = 8 * (lane + LANES * i);
            if (c < a.D) store_fp8(a.y, at + c, x[i], scale);
        }
    }
}

template <int DT, int OUT, bool RESIDUAL, int WAVES> int go_pieces(const NormCall& a)
{
    const int pieces = (a.D + 512 * WAVES - 1) / (512 * WAVES);
    const dim3 grid = long_grid(WAVES == 1 ? (a.N + 3) / 4 : a.N), block(WAVES == 1 ? 256 : 64 * WAVES);
    if constexpr (WAVES <= 4) {
        if (pieces <= 1) return launch_kernel(false, k_norm<DT, OUT, RESIDUAL, WAVES, 1>, grid, block, 0, a.stream, a);
    }
    if (pieces <= 2) return launch_kernel(false, k_norm<DT, OUT, RESIDUAL, WAVES, 2>, grid, block, 0, a.stream, a);
    if constexpr (WAVES == 4) {
        if (pieces <= 4) return launch_kernel(false, k_norm<DT, OUT, RESIDUAL, WAVES, 4>, grid, block, 0, a.stream, a);
    }
    return NOT_BUILT;
}
template <int DT, int OUT, bool RESIDUAL> int go_waves(const NormCall& a)
{
    // One wavefront a row against four, bf16, a scale a row, in us: D = 256, 65536 rows 38 and 88; D = 1024, 65536 rows 89 and 121, 4096 rows 8.7 and 9.8,
    // 1024 rows 5.1 and 4.8; D = 2048, 65536 rows 178 and 173, 1024 rows 8.0 and 6.0.
    if (a.D <= 1024 && a.N > 1024) return go_pieces<DT, OUT, RESIDUAL, 1>(a);
    if (a.D <= 8192) return go_pieces<DT, OUT, RESIDUAL, 4>(a);
    return go_pieces<DT, OUT, RESIDUAL, 16>(a);
}
template <int DT> int go_out(const NormCall& a)
{
    if (a.group < 0) return a.residual ? go_waves<DT, OUT_SAME, true>(a) : go_waves<DT, OUT_SAME, false>(a);
    if (a.group == 0) return a.residual ? go_waves<DT, OUT_ROW, true>(a) : go_waves<DT, OUT_ROW, false>(a);
    return a.residual ? go_waves<DT, OUT_GROUP, true>(a) : go_waves<DT, OUT_GROUP, false>(a);
}

// The gradient.  A workgroup takes rows in turn (row = group, group + groups, ...) and keeps its sum of dw in registers; the groups' sums
// are written out and added up by k_norm_dweight, always in the same order.
template <int DT, int PIECES, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_norm_bwd(NormBwdCall a)
{
    constexpr int LANES = 64 * WAVES;
    __shared__ v2f sums[2][WAVES];  // of one row and the next: one barrier a row
    const int lane = threadIdx.x, wave = lane >> 6;
    v8f w[PIECES], dw[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int c = 8 * (lane + LANES * i);
        dw[i] = w[i] = v8f{0, 0, 0, 0, 0, 0, 0, 0};
        if (c < a.D) w[i] = load8<DT>(a.weight, c);
    }
    Raw8<DT> rx[PIECES], rd[PIECES], rt[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) rx[i].clear(), rd[i].clear(), rt[i].clear();
    auto request = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int c = 8 * (lane + LANES * i);
            if (c >= a.D) continue;
            rx[i].load(a.x, row * a.D + c), rd[i].load(a.dy, row * a.D + c);
            if (a.dsum) rt[i].load(a.dsum, row * a.D + c);
        }
    };
    constexpr bool AHEAD = PIECES <= 2;  // the next row comes while one is at work; four pieces of both do not fit in registers
    if (AHEAD && blockIdx.x < a.N) request(blockIdx.x);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x, turn ^= 1) {
        const int64_t at = row * a.D;
        if (!AHEAD) request(row);
        v8f x[PIECES], d[PIECES], t[PIECES];
        v2f s = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < PIECES; ++i) x[i] = rx[i].wide(), d[i] = rd[i].wide(), t[i] = rt[i].wide();
        if (AHEAD && row + gridDim.x < a.N) request(row + gridDim.x);
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += x[i][e] * x[i][e], s[1] += d[i][e] * w[i][e] * x[i][e];
        s[0] = lanes_sum(s[0], 64), s[1] = lanes_sum(s[1], 64);
        if constexpr (WAVES > 1) {
            if ((lane & 63) == 0) sums[turn][wave] = s;
            __syncthreads();
            s = sums[turn][0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) s[0] += sums[turn][i][0], s[1] += sums[turn][i][1];
        }
        const float rstd = 1.f / sqrtf(s[0] / (float)a.D + a.eps), m = s[1] / (float)a.D * rstd * rstd;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int c = 8 * (lane + LANES * i);
            if (c >= a.D) continue;
            v8f dx;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dw[i][e] += d[i][e] * (x[i][e] * rstd);
                dx[e] = rstd * (d[i][e] * w[i][e] - x[i][e] * m) + t[i][e];
            }
            store8<DT>(a.dx, at + c, dx);
        }
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int c = 8 * (lane + LANES * i);
        if (c < a.D) store8<OP_F32>(a.partial, (int64_t)blockIdx.x * a.D + c, dw[i]);
    }
}

// dweight[c] = sum of partial[group][c]: 16 columns a workgroup, 64 threads a column, in the same order every time.
__global__ __launch_bounds__(1024) void k_norm_dweight(const float* partial, float* dweight, int groups, int D)
{
    __shared__ float part[64][17];
    const int cx = threadIdx.x & 15, y = threadIdx.x >> 4, c = 16 * blockIdx.x + cx;
    float s = 0.f;
    if (c < D) {
#pragma unroll 8
        for (int g = y; g < groups; g += 64) s += partial[(int64_t)g * D + c];
    }
    part[y][cx] = s;
    __syncthreads();
    for (int half = 32; half > 0; half /= 2) {
        if (y < half) part[y][cx] = s += part[y + half][cx];
        __syncthreads();
    }
    if (y == 0 && c < D) dweight[c] = s;
}

template <int DT, int WAVES> int bwd_pieces(const NormBwdCall& a)
{
    const int pieces = (a.D + 512 * WAVES - 1) / (512 * WAVES);
    const dim3 grid((unsigned)a.groups), block(64 * WAVES);
    if constexpr (WAVES < 8) {
        if (pieces <= 1) return launch_kernel(false, k_norm_bwd<DT, 1, WAVES>, grid, block, 0, a.stream, a);
    }
    if constexpr (WAVES > 1) {
        if (pieces <= 2) return launch_kernel(false, k_norm_bwd<DT, 2, WAVES>, grid, block, 0, a.stream, a);
    }
    if constexpr (WAVES == 8) {
        if (pieces <= 4) return launch_kernel(false, k_norm_bwd<DT, 4, WAVES>, grid, block, 0, a.stream, a);
    }
    return NOT_BUILT;
}
template <int DT> int bwd(const NormBwdCall& a)
{
    if (a.groups == 0) return launch_kernel(false, k_norm_dweight, dim3((unsigned)((a.D + 15) / 16)), dim3(1024), 0, a.stream, a.partial, a.dweight, 0, a.D);
    // One, four and eight wavefronts a row, bf16 (fp32 the same or level), in us: 65536 rows of 256 columns 94 / 108 / 117, of 512 96 / 108 / 118; 16384 rows of 768 37 / 34 / 38,
    // of 2048 56 / 40 / 42, of 4096 - / 79 / 79, of 5120 - / 98 / 105 (four with four pieces a lane, an instance more), of 8192 - / 154 / 153; 8192 rows of 16384 eight 167, sixteen 290.
    const int rc = a.D <= 512 ? bwd_pieces<DT, 1>(a) : a.D <= 4096 ? bwd_pieces<DT, 4>(a) : bwd_pieces<DT, 8>(a);
    if (rc != LAUNCHED) return rc;
    return launch_kernel(false, k_norm_dweight, dim3((unsigned)((a.D + 15) / 16)), dim3(1024), 0, a.stream, a.partial, a.dweight, a.groups, a.D);
}

}  // namespace

int launch_norm(const NormCall& a) { return a.dtype == OP_F32 ? go_out<OP_F32>(a) : a.dtype == OP_F16 ? go_out<OP_F16>(a) : go_out<OP_BF16>(a); }
int launch_norm_bwd(const NormBwdCall& a) { return a.dtype == OP_F32 ? bwd<OP_F32>(a) : a.dtype == OP_F16 ? bwd<OP_F16>(a) : bwd<OP_BF16>(a); }

}  // namespace triinv
