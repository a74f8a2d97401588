// The layer's single token: S <- exp(g) S + k v'^T with v' = beta (v - S^T k) (delta rule; without beta v' = v), S^T k taken of the
// decayed state, and o = scale S^T q, the state updated in place in a pool of slots.
//
// Bound by memory: every element of S (fp32) is read and written once, 8 bytes for 6 operations.  A workgroup takes some columns of one
// head, all its rows; a thread holds four columns of ROWS rows in registers, all loads in flight before the first is used; the two sums
// over the rows (S^T k, then S^T q of the new state) are closed through LDS in a fixed order.  Measured: 256 sequences of 32 heads of 128 x 128 in the slots of a pool, bf16,
// 200 us (5.4 TB/s), one of 16 heads 4.6 (a launch).
#include "layer.hpp"
#include "tile_ops.hpp"

namespace triinv {

namespace {

template <int DT> __device__ __forceinline__ float elem(const void* p, int64_t i)
{
    if constexpr (DT == OP_F32) return static_cast<const float*>(p)[i];
    const uint16_t x = static_cast<const uint16_t*>(p)[i];
    return DT == OP_F16 ? f16_to_f32(x) : bf16_to_f32(x);
}
template <int DT> __device__ __forceinline__ void put_elem(void* p, int64_t i, float x)
{
    if constexpr (DT == OP_F32)
        static_cast<float*>(p)[i] = x;
    else if constexpr (DT == OP_F16)
        static_cast<uint16_t*>(p)[i] = (uint16_t)pack2_f16(x, 0.f);
    else
        static_cast<uint16_t*>(p)[i] = (uint16_t)pack2_bf16(x, 0.f);
}

constexpr int THREADS = 256;

// CG threads side by side, four columns each; THREADS / CG of them take a row in turn.  PASSING: states that no cache keeps until the next token.
template <int DT, int CG, int ROWS> __global__ __launch_bounds__(THREADS) void k_gdn_step(StepCall a)
{
    constexpr int RG = THREADS / CG;
    constexpr bool PASSING = CG == 16;
    __shared__ float kq[2][RG * ROWS];
    __shared__ v4f part[RG][CG + 1];
    const int tid = threadIdx.x, cx = tid % CG, rg = tid / CG;
    const int groups = (a.d_v + 4 * CG - 1) / (4 * CG);
    const unsigned block = blockIdx.y * gridDim.x + blockIdx.x;
    const int cg = block % groups, bh = block / groups, h = bh % a.H, b = bh / a.H;
    if (b >= a.B) return;
    const int hk = h / (a.H / a.H_k);
    const int64_t slot = a.slots ? a.slots[b] : b;
    const int col = 4 * (cg * CG + cx);
    const bool mine = col < a.d_v;
    if (slot < 0 || slot >= a.n_slot) {  // no state: nothing is updated, the output is zero
        if (mine && rg == 0)
            for (int e = 0; e < 4; ++e) put_elem<DT>(a.o, ((int64_t)b * a.H + h) * a.d_v + col + e, 0.f);
        return;
    }
    float* const S = a.state + (slot * a.H + h) * a.d_k * a.d_v + col;
    v4f s[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int row = rg + RG * i;
        const v4f* const from = reinterpret_cast<const v4f*>(S + (int64_t)row * a.d_v);
        s[i] = !mine || row >= a.d_k ? zero4() : PASSING ? __builtin_nontemporal_load(from) : *from;
    }
    for (int i = tid; i < RG * ROWS; i += THREADS) {
        kq[0][i] = i < a.d_k ? elem<DT>(a.k, ((int64_t)b * a.H_k + hk) * a.d_k + i) : 0.f;
        kq[1][i] = i < a.d_k ? elem<DT>(a.q, ((int64_t)b * a.H_k + hk) * a.d_k + i) : 0.f;
    }
    v4f v = zero4();
    if (mine)
        for (int e = 0; e < 4; ++e) v[e] = elem<DT>(a.v, ((int64_t)b * a.H + h) * a.d_v + col + e);
    const float decay = a.g ? expf(a.g[(int64_t)b * a.H + h]) : 1.f;
    __syncthreads();
    if (a.g) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[i][e] *= decay;
    }
    auto sum_rows = [&](const float* w) {
        v4f x = zero4();
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] += w[rg + RG * i] * s[i][e];
        part[rg][cx] = x;
        __syncthreads();
        x = part[0][cx];
#pragma unroll
        for (int r = 1; r < RG; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] += part[r][cx][e];
        __syncthreads();
        return x;
    };
    if (a.beta) {
        const float beta = a.beta[(int64_t)b * a.H + h];
        const v4f kS = sum_rows(kq[0]);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = beta * (v[e] - kS[e]);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int row = rg + RG * i;
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] += kq[0][row] * v[e];
        v4f* const to = reinterpret_cast<v4f*>(S + (int64_t)row * a.d_v);
        if (mine && row < a.d_k) {
            if constexpr (PASSING) __builtin_nontemporal_store(s[i], to);
            else *to = s[i];
        }
    }
    const v4f o = sum_rows(kq[1]);
    if (mine && rg == 0)
        for (int e = 0; e < 4; ++e) put_elem<DT>(a.o, ((int64_t)b * a.H + h) * a.d_v + col + e, a.scale * o[e]);
}

template <int DT, int CG> int go(const StepCall& a)
{
    constexpr int RG = THREADS / CG;
    const int groups = (a.d_v + 4 * CG - 1) / (4 * CG);
    const dim3 grid = long_grid((int64_t)a.B * a.H * groups);
    if (a.d_k <= 64) return launch_kernel(false, k_gdn_step<DT, CG, 64 / RG>, grid, dim3(THREADS), 0, a.stream, a);
    if (a.d_k <= 128) return launch_kernel(false, k_gdn_step<DT, CG, 128 / RG>, grid, dim3(THREADS), 0, a.stream, a);
    return launch_kernel(false, k_gdn_step<DT, CG, 256 / RG>, grid, dim3(THREADS), 0, a.stream, a);
}
// 32 columns a workgroup where those of 64 would leave compute units without work (16 heads of 128 x 128, bf16, in us: one sequence 4.6 and 4.6, four 5.1 and 5.4,
// eight 6.7 and 6.2, sixteen 12.0 and 8.1, 64 36 and 28; 256 of 32 heads 224 and 200, where loads and stores that stay in the caches take 215).
template <int DT> int pick(const StepCall& a) { return (int64_t)a.B * a.H * ((a.d_v + 31) / 32) < 512 ? go<DT, 8>(a) : go<DT, 16>(a); }

}  // namespace

int launch_step(const StepCall& a) { return a.dtype == OP_F32 ? pick<OP_F32>(a) : a.dtype == OP_F16 ? pick<OP_F16>(a) : pick<OP_BF16>(a); }

}  // namespace triinv
