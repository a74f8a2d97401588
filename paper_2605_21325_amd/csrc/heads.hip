// Norms of queries and keys for each head, rotated by position in the same pass.  For a head x of d elements, its weight w and a token's position p:
//     n = 1 / sqrt(mean(x^2) + eps), or 1 / sqrt(sum(x^2) + eps) (to unit length);   y = x n w
//     pairs (a, b) of the first rot elements, angle t = p f_i:   a' = a cos t - b sin t,   b' = b cos t + a sin t
// with pairs (i, i + rot / 2) or (2 i, 2 i + 1).  The gradient, with dy turned back by the same angles:
//     dx = n (dy w - x n^2 m <dy w, x>), m = 1 / d or 1;   dw = sum over tokens and heads of dy x n.
//
// Angles: p f as a part of a turn, in two 64-bit parts (positions up to 2^53 in magnitude are whole numbers there, a turn is 1 / (2 pi) to 106 bits), the part of a turn
// that is left in 32.
#include "layer.hpp"
#include "elems.hpp"

namespace triinv {

namespace {

constexpr int WAVES = 4;  // of a workgroup
constexpr int MOST_PAIRS = 256;

__device__ __forceinline__ float lanes_sum(float x, int from, int to)
{
    for (int d = from; d < to; d *= 2) x += __shfl_xor(x, d);
    return x;
}

struct Angles {
    float c[WAVES][MOST_PAIRS], s[WAVES][MOST_PAIRS];
};

// cos and sin of a token's angles, a lane each, for the wavefront that asks.
__device__ __forceinline__ void turn_angles(Angles& at, int wave, const void* positions, bool pos64, const float* inv_freq, int pairs, int64_t n)
{
#pragma clang fp contract(off)  // (what a product loses is taken apart: no product may be fused into the difference)
    const double p = pos64 ? (double)static_cast<const int64_t*>(positions)[n] : (double)static_cast<const int32_t*>(positions)[n];
    for (int i = threadIdx.x & 63; i < pairs; i += 64) {
        constexpr double TURN = 0.15915494309189535, LOW = -9.839338337591243e-18;  // 1 / (2 pi) in two parts
        const double f = (double)inv_freq[i], t = p * f, turns = t * TURN;
        const double rest = fma(t, TURN, -turns) + fma(t, LOW, fma(p, f, -t) * TURN);
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns) + rest), &s, &c);
        at.c[wave][i] = c, at.s[wave][i] = s;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Elements of a pair: rotated ones first, then those that stay, two and two.
struct Pair {
    int i, j;  // j < 0: none
    bool turned;
};
__device__ __forceinline__ Pair pair_of(int s, int d, int rot, bool interleaved)
{
    const int r = rot / 2;
    if (s < r) return interleaved ? Pair{2 * s, 2 * s + 1, true} : Pair{s, s + r, true};
    const int i = rot + 2 * (s - r);
    return {i, i + 1 < d ? i + 1 : -1, false};
}

// A wavefront a head.
template <int DT, int SLOTS> __global__ __launch_bounds__(64 * WAVES) void k_heads(HeadsCall a)
{
    __shared__ Angles angles;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = a.H + a.H_k, pairs = (a.d + 1) / 2;
    const int64_t unit = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * WAVES + wave;
    const int64_t n = unit / heads;
    const int head = (int)(unit - n * heads);
    if (n >= a.N) return;
    const bool key = head >= a.H;
    const int64_t from = key ? n * a.k_stride + (int64_t)(head - a.H) * a.d : n * a.q_stride + (int64_t)head * a.d;
    const int64_t to = key ? n * a.k_out_stride + (int64_t)(head - a.H) * a.d : n * a.q_out_stride + (int64_t)head * a.d;
    const void *const x = key ? a.k : a.q, *const weight = key ? a.k_weight : a.q_weight;
    void* const y = key ? a.k_out : a.q_out;
    float u[SLOTS], v[SLOTS], sq = 0.f;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        const int s = lane + 64 * i;
        u[i] = v[i] = 0.f;
        if (s >= pairs) continue;
        const Pair p = pair_of(s, a.d, a.rot, a.interleaved);
        Elems<DT, 1> e;
        e.load(x, from + p.i), u[i] = e[0];
        if (p.j >= 0) e.load(x, from + p.j), v[i] = e[0];
        sq += u[i] * u[i] + v[i] * v[i];
    }
    if (a.rot) turn_angles(angles, wave, a.positions, a.pos64, a.inv_freq, a.rot / 2, n);
    sq = lanes_sum(sq, 1, 64);
    const float norm = 1.f / sqrtf((a.unit ? sq : sq / (float)a.d) + a.eps);
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        const int s = lane + 64 * i;
        if (s >= pairs) continue;
        const Pair p = pair_of(s, a.d, a.rot, a.interleaved);
        float b[1] = {u[i] * norm}, c[1] = {v[i] * norm};
        if (weight) {
            Elems<DT, 1> w;
            w.load(weight, p.i), b[0] *= w[0];
            if (p.j >= 0) w.load(weight, p.j), c[0] *= w[0];
        }
        if (p.turned) {
            const float co = angles.c[wave][s], si = angles.s[wave][s], t = b[0];
            b[0] = t * co - c[0] * si, c[0] = c[0] * co + t * si;
        }
        store_rounded<DT, 1>(y, to + p.i, b);
        if (p.j >= 0) store_rounded<DT, 1>(y, to + p.j, c);
    }
}

// The gradient: a wavefront takes tokens in turn, all heads of each, and keeps its sums of the weights' gradients; those of a workgroup are written out and
// added up by k_heads_dweight, always in the same order.
template <int DT, int SLOTS> __global__ __launch_bounds__(64 * WAVES) void k_heads_bwd(HeadsBwdCall a)
{
    __shared__ Angles angles;
    __shared__ float sums[WAVES][2 * 2 * MOST_PAIRS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = a.H + a.H_k, pairs = (a.d + 1) / 2;
    float dw[2][SLOTS][2] = {};
    for (int64_t n = (int64_t)blockIdx.x * WAVES + wave; n < a.N; n += (int64_t)gridDim.x * WAVES) {
        if (a.rot) turn_angles(angles, wave, a.positions, a.pos64, a.inv_freq, a.rot / 2, n);
        for (int head = 0; head < heads; ++head) {
            const bool key = head >= a.H;
            const int64_t h = (int64_t)(key ? head - a.H : head) * a.d;
            const int64_t at = n * (key ? a.k_stride : a.q_stride) + h, up = n * (key ? a.dk_out_stride : a.dq_out_stride) + h, to = n * (key ? a.dk_stride : a.dq_stride) + h;
            const void *const x = key ? a.k : a.q, *const dy = key ? a.dk_out : a.dq_out, *const weight = key ? a.k_weight : a.q_weight;
            float u[SLOTS][2], e[SLOTS][2], f[SLOTS][2], sq = 0.f, dot = 0.f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                const int s = lane + 64 * i;
                u[i][0] = u[i][1] = e[i][0] = e[i][1] = f[i][0] = f[i][1] = 0.f;
                if (s >= pairs) continue;
                const Pair p = pair_of(s, a.d, a.rot, a.interleaved);
                Elems<DT, 1> r;
                r.load(x, at + p.i), u[i][0] = r[0];
                r.load(dy, up + p.i), e[i][0] = r[0];
                if (p.j >= 0) r.load(x, at + p.j), u[i][1] = r[0];
                if (p.j >= 0) r.load(dy, up + p.j), e[i][1] = r[0];
                if (p.turned) {
                    const float co = angles.c[wave][s], si = angles.s[wave][s], t = e[i][0];
                    e[i][0] = t * co + e[i][1] * si, e[i][1] = e[i][1] * co - t * si;
                }
                f[i][0] = e[i][0], f[i][1] = e[i][1];
                if (weight) {
                    r.load(weight, p.i), f[i][0] *= r[0];
                    if (p.j >= 0) r.load(weight, p.j), f[i][1] *= r[0];
                }
                sq += u[i][0] * u[i][0] + u[i][1] * u[i][1];
                dot += f[i][0] * u[i][0] + f[i][1] * u[i][1];
            }
            sq = lanes_sum(sq, 1, 64), dot = lanes_sum(dot, 1, 64);
            const float norm = 1.f / sqrtf((a.unit ? sq : sq / (float)a.d) + a.eps), m = (a.unit ? dot : dot / (float)a.d) * norm * norm;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                const int s = lane + 64 * i;
                if (s >= pairs) continue;
                const Pair p = pair_of(s, a.d, a.rot, a.interleaved);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    dw[0][i][j] += key ? 0.f : e[i][j] * (u[i][j] * norm);
                    dw[1][i][j] += key ? e[i][j] * (u[i][j] * norm) : 0.f;
                    const float dx[1] = {norm * (f[i][j] - u[i][j] * m)};
                    if (j == 0 || p.j >= 0) store_rounded<DT, 1>(key ? a.dk : a.dq, to + (j ? p.j : p.i), dx);
                }
            }
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        const int s = lane + 64 * i;
        if (s >= pairs) continue;
        const Pair p = pair_of(s, a.d, a.rot, a.interleaved);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            sums[wave][k * a.d + p.i] = dw[k][i][0];
            if (p.j >= 0) sums[wave][k * a.d + p.j] = dw[k][i][1];
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.d; c += 64 * WAVES) {
        float t = sums[0][c];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) t += sums[w][c];
        a.partial[(int64_t)blockIdx.x * 2 * a.d + c] = t;
    }
}

// Column c of [dq_weight, dk_weight] = sum of partial[group][c]: 16 columns a workgroup, 64 threads a column, in the same order every time.
__global__ __launch_bounds__(1024) void k_heads_dweight(const float* partial, float* dq, float* dk, int groups, int d)
{
    __shared__ float part[64][17];
    const int cx = threadIdx.x & 15, y = threadIdx.x >> 4, c = 16 * blockIdx.x + cx;
    float s = 0.f;
    if (c < 2 * d) {
#pragma unroll 8
        for (int g = y; g < groups; g += 64) s += partial[(int64_t)g * 2 * d + c];
    }
    part[y][cx] = s;
    __syncthreads();
    for (int half = 32; half > 0; half /= 2) {
        if (y < half) part[y][cx] = s += part[y + half][cx];
        __syncthreads();
    }
    float* const to = c < d ? dq : dk;
    if (y == 0 && c < 2 * d && to) to[c < d ? c : c - d] = s;
}

template <int DT> int heads(const HeadsCall& a)
{
    const dim3 grid = long_grid((a.N * (a.H + a.H_k) + WAVES - 1) / WAVES), block(64 * WAVES);
    if (a.d <= 128) return launch_kernel(false, k_heads<DT, 1>, grid, block, 0, a.stream, a);
    if (a.d <= 256) return launch_kernel(false, k_heads<DT, 2>, grid, block, 0, a.stream, a);
    return launch_kernel(false, k_heads<DT, 4>, grid, block, 0, a.stream, a);
}
template <int DT> int heads_bwd(const HeadsBwdCall& a)
{
    int rc = LAUNCHED;
    if (a.groups > 0) {
        const dim3 grid((unsigned)a.groups), block(64 * WAVES);
        rc = a.d <= 128   ? launch_kernel(false, k_heads_bwd<DT, 1>, grid, block, 0, a.stream, a)
             : a.d <= 256 ? launch_kernel(false, k_heads_bwd<DT, 2>, grid, block, 0, a.stream, a)
                          : launch_kernel(false, k_heads_bwd<DT, 4>, grid, block, 0, a.stream, a);
    }
    if (rc != LAUNCHED || (!a.dq_weight && !a.dk_weight)) return rc;
    return launch_kernel(false, k_heads_dweight, dim3((unsigned)((2 * a.d + 15) / 16)), dim3(1024), 0, a.stream, a.partial, a.dq_weight, a.dk_weight, a.groups, a.d);
}

}  // namespace

int heads_bwd_groups(int64_t N, int, int, int)
{
    const int64_t n = (N + WAVES - 1) / WAVES;
    return (int)(n < 1024 ? n : 1024);
}
int launch_heads(const HeadsCall& a) { return a.dtype == OP_F32 ? heads<OP_F32>(a) : a.dtype == OP_F16 ? heads<OP_F16>(a) : heads<OP_BF16>(a); }
int launch_heads_bwd(const HeadsBwdCall& a) { return a.dtype == OP_F32 ? heads_bwd<OP_F32>(a) : a.dtype == OP_F16 ? heads_bwd<OP_F16>(a) : heads_bwd<OP_BF16>(a); }

}  // namespace triinv
