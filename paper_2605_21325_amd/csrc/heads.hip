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

// A neighbour's value, within a row of sixteen lanes.
template <int CTRL> __device__ __forceinline__ float from_lane(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// The sum over G neighbouring lanes, in all of them; the same order in each.
template <int G> __device__ __forceinline__ float lanes_sum(float x)
{
    if constexpr (G > 1) x += from_lane<0xb1>(x);   // lane ^ 1
    if constexpr (G > 2) x += from_lane<0x4e>(x);   // lane ^ 2
    if constexpr (G > 4) x += from_lane<0x141>(x);  // 7 - lane of eight
    if constexpr (G > 8) x += from_lane<0x140>(x);  // 15 - lane of sixteen
    if constexpr (G > 16) x += __shfl_xor(x, 16);
    if constexpr (G > 32) x += __shfl_xor(x, 32);
    return x;
}

struct Angles {
    float c[WAVES][MOST_PAIRS], s[WAVES][MOST_PAIRS];
};
struct NoAngles {};

// cos and sin of a token's angles, a lane each, for the wavefront that asks.
__device__ __forceinline__ void turn_angles(Angles& at, int wave, const void* positions, bool pos64, const float* inv_freq, int pairs, int64_t n)
{
#pragma clang fp contract(off)  // (what a product loses is taken apart: no product may be fused into the difference)
    __builtin_amdgcn_wave_barrier();
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

// A head lies in pieces of VEC elements, two to a slot, SLOTS slots a lane of the G that share it.  HALVES: what is rotated first, a piece and the one rot / 2 elements behind it
// (or, of single elements, its neighbour); then the rest, in two halves.  NEIGHBOURS: pairs lie inside a piece.
enum : int { STILL = 0, HALVES = 1, NEIGHBOURS = 2 };
struct Slot {
    int i[2];     // first elements of its pieces
    bool there[2];
    bool turned;  // (HALVES)
};
template <int VEC, int ROT> __device__ __forceinline__ Slot slot_of(int s, int d, int rot, bool interleaved)
{
    const int pieces = d / VEC, first = ROT == HALVES ? rot / 2 / VEC : 0;  // turned slots
    if (ROT == HALVES && s < first) {
        if (VEC == 1 && interleaved) return {{2 * s, 2 * s + 1}, {true, true}, true};
        return {{s * VEC, s * VEC + rot / 2}, {true, true}, true};
    }
    const int rest = pieces - 2 * first, half = (rest + 1) / 2, r = s - first, i = 2 * first + r;
    return {{i * VEC, (i + half) * VEC}, {r < half, r < half && r + half < rest}, false};
}
// cos and sin for the pairs of a slot.
template <int VEC, int ROT> struct Turn {
    float c[ROT == STILL ? 1 : VEC], s[ROT == STILL ? 1 : VEC];
    __device__ __forceinline__ void load(const Angles& at, int wave, const Slot& p, int rot, int slot)
    {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if constexpr (ROT == HALVES) {
                c[e] = p.turned ? at.c[wave][slot * VEC + e] : 1.f, s[e] = p.turned ? at.s[wave][slot * VEC + e] : 0.f;
            } else if constexpr (ROT == NEIGHBOURS) {
                const int i = p.i[e / (VEC / 2)] / 2 + e % (VEC / 2);
                const bool on = p.there[e / (VEC / 2)] && 2 * i < rot;
                c[e] = on ? at.c[wave][i] : 1.f, s[e] = on ? at.s[wave][i] : 0.f;
            }
        }
    }
    // The slot's elements turned; WAY = -1: back.  What is not turned stays as it is (an infinity beside it too).
    template <int WAY> __device__ __forceinline__ void turn(float (&x)[2][VEC]) const
    {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if constexpr (ROT == STILL) continue;
            float& a = ROT == HALVES ? x[0][e] : x[e / (VEC / 2 ? VEC / 2 : 1)][2 * (e % (VEC / 2 ? VEC / 2 : 1))];
            float& b = ROT == HALVES ? x[1][e] : x[e / (VEC / 2 ? VEC / 2 : 1)][2 * (e % (VEC / 2 ? VEC / 2 : 1)) + 1 < VEC ? 2 * (e % (VEC / 2 ? VEC / 2 : 1)) + 1 : 0];
            const float t = a, sn = WAY * s[e];
            const bool on = s[e] != 0.f || c[e] != 1.f;
            a = on ? t * c[e] - b * sn : t, b = on ? b * c[e] + t * sn : b;
        }
    }
};

// Heads [first, end) of a token for one wavefront.
struct Part {
    int64_t n;
    int first, end;
};
__device__ __forceinline__ Part part_of(int64_t unit, int parts, int per, int heads)
{
    const int64_t n = unit / parts;
    const int first = (int)(unit - n * parts) * per;
    return {n, first, first + per < heads ? first + per : heads};
}
struct HeadsPlan {
    int64_t units;   // N parts
    int parts, per;  // of a token's heads; heads of a part
};

// A wavefront takes a part of a token's heads, 64 / G side by side; rows are requested AT_ONCE heads of a lane at a time.  Bound by memory: each element is read and written once,
// 16 bytes a lane where rows begin on 16 bytes (VEC = 8; of fp32 twice as many).
template <int DT, int VEC, int G, int SLOTS, int ROT> __global__ __launch_bounds__(64 * WAVES) void k_heads(HeadsCall a, HeadsPlan p)
{
    constexpr int SIDE = 64 / G, AT_ONCE = VEC * SLOTS >= 8 ? 2 : 4;
    __shared__ std::conditional_t<ROT == STILL, NoAngles, Angles> angles;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = a.H + a.H_k;
    const int64_t unit = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * WAVES + __builtin_amdgcn_readfirstlane(wave);
    if (unit >= p.units) return;
    const Part part = part_of(unit, p.parts, p.per, heads);
    const int64_t n = part.n;
    Slot slots[SLOTS];
    Elems<DT, VEC> w[2][SLOTS][2];  // of queries and keys
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        slots[i] = slot_of<VEC, ROT>(lane % G + G * i, a.d, a.rot, a.interleaved);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            w[0][i][j].clear(), w[1][i][j].clear();
            if (a.q_weight && slots[i].there[j]) w[0][i][j].load(a.q_weight, slots[i].i[j]);
            if (a.k_weight && slots[i].there[j]) w[1][i][j].load(a.k_weight, slots[i].i[j]);
        }
    }
    Turn<VEC, ROT> turn[SLOTS];
    for (int h0 = part.first + lane / G; __any(h0 < part.end); h0 += SIDE * AT_ONCE) {
        Elems<DT, VEC> raw[AT_ONCE][SLOTS][2];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int head = h0 + SIDE * u;
            const bool key = head >= a.H;
            const int64_t from = key ? n * a.k_stride + (int64_t)(head - a.H) * a.d : n * a.q_stride + (int64_t)head * a.d;
            const void* const x = key ? a.k : a.q;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    raw[u][i][j].clear();
                    if (head < part.end && slots[i].there[j]) raw[u][i][j].load(x, from + slots[i].i[j]);
                }
        }
        if constexpr (ROT != STILL) {
            if (h0 < part.first + SIDE) {  // (behind the first requests)
                turn_angles(angles, wave, a.positions, a.pos64, a.inv_freq, a.rot / 2, n);
#pragma unroll
                for (int i = 0; i < SLOTS; ++i) turn[i].load(angles, wave, slots[i], a.rot, lane % G + G * i);
            }
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int head = h0 + SIDE * u;
            const bool key = head >= a.H, weighted = key ? a.k_weight != nullptr : a.q_weight != nullptr;
            float x[SLOTS][2][VEC], sq = 0.f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[i][j][e] = raw[u][i][j][e], sq += x[i][j][e] * x[i][j][e];
            sq = lanes_sum<G>(sq);
            const float norm = 1.f / sqrtf((a.unit ? sq : sq / (float)a.d) + a.eps);
            if (head >= part.end) continue;
            const int64_t to = key ? n * a.k_out_stride + (int64_t)(head - a.H) * a.d : n * a.q_out_stride + (int64_t)head * a.d;
            void* const y = key ? a.k_out : a.q_out;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    Elems<DT, VEC> v;
#pragma unroll
                    for (int k = 0; k < Elems<DT, VEC>::WORDS; ++k) {
                        const uint32_t of_q = w[0][i][j].w[k], of_k = w[1][i][j].w[k];
                        v.w[k] = key ? of_k : of_q;
                    }
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[i][j][e] *= norm, x[i][j][e] *= weighted ? v[e] : 1.f;
                }
                turn[i].template turn<1>(x[i]);
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (slots[i].there[j]) store_rounded<DT, VEC>(y, to + slots[i].i[j], x[i][j]);
            }
        }
    }
}

// The gradient, the same way; a wavefront takes parts in turn and keeps its sums of the weights' gradients; those of a workgroup are written out and added up by k_heads_dweight,
// always in the same order.
template <int DT, int VEC, int G, int SLOTS, int ROT> __global__ __launch_bounds__(64 * WAVES) void k_heads_bwd(HeadsBwdCall a, HeadsPlan p)
{
    constexpr int SIDE = 64 / G;
    __shared__ std::conditional_t<ROT == STILL, NoAngles, Angles> angles;
    extern __shared__ float sums[];  // [WAVES][2 d] where weights' gradients are asked for
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = a.H + a.H_k;
    Slot slots[SLOTS];
    Elems<DT, VEC> w[2][SLOTS][2];
    float dw[2][SLOTS][2][VEC];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        slots[i] = slot_of<VEC, ROT>(lane % G + G * i, a.d, a.rot, a.interleaved);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) dw[0][i][j][e] = dw[1][i][j][e] = 0.f;
            w[0][i][j].clear(), w[1][i][j].clear();
            if (a.q_weight && slots[i].there[j]) w[0][i][j].load(a.q_weight, slots[i].i[j]);
            if (a.k_weight && slots[i].there[j]) w[1][i][j].load(a.k_weight, slots[i].i[j]);
        }
    }
    Turn<VEC, ROT> turn[SLOTS];
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, blocks = (int64_t)gridDim.y * gridDim.x;
    for (int64_t unit = block * WAVES + __builtin_amdgcn_readfirstlane(wave); unit < p.units; unit += blocks * WAVES) {
        const Part part = part_of(unit, p.parts, p.per, heads);
        const int64_t n = part.n;
        for (int h0 = part.first + lane / G; __any(h0 < part.end); h0 += SIDE) {
            const int head = h0;
            const bool key = head >= a.H, on = head < part.end, weighted = key ? a.k_weight != nullptr : a.q_weight != nullptr;
            const int64_t h = (int64_t)(key ? head - a.H : head) * a.d;
            Elems<DT, VEC> rx[SLOTS][2], rd[SLOTS][2];
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    rx[i][j].clear(), rd[i][j].clear();
                    if (!on || !slots[i].there[j]) continue;
                    rx[i][j].load(key ? a.k : a.q, n * (key ? a.k_stride : a.q_stride) + h + slots[i].i[j]);
                    rd[i][j].load(key ? a.dk_out : a.dq_out, n * (key ? a.dk_out_stride : a.dq_out_stride) + h + slots[i].i[j]);
                }
            if constexpr (ROT != STILL) {
                if (h0 < part.first + SIDE) {
                    turn_angles(angles, wave, a.positions, a.pos64, a.inv_freq, a.rot / 2, n);
#pragma unroll
                    for (int i = 0; i < SLOTS; ++i) turn[i].load(angles, wave, slots[i], a.rot, lane % G + G * i);
                }
            }
            float x[SLOTS][2][VEC], z[SLOTS][2][VEC], sq = 0.f, dot = 0.f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[i][j][e] = rx[i][j][e], z[i][j][e] = rd[i][j][e], sq += x[i][j][e] * x[i][j][e];
                turn[i].template turn<-1>(z[i]);
            }
            const float sum = lanes_sum<G>(sq), norm = 1.f / sqrtf((a.unit ? sum : sum / (float)a.d) + a.eps);
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    Elems<DT, VEC> v;
#pragma unroll
                    for (int k = 0; k < Elems<DT, VEC>::WORDS; ++k) {
                        const uint32_t of_q = w[0][i][j].w[k], of_k = w[1][i][j].w[k];
                        v.w[k] = key ? of_k : of_q;
                    }
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float t = z[i][j][e] * (x[i][j][e] * norm);
                        if (on && key) dw[1][i][j][e] += t;
                        if (on && !key) dw[0][i][j][e] += t;
                        z[i][j][e] *= weighted ? v[e] : 1.f;
                        dot += z[i][j][e] * x[i][j][e];
                    }
                }
            dot = lanes_sum<G>(dot);
            const float m = (a.unit ? dot : dot / (float)a.d) * norm * norm;
            if (!on) continue;
            const int64_t to = n * (key ? a.dk_stride : a.dq_stride) + h;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (!slots[i].there[j]) continue;
                    float dx[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) dx[e] = norm * (z[i][j][e] - x[i][j][e] * m);
                    store_rounded<DT, VEC>(key ? a.dk : a.dq, to + slots[i].i[j], dx);
                }
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float t = dw[k][i][j][e];
                    for (int o = G; o < 64; o *= 2) t += __shfl_xor(t, o);
                    if (lane < G && slots[i].there[j]) sums[wave * 2 * a.d + k * a.d + slots[i].i[j] + e] = t;
                }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.d; c += 64 * WAVES) {
        float t = sums[c];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) t += sums[w * 2 * a.d + c];
        a.partial[block * 2 * a.d + c] = t;
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

// A wavefront's part of a token: all its heads where tokens are many, as few as stand side by side where they are few.
HeadsPlan plan(int64_t N, int heads, int side)
{
    const int64_t steps = (heads + side - 1) / side, wanted = N > 0 ? (2048 + N - 1) / N : 1;
    const int per = (int)((steps + (wanted < steps ? wanted : steps) - 1) / (wanted < steps ? wanted : steps)) * side, parts = (heads + per - 1) / per;
    return {N * parts, parts, per};
}
// Elements of a piece: what all rows and weights allow.
template <class... P> int piece(int d, int rot, bool interleaved, int size, std::initializer_list<int64_t> strides, P... pointers)
{
    for (const int v : {8, 2}) {
        bool good = d % v == 0 && (interleaved || rot % (2 * v) == 0);
        for (const int64_t s : strides) good = good && s % v == 0;
        for (const void* p : {static_cast<const void*>(pointers)...}) good = good && reinterpret_cast<uintptr_t>(p) % (v * size < 16 ? v * size : 16) == 0;
        if (good) return v;
    }
    return 1;
}

// f with the piece, the lanes of a head and the slots of a lane as its template's arguments: slots of two pieces each.
template <int ROT, class F> int shapes(int vec, int d, F f)
{
    if (vec == 8) return d <= 64 ? f.template go<8, 4, 1, ROT>() : d <= 128 ? f.template go<8, 8, 1, ROT>() : d <= 256 ? f.template go<8, 16, 1, ROT>() : f.template go<8, 32, 1, ROT>();
    if (vec == 2) return d <= 64 ? f.template go<2, 16, 1, ROT>() : d <= 256 ? f.template go<2, 64, 1, ROT>() : f.template go<2, 64, 2, ROT>();
    constexpr int R = ROT == NEIGHBOURS ? HALVES : ROT;  // (pairs of single elements are slots either way)
    return d <= 32 ? f.template go<1, 16, 1, R>() : d <= 128 ? f.template go<1, 64, 1, R>() : f.template go<1, 64, 4, R>();
}
template <class F> int rotations(int rot, bool interleaved, int vec, int d, F f)
{
    return rot == 0 ? shapes<STILL>(vec, d, f) : interleaved ? shapes<NEIGHBOURS>(vec, d, f) : shapes<HALVES>(vec, d, f);
}

template <int DT> struct Forward {
    const HeadsCall& a;
    template <int VEC, int G, int SLOTS, int ROT> int go() const
    {
        const HeadsPlan p = plan(a.N, a.H + a.H_k, 64 / G);
        return launch_kernel(false, k_heads<DT, VEC, G, SLOTS, ROT>, long_grid((p.units + WAVES - 1) / WAVES), dim3(64 * WAVES), 0, a.stream, a, p);
    }
};
template <int DT> struct Backward {
    const HeadsBwdCall& a;
    template <int VEC, int G, int SLOTS, int ROT> int go() const
    {
        const HeadsPlan p = plan(a.N, a.H + a.H_k, 64 / G);
        const dim3 grid = a.partial ? dim3((unsigned)a.groups) : long_grid((p.units + WAVES - 1) / WAVES);
        return launch_kernel(false, k_heads_bwd<DT, VEC, G, SLOTS, ROT>, grid, dim3(64 * WAVES), a.partial ? WAVES * 2 * a.d * 4 : 0, a.stream, a, p);
    }
};
template <int DT> int heads(const HeadsCall& a)
{
    const int vec = piece(a.d, a.rot, a.interleaved, DT == OP_F32 ? 4 : 2, {a.q_stride, a.k_stride, a.q_out_stride, a.k_out_stride}, a.q, a.k, a.q_out, a.k_out, a.q_weight, a.k_weight);
    return rotations(a.rot, a.interleaved, vec, a.d, Forward<DT>{a});
}
template <int DT> int heads_bwd(const HeadsBwdCall& a)
{
    int rc = LAUNCHED;
    if (a.N > 0) {
        const int vec = piece(a.d, a.rot, a.interleaved, DT == OP_F32 ? 4 : 2, {a.q_stride, a.k_stride, a.dq_out_stride, a.dk_out_stride, a.dq_stride, a.dk_stride}, a.q, a.k, a.dq_out, a.dk_out,
                              a.dq, a.dk, a.q_weight, a.k_weight);
        rc = rotations(a.rot, a.interleaved, vec, a.d, Backward<DT>{a});
    }
    if (rc != LAUNCHED || (!a.dq_weight && !a.dk_weight)) return rc;
    return launch_kernel(false, k_heads_dweight, dim3((unsigned)((2 * a.d + 15) / 16)), dim3(1024), 0, a.stream, a.partial, a.dq_weight, a.dk_weight, a.groups, a.d);
}

}  // namespace

int heads_bwd_groups(int64_t N, int H, int H_k, int)
{
    const int64_t n = (N * (H + H_k) + 4 * WAVES - 1) / (4 * WAVES);
    return (int)(n < 1024 ? n : 1024);
}
int launch_heads(const HeadsCall& a) { return a.dtype == OP_F32 ? heads<OP_F32>(a) : a.dtype == OP_F16 ? heads<OP_F16>(a) : heads<OP_BF16>(a); }
int launch_heads_bwd(const HeadsBwdCall& a) { return a.dtype == OP_F32 ? heads_bwd<OP_F32>(a) : a.dtype == OP_F16 ? heads_bwd<OP_F16>(a) : heads_bwd<OP_BF16>(a); }

}  // namespace triinv
