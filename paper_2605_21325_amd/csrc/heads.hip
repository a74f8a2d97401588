// Norms of queries and keys for each head, rotated by position in the same pass.  For a head x of d elements, its weight w and a token's position p:
//     n = 1 / sqrt(mean(x^2) + eps), or 1 / sqrt(sum(x^2) + eps) (to unit length);   y = x n w
//     pairs (a, b) of the first rot elements, angle t = p f_i:   a' = a cos t - b sin t,   b' = b cos t + a sin t
// with pairs (i, i + rot / 2) or (2 i, 2 i + 1).  The gradient, with dy turned back by the same angles:
//     dx = n (dy w - x n^2 m <dy w, x>), m = 1 / d or 1;   dw = sum over tokens and heads of dy x n.
//
// Angles: p f as a part of a turn, in two 64-bit parts (positions up to 2^53 in magnitude are whole numbers there, a turn is 1 / (2 pi) to 106 bits), the part of a turn
// that is left in 32.
#include <algorithm>
#include "layer.hpp"
#include "elems.hpp"

namespace triinv {

namespace {

constexpr int WAVES = 4;  // of a workgroup
constexpr int MOST_D = 512;

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

constexpr int MOST_ANGLES = 512;  // of the tokens that a wavefront has at a time
struct Angles {
    float c[WAVES][MOST_ANGLES], s[WAVES][MOST_ANGLES];
};
struct Nothing {};

// cos and sin of the angles of tokens n to n + tokens - 1, a lane each, for the wavefront that asks; not beyond the last token.
template <class Call> __device__ __forceinline__ void turn_angles(Angles& at, int wave, const Call& a, int64_t n, int tokens)
{
#pragma clang fp contract(off)  // (what a product loses is taken apart: no product may be fused into the difference)
    const int pairs = a.rot / 2, left = (int)(a.N - n < tokens ? a.N - n : tokens);
    __builtin_amdgcn_wave_barrier();
    for (int i = threadIdx.x & 63; i < pairs * left; i += 64) {
        constexpr double TURN = 0.15915494309189535, LOW = -9.839338337591243e-18;  // 1 / (2 pi) in two parts
        const int token = tokens == 1 ? 0 : (int)((uint32_t)i / (uint32_t)pairs);
        const double p = a.pos64 ? (double)static_cast<const int64_t*>(a.positions)[n + token] : (double)static_cast<const int32_t*>(a.positions)[n + token];
        const double f = (double)a.inv_freq[i - token * pairs], t = p * f, turns = t * TURN;
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
// The slot's elements turned by the angles of its token, which are the wavefront's from `first` on; WAY = -1: back.  What is not turned stays as it is (beside an infinity too).
template <int WAY> __device__ __forceinline__ void turn_pair(float& a, float& b, float c, float s)
{
    const float t = a;
    a = t * c - b * (WAY * s), b = b * c + t * (WAY * s);
}
template <int WAY, int VEC, int ROT, class Lds> __device__ __forceinline__ void turn(float (&x)[2][VEC], const Lds& at, int wave, int first, const Slot& p, int rot, int slot)
{
    if constexpr (ROT == HALVES) {
        if (!p.turned) return;
#pragma unroll
        for (int e = 0; e < VEC; ++e) turn_pair<WAY>(x[0][e], x[1][e], at.c[wave][first + slot * VEC + e], at.s[wave][first + slot * VEC + e]);
    } else if constexpr (ROT == NEIGHBOURS) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (!p.there[j] || p.i[j] >= rot) continue;
#pragma unroll
            for (int e = 0; e < VEC / 2; ++e)
                if (p.i[j] + 2 * e < rot) turn_pair<WAY>(x[j][2 * e], x[j][2 * e + 1], at.c[wave][first + p.i[j] / 2 + e], at.s[wave][first + p.i[j] / 2 + e]);
        }
    }
}

// Queries and keys are taken by workgroups of their own.  What a wavefront has at a time, a unit: `tokens` tokens with few heads, or a part of one token's heads (parts of `per`).
// Their heads are counted on: row k of the unit is head k mod H of its token k / H.
struct HeadsPlan {
    int64_t units;
    int blocks, tokens, parts, per;
};
struct Unit {
    int64_t n;
    int first, end;
};
__device__ __forceinline__ Unit unit_of(int64_t unit, const HeadsPlan& p, int64_t N, int H)
{
    if (p.parts == 1) {
        const int64_t n = unit * p.tokens;
        return {n, 0, (int)(N - n < p.tokens ? N - n : p.tokens) * H};
    }
    const int64_t n = unit / p.parts;
    const int first = (int)(unit - n * p.parts) * p.per;
    return {n, first, first + p.per < H ? first + p.per : H};
}
__device__ __forceinline__ int token_of(int k, const HeadsPlan& p, int H) { return p.tokens == 1 ? 0 : (int)((uint32_t)k / (uint32_t)H); }

// The weight in LDS as it is.
template <int DT, class Call> __device__ __forceinline__ void stage_weight(void* lds, const void* weight, const Call& a)
{
    if (!weight) return;
    for (int i = threadIdx.x; i < a.d; i += 64 * WAVES) {
        Elems<DT, 1> e;
        e.load(weight, i);
        e.store(lds, i);
    }
    __syncthreads();
}
template <int DT, int VEC> __device__ __forceinline__ void weigh(float (&x)[VEC], const void* lds, int i)
{
    Elems<DT, VEC> w;
    w.load(lds, i);
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] *= w[e];
}
// Rows of the unit's tokens from its first one's on: a slot's pieces, `row` elements behind that.
template <int DT, int VEC> __device__ __forceinline__ void load_slot(Elems<DT, VEC> (&to)[2], const void* base, uint32_t row, const Slot& s, bool on)
{
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        to[j].clear();
        if (on && s.there[j]) to[j].load(static_cast<const char*>(base) + (row + (uint32_t)s.i[j]) * Elems<DT, 1>::SIZE, 0);
    }
}
template <int DT> __device__ __forceinline__ char* rows_of(const void* p, int64_t n, int64_t stride)
{
    return const_cast<char*>(static_cast<const char*>(p)) + n * stride * Elems<DT, 1>::SIZE;
}

// A wavefront takes 64 / G heads side by side, requested AT_ONCE of a lane at a time: sums stay within rows of lanes, and a head's pairs in one lane (two pieces a slot).  Bound by
// memory: each element is read and written once, 16 bytes a lane where rows begin on 16 bytes (VEC = 8; of fp32 twice as many).  65536 tokens of 32 heads of 128, bf16, 182 to 192 us,
// 5.6 to 5.9 TB/s; one head a wavefront, an element at a time, 535.  One token 3 us, the launch and the angles.
template <int DT, int VEC, int G, int SLOTS, int ROT> __global__ __launch_bounds__(64 * WAVES) void k_heads(HeadsCall a, HeadsPlan of_q, HeadsPlan of_k)
{
    constexpr int SIDE = 64 / G, AT_ONCE = VEC * SLOTS >= 8 ? 2 : 4;
    __shared__ std::conditional_t<ROT == STILL, Nothing, Angles> angles;
    __shared__ alignas(16) uint32_t lds[MOST_D * Elems<DT, 1>::SIZE / 4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const bool key = block >= of_q.blocks;
    if (key) block -= of_q.blocks;
    const HeadsPlan p = key ? of_k : of_q;
    const int H = key ? a.H_k : a.H;
    const void *const x_rows = key ? a.k : a.q, *const weight = key ? a.k_weight : a.q_weight;
    const int64_t stride = key ? a.k_stride : a.q_stride, out_stride = key ? a.k_out_stride : a.q_out_stride;
    if (block >= p.blocks) return;
    stage_weight<DT>(lds, weight, a);
    const int64_t unit = block * WAVES + __builtin_amdgcn_readfirstlane(wave);
    if (unit >= p.units) return;
    const Unit u0 = unit_of(unit, p, a.N, H);
    const char* const from = rows_of<DT>(x_rows, u0.n, stride);
    char* const to = rows_of<DT>(key ? a.k_out : a.q_out, u0.n, out_stride);
    Slot slots[SLOTS];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) slots[i] = slot_of<VEC, ROT>(lane % G + G * i, a.d, a.rot, a.interleaved);
    for (int k0 = u0.first; k0 < u0.end; k0 += SIDE * AT_ONCE) {
        Elems<DT, VEC> raw[AT_ONCE][SLOTS][2];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int k = k0 + SIDE * u + lane / G, token = token_of(k, p, H);
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) load_slot<DT, VEC>(raw[u][i], from, (uint32_t)token * (uint32_t)stride + (uint32_t)(k - token * H) * a.d, slots[i], k < u0.end);
        }
        if constexpr (ROT != STILL) {
            if (k0 == u0.first) turn_angles(angles, wave, a, u0.n, p.tokens);  // (behind the first requests)
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            float x[SLOTS][2][VEC], sq = 0.f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[i][j][e] = raw[u][i][j][e], sq += x[i][j][e] * x[i][j][e];
            sq = lanes_sum<G>(sq);
            const float norm = 1.f / sqrtf((a.unit ? sq : sq / (float)a.d) + a.eps);
            const int k = k0 + SIDE * u + lane / G, token = token_of(k, p, H);
            if (k >= u0.end) continue;
            const uint32_t row = (uint32_t)token * (uint32_t)out_stride + (uint32_t)(k - token * H) * a.d;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[i][j][e] *= norm;
                    if (weight) weigh<DT, VEC>(x[i][j], lds, slots[i].there[j] ? slots[i].i[j] : 0);
                }
                if constexpr (ROT != STILL) turn<1, VEC, ROT>(x[i], angles, wave, token * (a.rot / 2), slots[i], a.rot, lane % G + G * i);
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (slots[i].there[j]) store_rounded<DT, VEC>(to + (row + (uint32_t)slots[i].i[j]) * Elems<DT, 1>::SIZE, 0, x[i][j]);
            }
        }
    }
}

// The gradient, the same way; a wavefront takes units in turn, asks for its next heads before it works on those it has, and (WEIGHT) keeps its sums of the weight's gradient; those
// of a workgroup are written out and added up by k_heads_dweight, always in the same order.  Bound by memory, three rows a head: 16384 tokens of 40 heads of 128, bf16, rotated, with
// weights, 107 us (4.7 TB/s) and 5 for the sums.  122 registers, four wavefronts a SIMD: queries and keys in one wavefront's turn, which spares nothing, took 110 to 123.
template <int DT, int VEC, int G, int SLOTS, int ROT, bool WEIGHT> __global__ __launch_bounds__(64 * WAVES) void k_heads_bwd(HeadsBwdCall a, HeadsPlan of_q, HeadsPlan of_k)
{
    constexpr int SIDE = 64 / G;
    __shared__ std::conditional_t<ROT == STILL, Nothing, Angles> angles;
    __shared__ alignas(16) uint32_t lds[MOST_D * Elems<DT, 1>::SIZE / 4];
    extern __shared__ float sums[];  // [WAVES][d] (WEIGHT)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t place = block;
    const bool key = block >= of_q.blocks;
    if (key) block -= of_q.blocks;
    const HeadsPlan p = key ? of_k : of_q;
    const int H = key ? a.H_k : a.H;
    const void *const x_rows = key ? a.k : a.q, *const d_rows = key ? a.dk_out : a.dq_out, *const weight = key ? a.k_weight : a.q_weight;
    void* const out_rows = key ? a.dk : a.dq;
    const int64_t stride = key ? a.k_stride : a.q_stride, d_stride = key ? a.dk_out_stride : a.dq_out_stride, out_stride = key ? a.dk_stride : a.dq_stride;
    if (block >= p.blocks) return;
    stage_weight<DT>(lds, weight, a);
    Slot slots[SLOTS];
    float dw[WEIGHT ? SLOTS : 1][2][VEC];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        slots[i] = slot_of<VEC, ROT>(lane % G + G * i, a.d, a.rot, a.interleaved);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if constexpr (WEIGHT) dw[i][0][e] = dw[i][1][e] = 0.f;
    }
    for (int64_t unit = block * WAVES + __builtin_amdgcn_readfirstlane(wave); unit < p.units; unit += (int64_t)p.blocks * WAVES) {
        const Unit u0 = unit_of(unit, p, a.N, H);
        const char *const from = rows_of<DT>(x_rows, u0.n, stride), *const d_from = rows_of<DT>(d_rows, u0.n, d_stride);
        char* const to = rows_of<DT>(out_rows, u0.n, out_stride);
        Elems<DT, VEC> rx[SLOTS][2], rd[SLOTS][2];
        const auto request = [&](int k) {
            const int token = token_of(k, p, H);
            const uint32_t h = (uint32_t)(k - token * H) * a.d;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                load_slot<DT, VEC>(rx[i], from, (uint32_t)token * (uint32_t)stride + h, slots[i], k < u0.end);
                load_slot<DT, VEC>(rd[i], d_from, (uint32_t)token * (uint32_t)d_stride + h, slots[i], k < u0.end);
            }
        };
        request(u0.first + lane / G);
        if constexpr (ROT != STILL) turn_angles(angles, wave, a, u0.n, p.tokens);
        for (int k0 = u0.first; k0 < u0.end; k0 += SIDE) {
            const int k = k0 + lane / G, token = token_of(k, p, H);
            const bool on = k < u0.end;
            float x[SLOTS][2][VEC], z[SLOTS][2][VEC], sq = 0.f, dot = 0.f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[i][j][e] = rx[i][j][e], z[i][j][e] = rd[i][j][e], sq += x[i][j][e] * x[i][j][e];
            if (k0 + SIDE < u0.end) request(k + SIDE);
            if constexpr (ROT != STILL) {
#pragma unroll
                for (int i = 0; i < SLOTS; ++i) turn<-1, VEC, ROT>(z[i], angles, wave, (on ? token : 0) * (a.rot / 2), slots[i], a.rot, lane % G + G * i);
            }
            const float sum = lanes_sum<G>(sq), norm = 1.f / sqrtf((a.unit ? sum : sum / (float)a.d) + a.eps), counted = on ? norm : 0.f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if constexpr (WEIGHT) {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) dw[i][j][e] += z[i][j][e] * (x[i][j][e] * counted);
                    }
                    if (weight) weigh<DT, VEC>(z[i][j], lds, slots[i].there[j] ? slots[i].i[j] : 0);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) dot += z[i][j][e] * x[i][j][e];
                }
            dot = lanes_sum<G>(dot);
            const float m = (a.unit ? dot : dot / (float)a.d) * norm * norm;
            if (!on) continue;
            const uint32_t row = (uint32_t)token * (uint32_t)out_stride + (uint32_t)(k - token * H) * a.d;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (!slots[i].there[j]) continue;
                    float dx[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) dx[e] = norm * (z[i][j][e] - x[i][j][e] * m);
                    store_rounded<DT, VEC>(to + (row + (uint32_t)slots[i].i[j]) * Elems<DT, 1>::SIZE, 0, dx);
                }
        }
    }
    if constexpr (WEIGHT) {
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float t = dw[i][j][e];
                    for (int o = G; o < 64; o *= 2) t += __shfl_xor(t, o);
                    if (lane < G && slots[i].there[j]) sums[wave * a.d + slots[i].i[j] + e] = t;
                }
        __syncthreads();
        for (int c = threadIdx.x; c < a.d; c += 64 * WAVES) {
            float t = sums[c];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) t += sums[w * a.d + c];
            a.partial[place * a.d + c] = t;
        }
    }
}

// dq_weight[c] and, behind its workgroups, dk_weight[c] = sum of the groups' partial[group][c]: four columns a workgroup, 256 threads a column, in the same order every time.
__global__ __launch_bounds__(1024) void k_heads_dweight(const float* partial, float* dq, float* dk, int groups_q, int groups_k, int d)
{
    __shared__ float part[256][5];
    const bool key = blockIdx.y == 1;
    const int groups = key ? groups_k : groups_q;
    const int cx = threadIdx.x & 3, y = threadIdx.x >> 2, c = 4 * blockIdx.x + cx;
    float* const to = key ? dk : dq;
    if (!to) return;
    if (key) partial += (int64_t)groups_q * d;
    float s = 0.f;
    if (c < d) {
#pragma unroll 8
        for (int g = y; g < groups; g += 256) s += partial[(int64_t)g * d + c];
    }
    part[y][cx] = s;
    __syncthreads();
    for (int half = 128; half > 0; half /= 2) {
        if (y < half) part[y][cx] = s += part[y + half][cx];
        __syncthreads();
    }
    if (y == 0 && c < d) to[c] = s;
}

// A wavefront's unit.  Where tokens are many: as many of them as have ROWS times the heads that stand side by side, so that one's angles and addresses and the way to memory
// come once for several rows (their rows by 32-bit offsets, their angles as far as LDS has room), as long as all of `waves` have a unit (the gradient with weights: 3154 tokens of 6 heads
// of 80 18 us with a token each, 12.5 so).  Where they are few: a part of a token's heads.
constexpr int ROWS = 2;
HeadsPlan plan(int64_t N, int H, int side, int64_t stride, int pairs, int64_t waves = 2048)
{
    if (H <= 0 || N <= 0) return {0, 0, 1, 1, 1};
    const auto blocks = [](int64_t units) { return (int)((units + WAVES - 1) / WAVES); };
    int64_t tokens = std::min<int64_t>({(int64_t)ROWS * side / H, N / waves, (int64_t)(pairs ? MOST_ANGLES / pairs : 64), (1LL << 29) / std::max<int64_t>(stride, 1)});
    if (tokens * H > side && tokens * H % side < side / 2) tokens = tokens * H / side * side / H;  // (no step for a few rows)
    if (tokens > 1) {
        const int64_t units = (N + tokens - 1) / tokens;
        return {units, blocks(units), (int)tokens, 1, H};
    }
    const int64_t steps = (H + side - 1) / side, most = (2048 + N - 1) / N, wanted = most < steps ? most : steps;
    const int per = (int)((steps + wanted - 1) / wanted) * side, parts = (H + per - 1) / per;
    return {N * parts, blocks(N * parts), 1, parts, per};
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
        const HeadsPlan q = plan(a.N, a.H, 64 / G, std::max<int64_t>({a.q_stride, a.q_out_stride}), a.rot / 2), k = plan(a.N, a.H_k, 64 / G, std::max<int64_t>({a.k_stride, a.k_out_stride}), a.rot / 2);
        return launch_kernel(false, k_heads<DT, VEC, G, SLOTS, ROT>, long_grid((int64_t)q.blocks + k.blocks), dim3(64 * WAVES), 0, a.stream, a, q, k);
    }
};
template <int DT> struct Backward {
    const HeadsBwdCall& a;
    template <int VEC, int G, int SLOTS, int ROT> int go() const
    {
        const auto waves = [&](int groups) { return a.partial ? (int64_t)groups * WAVES : 2048; };
        HeadsPlan q = plan(a.N, a.H, 64 / G, std::max<int64_t>({a.q_stride, a.dq_out_stride, a.dq_stride}), a.rot / 2, waves(a.groups_q));
        HeadsPlan k = plan(a.N, a.H_k, 64 / G, std::max<int64_t>({a.k_stride, a.dk_out_stride, a.dk_stride}), a.rot / 2, waves(a.groups_k));
        if (a.partial) {
            q.blocks = a.groups_q, k.blocks = a.groups_k;
            return launch_kernel(false, k_heads_bwd<DT, VEC, G, SLOTS, ROT, true>, dim3((unsigned)(a.groups_q + a.groups_k)), dim3(64 * WAVES), WAVES * a.d * 4, a.stream, a, q, k);
        }
        return launch_kernel(false, k_heads_bwd<DT, VEC, G, SLOTS, ROT, false>, long_grid((int64_t)q.blocks + k.blocks), dim3(64 * WAVES), 0, a.stream, a, q, k);
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
    return launch_kernel(false, k_heads_dweight, dim3((unsigned)((a.d + 3) / 4), 2), dim3(1024), 0, a.stream, a.partial, a.dq_weight, a.dk_weight, a.groups_q, a.groups_k, a.d);
}

}  // namespace

// Workgroups that keep a sum each, for queries and keys together in proportion; each with sixteen rows a wavefront, 1024 of them at most, which the card holds at once, and more, up to
// 2048, from 64 rows a wavefront on (42115 tokens of two heads of 32 17.4 us with 1318, 13.1 so, with 512 14.6; 3898 of 48 22.4 with 2048, 19).  In us, both launches, with 512 / 768 / 1024 /
// 2048 / 4096 of them at most (heads of 128, bf16, rotated): 16384 tokens of 40 heads 129 / 140 / 127 / 115 / 117, 65536 of 10 182 / 172 / 153 / 131 / 130; rows a wavefront 4 / 16
// / 32 / 64: 256 tokens of 24 heads 9.5 / 10 / 13 / 20, 1024 17.8 / 13.8 / 16 / 23, 4096 31 / 29 / 26 / 30.
int heads_bwd_groups(int64_t N, int H, int heads)
{
    const int64_t n = (N * H + 16 * WAVES - 1) / (16 * WAVES), most = std::clamp<int64_t>(N * heads / (64 * WAVES), 1024, 2048), share = (most * H + heads - 1) / heads;
    return (int)(n < share ? n : share);
}
int launch_heads(const HeadsCall& a) { return a.dtype == OP_F32 ? heads<OP_F32>(a) : a.dtype == OP_F16 ? heads<OP_F16>(a) : heads<OP_BF16>(a); }
int launch_heads_bwd(const HeadsBwdCall& a) { return a.dtype == OP_F32 ? heads_bwd<OP_F32>(a) : a.dtype == OP_F16 ? heads_bwd<OP_F16>(a) : heads_bwd<OP_BF16>(a); }

}  // namespace triinv
